// C ABI of the cache operators (include/cobs_cache.h): argument validation and
// parameter blocks.  Every entry point validates on the host before it enqueues
// anything, never synchronises and keeps nothing.
#include <math.h>

#include "cache_kernels.h"
#include "cobs_cache.h"

using namespace cobs;

namespace {

static_assert(kMaxQueries == COBS_MAX_QUERIES, "the header's bound");

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

cobs_status_t hip_status(hipError_t e) { return e == hipSuccess ? COBS_OK : COBS_ERR_HIP; }

// The fields of cobs_config_t that these calls read, with the decode path's limits.
cobs_status_t check_shape(const cobs_config_t* c) {
  if (!c) return COBS_ERR_INVALID_ARG;
  if (c->batch < 1 || c->num_kv_heads < 1 || c->num_q_heads < 1) return COBS_ERR_INVALID_ARG;
  if (c->num_q_heads % c->num_kv_heads != 0) return COBS_ERR_INVALID_ARG;
  if (c->head_dim < 1 || c->block_size < 1 || c->max_seq_len < 1) return COBS_ERR_INVALID_ARG;
  if (c->budget < 0 || c->window < 0) return COBS_ERR_INVALID_ARG;
  if (c->kv_dtype != COBS_F32 && c->kv_dtype != COBS_BF16) return COBS_ERR_INVALID_ARG;
  if (!(c->softmax_scale >= 0.0f) || !isfinite(c->softmax_scale)) return COBS_ERR_INVALID_ARG;
  if (c->max_seq_len % c->block_size != 0) return COBS_ERR_INVALID_ARG;
  const int g = c->num_q_heads / c->num_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8 && g != 16) return COBS_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return COBS_ERR_UNSUPPORTED;
  if (c->block_size != 32 && c->block_size != 64 && c->block_size != 128) return COBS_ERR_UNSUPPORTED;
  if (c->max_seq_len / c->block_size > kMaxBlocksPerSeq) return COBS_ERR_UNSUPPORTED;
  // grid dimensions, and row indices of 32 bits
  if (c->batch > 65535 || c->num_kv_heads > 65535 || (int64_t)c->batch * c->num_q_heads > (1 << 22))
    return COBS_ERR_UNSUPPORTED;
  return COBS_OK;
}

cobs_status_t check_cache(const cobs_config_t* c, const cobs_kv_t* kv) {
  if (!kv || !kv->k || !kv->v || !aligned(kv->k, 16) || !aligned(kv->v, 16)) return COBS_ERR_INVALID_ARG;
  if (kv->block_table) return kv->num_pages < 1 ? COBS_ERR_INVALID_ARG : COBS_OK;
  const int64_t vec = c->kv_dtype == COBS_F32 ? 4 : 8;      // elements of 16 bytes
  if (kv->stride_t < c->head_dim || kv->stride_h < 0 || kv->stride_b < 0) return COBS_ERR_INVALID_ARG;
  if (kv->stride_t % vec || kv->stride_h % vec || kv->stride_b % vec) return COBS_ERR_INVALID_ARG;
  if (kv->stride_t > (int64_t)1 << 22) return COBS_ERR_UNSUPPORTED;
  return COBS_OK;
}

int log2_of(int block_size) { return block_size == 32 ? 5 : (block_size == 64 ? 6 : 7); }

KvView view_of(const cobs_config_t* c, const cobs_kv_t* kv, int capacity) {
  KvView x;
  x.k = kv->k;
  x.v = kv->v;
  x.sb = kv->stride_b;
  x.sh = kv->stride_h;
  x.st = kv->stride_t;
  x.table = kv->block_table;
  x.num_pages = kv->num_pages;
  x.nbmax = capacity / c->block_size;
  x.hkv = c->num_kv_heads;
  x.d = c->head_dim;
  x.lsh = log2_of(c->block_size);
  return x;
}

void shape_of(const cobs_config_t* c, int32_t num_queries, AttendParams* a) {
  a->B = c->batch;
  a->hkv = c->num_kv_heads;
  a->hq = c->num_q_heads;
  a->G = a->hq / a->hkv;
  a->N = num_queries;
  a->d = c->head_dim;
  a->tmax = c->max_seq_len;
  a->s = c->budget;
  a->w = c->window;
  a->lsh = log2_of(c->block_size);
  a->kv_f32 = c->kv_dtype == COBS_F32;
  a->c = c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
}

// The arguments that cobs_tree_decode and cobs_attention_weights share.
cobs_status_t attend_params(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                            const cobs_kv_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                            const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, AttendParams* a) {
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache(cfg, kv)) != COBS_OK) return s;
  if (num_queries < 1) return COBS_ERR_INVALID_ARG;
  if (num_queries > kMaxQueries) return COBS_ERR_UNSUPPORTED;
  if (io_dtype != COBS_F32 && io_dtype != COBS_BF16) return COBS_ERR_INVALID_ARG;
  if (!q || !aligned(q, 16) || !seq_lens) return COBS_ERR_INVALID_ARG;
  if ((draft_lens == nullptr) != (tree_mask == nullptr) || !aligned(tree_mask, 8)) return COBS_ERR_INVALID_ARG;
  if (sparse != 0 && sparse != 1) return COBS_ERR_INVALID_ARG;
  if (sparse ? (!sel && cfg->budget > 0) : sel != nullptr) return COBS_ERR_INVALID_ARG;
  shape_of(cfg, num_queries, a);
  a->kv = view_of(cfg, kv, cfg->max_seq_len);
  a->q = q;
  a->seq_lens = seq_lens;
  a->draft_lens = draft_lens;
  a->mask = tree_mask;
  a->sel = sel;
  a->sparse = sparse;
  a->io_bf16 = io_dtype == COBS_BF16;
  return COBS_OK;
}

}  // namespace

extern "C" {

size_t cobs_tree_workspace_bytes(const cobs_config_t* cfg, int32_t num_queries) {
  if (check_shape(cfg) != COBS_OK || num_queries < 1 || num_queries > kMaxQueries) return 0;
  AttendParams a = {};
  shape_of(cfg, num_queries, &a);
  return tree_workspace(a);
}

cobs_status_t cobs_tree_decode(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                               const cobs_kv_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                               const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, void* out, float* lse,
                               void* ws, size_t ws_bytes, void* stream) {
  TreeParams p = {};
  const cobs_status_t s = attend_params(cfg, q, io_dtype, num_queries, kv, seq_lens, draft_lens, tree_mask, sparse, sel,
                                        &p.a);
  if (s != COBS_OK) return s;
  if (!out || !aligned(out, 16) || out == q) return COBS_ERR_INVALID_ARG;
  const size_t need = tree_workspace(p.a);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 256))) return COBS_ERR_WORKSPACE;
  p.out = out;
  p.lse = lse;
  p.part_ml = static_cast<float*>(ws);
  return hip_status(launch_tree(p, static_cast<hipStream_t>(stream)));
}

cobs_status_t cobs_attention_weights(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype,
                                     int32_t num_queries, const cobs_kv_t* kv, const int32_t* seq_lens,
                                     const int32_t* draft_lens, const uint64_t* tree_mask, int32_t sparse,
                                     const int32_t* sel, const float* lse, const float* prev, float* weights,
                                     void* stream) {
  WeightsParams p = {};
  const cobs_status_t s = attend_params(cfg, q, io_dtype, num_queries, kv, seq_lens, draft_lens, tree_mask, sparse, sel,
                                        &p.a);
  if (s != COBS_OK) return s;
  if (!lse || !weights) return COBS_ERR_INVALID_ARG;
  p.lse = lse;
  p.prev = prev;
  p.weights = weights;
  return hip_status(launch_weights(p, static_cast<hipStream_t>(stream)));
}

size_t cobs_evict_workspace_bytes(const cobs_config_t* cfg) {
  return check_shape(cfg) == COBS_OK ? evict_workspace(cfg->batch, cfg->num_kv_heads, cfg->max_seq_len) : 0;
}

cobs_status_t cobs_evict(const cobs_config_t* cfg, const float* weights, const int32_t* seq_lens, int32_t keep,
                         int32_t sinks, int32_t recent, int32_t* kept, int32_t* new_lens, void* ws, size_t ws_bytes,
                         void* stream) {
  const cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if (!weights || !seq_lens || !kept || new_lens == seq_lens) return COBS_ERR_INVALID_ARG;
  if (keep < 1 || keep > cfg->max_seq_len || sinks < 0 || recent < 0 || sinks > keep || recent > keep - sinks)
    return COBS_ERR_INVALID_ARG;
  const size_t bytes = cobs_evict_workspace_bytes(cfg);
  if (bytes > 0 && (!ws || ws_bytes < bytes || !aligned(ws, 256))) return COBS_ERR_WORKSPACE;
  EvictParams p = {};
  p.hist = static_cast<uint16_t*>(ws);
  p.weights = weights;
  p.seq_lens = seq_lens;
  p.kept = kept;
  p.new_lens = new_lens;
  p.B = cfg->batch;
  p.hkv = cfg->num_kv_heads;
  p.tmax = cfg->max_seq_len;
  p.keep = keep;
  p.sinks = sinks;
  p.recent = recent;
  return hip_status(launch_evict(p, static_cast<hipStream_t>(stream)));
}

cobs_status_t cobs_compact_cache(const cobs_config_t* cfg, const cobs_kv_t* kv, const int32_t* kept, int32_t per_head,
                                 int32_t num_kept, const int32_t* seq_lens, const int32_t* first,
                                 const cobs_kv_t* dst, int32_t dst_max_seq_len, const float* weights,
                                 float* weights_out, void* stream) {
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache(cfg, kv)) != COBS_OK) return s;
  if (dst && (s = check_cache(cfg, dst)) != COBS_OK) return s;
  if (num_kept < 0 || num_kept > cfg->max_seq_len || (per_head != 0 && per_head != 1)) return COBS_ERR_INVALID_ARG;
  if ((!kept && num_kept > 0) || !seq_lens) return COBS_ERR_INVALID_ARG;
  if (dst_max_seq_len < 1 || dst_max_seq_len % cfg->block_size != 0) return COBS_ERR_INVALID_ARG;
  if (dst_max_seq_len / cfg->block_size > kMaxBlocksPerSeq) return COBS_ERR_UNSUPPORTED;
  if (!dst && dst_max_seq_len != cfg->max_seq_len) return COBS_ERR_INVALID_ARG;
  // apart in memory: the same cache as its own destination is the call in place; other pages of the same pool are apart
  if (dst && (dst->k == kv->v || dst->v == kv->k)) return COBS_ERR_INVALID_ARG;
  if (dst && (dst->k == kv->k || dst->v == kv->v) &&
      !(dst->block_table && kv->block_table && dst->block_table != kv->block_table))
    return COBS_ERR_INVALID_ARG;
  // rows and heads that share memory cannot be written apart
  const cobs_kv_t* to = dst ? dst : kv;
  if (!to->block_table && ((cfg->batch > 1 && to->stride_b == 0) || (cfg->num_kv_heads > 1 && to->stride_h == 0)))
    return COBS_ERR_INVALID_ARG;
  if ((weights == nullptr) != (weights_out == nullptr)) return COBS_ERR_INVALID_ARG;
  if (weights && (weights == weights_out) != (dst == nullptr)) return COBS_ERR_INVALID_ARG;
  CompactParams p = {};
  p.src = view_of(cfg, kv, cfg->max_seq_len);
  p.dst = view_of(cfg, dst ? dst : kv, dst_max_seq_len);
  p.kept = kept;
  p.seq_lens = seq_lens;
  p.first = first;
  p.weights = weights;
  p.weights_out = weights_out;
  p.per_head = per_head;
  p.num_kept = num_kept;
  p.B = cfg->batch;
  p.hkv = cfg->num_kv_heads;
  p.d = cfg->head_dim;
  p.tmax = cfg->max_seq_len;
  p.dst_max = dst_max_seq_len;
  p.kv_f32 = cfg->kv_dtype == COBS_F32;
  p.in_place = dst == nullptr;
  return hip_status(launch_compact(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

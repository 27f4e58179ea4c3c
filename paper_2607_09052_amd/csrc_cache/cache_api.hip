// C ABI of the cache operators (include/cobs_cache.h): argument validation and
// parameter blocks.  Every entry point validates on the host before it enqueues
// anything, never synchronises and keeps nothing.
#include "cache_check.h"
#include "cobs_cache.h"

using namespace cobs;

namespace {

static_assert(kMaxQueries == COBS_MAX_QUERIES, "the header's bound");

// The arguments that cobs_tree_decode and cobs_attention_weights share.
cobs_status_t attend_params(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                            const cobs_kv_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                            const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, AttendParams* a) {
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache(cfg, kv)) != COBS_OK) return s;
  if ((s = check_queries(cfg, q, io_dtype, num_queries, seq_lens, draft_lens, tree_mask, sparse, sel, a)) != COBS_OK) return s;
  a->kv = view_of(cfg, kv, cfg->max_seq_len);
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

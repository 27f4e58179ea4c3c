// C ABI of the token operators (include/cobs_tokens.h): argument validation and parameter
// blocks.  Every entry point validates on the host before it enqueues anything, never synchronises
// and keeps nothing.
#include "cache_check.h"
#include "cobs_cache.h"
#include "cobs_tokens.h"
#include "tokens_kernels.h"

using namespace cobs;

namespace {

bool io_type(cobs_dtype_t t) { return t == COBS_F32 || t == COBS_BF16; }

// Heads [batch, tokens, heads, d]; the stride of a dimension of 1 is not used and may be anything.
struct HeadsShape {
  int64_t batch, tokens, heads, d;
};

cobs_status_t check_heads(const cobs_heads_t* x, cobs_dtype_t type, const HeadsShape& n) {
  if (!x || !x->p || !aligned(x->p, 16)) return COBS_ERR_INVALID_ARG;
  const int64_t vec = type == COBS_F32 ? 4 : 8;          // elements of 16 bytes
  if (n.batch > 1 && (x->stride_b < 0 || x->stride_b % vec)) return COBS_ERR_INVALID_ARG;
  if (n.tokens > 1 && (x->stride_n < 0 || x->stride_n % vec)) return COBS_ERR_INVALID_ARG;
  if (n.heads > 1 && (x->stride_h < 0 || x->stride_h % vec)) return COBS_ERR_INVALID_ARG;
  return COBS_OK;
}

// Whether no two elements share memory: sorted, each stride spans the dimensions of smaller ones and the d elements of a row.
bool apart(const int64_t (&stride)[3], const int64_t (&shape)[3], int64_t d) {
  int64_t size[3] = {shape[0], shape[1], shape[2]}, extent = d;
  for (int k = 0; k < 3; ++k) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (size[i] > 1 && (at < 0 || stride[i] < stride[at])) at = i;
    if (at < 0) break;
    if (stride[at] < extent || stride[at] > INT64_MAX / size[at]) return false;
    extent = stride[at] * (size[at] - 1) + extent;
    size[at] = 1;
  }
  return true;
}

HeadsView view_heads(const cobs_heads_t* x, cobs_dtype_t type) {
  return {x->p, x->stride_b, x->stride_n, x->stride_h, type == COBS_F32};
}

cobs_status_t check_rope(const cobs_rope_t* r, int32_t d) {
  if (!r->inv_freq || !isfinite(r->scale) || (r->interleaved != 0 && r->interleaved != 1)) return COBS_ERR_INVALID_ARG;
  if (r->rotary_dim < 1 || r->rotary_dim > d) return COBS_ERR_INVALID_ARG;
  return r->rotary_dim % 16 ? COBS_ERR_UNSUPPORTED : COBS_OK;
}

RopeView view_rope(const cobs_rope_t* r, const int32_t* positions) {
  return {r->inv_freq, positions, r->rotary_dim / 2, r->interleaved, r->scale};
}

// Queries and where they go: both checked, and the one itself or apart from the other.
cobs_status_t check_out(const cobs_heads_t* x, cobs_dtype_t in, const cobs_heads_t* y, cobs_dtype_t out, const HeadsShape& n) {
  cobs_status_t s;
  if (!io_type(in) || !io_type(out)) return COBS_ERR_INVALID_ARG;
  if ((s = check_heads(x, in, n)) != COBS_OK || (s = check_heads(y, out, n)) != COBS_OK) return s;
  if (!apart({y->stride_b, y->stride_n, y->stride_h}, {n.batch, n.tokens, n.heads}, n.d)) return COBS_ERR_INVALID_ARG;
  const bool same = (n.batch == 1 || x->stride_b == y->stride_b) && (n.tokens == 1 || x->stride_n == y->stride_n) &&
                    (n.heads == 1 || x->stride_h == y->stride_h) && in == out;
  return x->p == y->p && !same ? COBS_ERR_INVALID_ARG : COBS_OK;
}

// What cobs_append and cobs_append8 share.
cobs_status_t new_tokens(const cobs_config_t* cfg, const cobs_heads_t* k_new, const cobs_heads_t* v_new, cobs_dtype_t in_dtype,
                         int32_t num_new, const int32_t* seq_lens, const int32_t* new_lens, const cobs_rope_t* rope,
                         const int32_t* positions, const cobs_heads_t* q, const cobs_heads_t* q_out, cobs_dtype_t q_dtype,
                         int32_t* new_seq_lens, NewTokens* t) {
  cobs_status_t s;
  const int d = cfg->head_dim;
  if (!io_type(in_dtype) || num_new < 1 || !seq_lens) return COBS_ERR_INVALID_ARG;
  if (new_seq_lens && (new_seq_lens == seq_lens || new_seq_lens == new_lens || new_seq_lens == positions))
    return COBS_ERR_INVALID_ARG;
  const HeadsShape kv_shape = {cfg->batch, num_new, cfg->num_kv_heads, d}, q_shape = {cfg->batch, num_new, cfg->num_q_heads, d};
  if ((s = check_heads(k_new, in_dtype, kv_shape)) != COBS_OK || (s = check_heads(v_new, in_dtype, kv_shape)) != COBS_OK) return s;
  if (rope && (s = check_rope(rope, d)) != COBS_OK) return s;
  if ((q == nullptr) != (q_out == nullptr)) return COBS_ERR_INVALID_ARG;
  if (q) {
    if ((s = check_out(q, in_dtype, q_out, q_dtype, q_shape)) != COBS_OK) return s;
    if (q_out->p == k_new->p || q_out->p == v_new->p) return COBS_ERR_INVALID_ARG;
    t->hq = cfg->num_q_heads;
    t->q = view_heads(q, in_dtype);
    t->q_out = view_heads(q_out, q_dtype);
  }
  if ((int64_t)cfg->batch * num_new > (1 << 24)) return COBS_ERR_UNSUPPORTED;
  if (rope) t->rope = view_rope(rope, positions);
  t->k = view_heads(k_new, in_dtype);
  t->v = view_heads(v_new, in_dtype);
  t->seq_lens = seq_lens;
  t->new_lens = new_lens;
  t->new_seq_lens = new_seq_lens;
  t->B = cfg->batch;
  t->N = num_new;
  t->hkv = cfg->num_kv_heads;
  t->d = d;
  t->tmax = cfg->max_seq_len;
  return COBS_OK;
}

// A cache that is written: keys and values, or rows, heads and tokens, that share memory cannot be.
template <typename Kv>
bool shares_memory(const cobs_config_t* c, const Kv* kv) {
  if (kv->k == kv->v) return true;
  return !kv->block_table && !apart({kv->stride_b, kv->stride_h, kv->stride_t}, {c->batch, c->num_kv_heads, c->max_seq_len}, c->head_dim);
}

cobs_status_t check_cache8(const cobs_config_t* c, const cobs_kv8_t* kv) {
  if (!kv || !kv->k || !kv->v || !aligned(kv->k, 16) || !aligned(kv->v, 16)) return COBS_ERR_INVALID_ARG;
  if (!kv->k_scale || !kv->v_scale || !aligned(kv->k_scale, 4) || !aligned(kv->v_scale, 4)) return COBS_ERR_INVALID_ARG;
  if (kv->block_table) return kv->num_pages < 1 ? COBS_ERR_INVALID_ARG : COBS_OK;
  if (kv->stride_t < c->head_dim || kv->stride_h < 0 || kv->stride_b < 0) return COBS_ERR_INVALID_ARG;
  if (kv->stride_t % 16 || kv->stride_h % 16 || kv->stride_b % 16) return COBS_ERR_INVALID_ARG;
  return kv->stride_t > (int64_t)1 << 22 ? COBS_ERR_UNSUPPORTED : COBS_OK;
}

KvView view_of8(const cobs_config_t* c, const cobs_kv8_t* kv) {
  const cobs_kv_t x = {kv->k, kv->v, kv->stride_b, kv->stride_h, kv->stride_t, kv->block_table, kv->num_pages};
  return view_of(c, &x, c->max_seq_len);
}

}  // namespace

extern "C" {

cobs_status_t cobs_rotate(const cobs_heads_t* x, cobs_dtype_t in_dtype, int32_t batch, int32_t num_tokens,
                          int32_t num_heads, int32_t head_dim, const cobs_rope_t* rope, const int32_t* positions,
                          const cobs_heads_t* out, cobs_dtype_t out_dtype, void* stream) {
  cobs_status_t s;
  if (batch < 1 || num_tokens < 1 || num_heads < 1 || head_dim < 1 || !rope || !positions) return COBS_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return COBS_ERR_UNSUPPORTED;
  if ((s = check_rope(rope, head_dim)) != COBS_OK) return s;
  const int64_t tokens = (int64_t)batch * num_tokens;
  if (tokens > ((int64_t)1 << 31) / num_heads) return COBS_ERR_UNSUPPORTED;
  if ((s = check_out(x, in_dtype, out, out_dtype, {batch, num_tokens, num_heads, head_dim})) != COBS_OK) return s;
  AppendParams p = {};
  p.t.rope = view_rope(rope, positions);
  p.t.q = view_heads(x, in_dtype);
  p.t.q_out = view_heads(out, out_dtype);
  p.t.B = batch;
  p.t.N = num_tokens;
  p.t.hq = num_heads;
  p.t.d = head_dim;
  return hip_status(launch_append(p, static_cast<hipStream_t>(stream)));
}

cobs_status_t cobs_append(const cobs_config_t* cfg, const cobs_heads_t* k_new, const cobs_heads_t* v_new,
                          cobs_dtype_t in_dtype, int32_t num_new, const cobs_kv_t* kv, const int32_t* seq_lens,
                          const int32_t* new_lens, const cobs_rope_t* rope, const int32_t* positions,
                          const cobs_heads_t* q, const cobs_heads_t* q_out, cobs_dtype_t q_dtype,
                          int32_t* new_seq_lens, void* stream) {
  AppendParams p = {};
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache(cfg, kv)) != COBS_OK) return s;
  if (shares_memory(cfg, kv)) return COBS_ERR_INVALID_ARG;
  s = new_tokens(cfg, k_new, v_new, in_dtype, num_new, seq_lens, new_lens, rope, positions, q, q_out, q_dtype, new_seq_lens,
                 &p.t);
  if (s != COBS_OK) return s;
  p.kv = view_of(cfg, kv, cfg->max_seq_len);
  p.kv_f32 = cfg->kv_dtype == COBS_F32;
  return hip_status(launch_append(p, static_cast<hipStream_t>(stream)));
}

cobs_status_t cobs_append8(const cobs_config_t* cfg, const cobs_heads_t* k_new, const cobs_heads_t* v_new,
                           cobs_dtype_t in_dtype, int32_t num_new, const cobs_kv8_t* kv, const int32_t* seq_lens,
                           const int32_t* new_lens, const cobs_rope_t* rope, const int32_t* positions,
                           const cobs_heads_t* q, const cobs_heads_t* q_out, cobs_dtype_t q_dtype,
                           int32_t* new_seq_lens, void* stream) {
  Append8Params p = {};
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache8(cfg, kv)) != COBS_OK) return s;
  if (shares_memory(cfg, kv) || kv->k_scale == kv->v_scale) return COBS_ERR_INVALID_ARG;
  s = new_tokens(cfg, k_new, v_new, in_dtype, num_new, seq_lens, new_lens, rope, positions, q, q_out, q_dtype, new_seq_lens,
                 &p.t);
  if (s != COBS_OK) return s;
  p.kv = view_of8(cfg, kv);
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  return hip_status(launch_append8(p, static_cast<hipStream_t>(stream)));
}

size_t cobs_decode8_workspace_bytes(const cobs_config_t* cfg, int32_t num_queries) {
  if (check_shape(cfg) != COBS_OK || num_queries < 1 || num_queries > kMaxQueries) return 0;
  AttendParams a = {};
  shape_of(cfg, num_queries, &a);
  return decode8_workspace(a);
}

cobs_status_t cobs_decode8(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                           const cobs_kv8_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                           const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, void* out, float* lse,
                           void* ws, size_t ws_bytes, void* stream) {
  Decode8Params p = {};
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache8(cfg, kv)) != COBS_OK) return s;
  if ((s = check_queries(cfg, q, io_dtype, num_queries, seq_lens, draft_lens, tree_mask, sparse, sel, &p.t.a)) != COBS_OK)
    return s;
  if (!out || !aligned(out, 16) || out == q) return COBS_ERR_INVALID_ARG;
  p.t.a.kv = view_of8(cfg, kv);
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  const size_t need = decode8_workspace(p.t.a);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 256))) return COBS_ERR_WORKSPACE;
  p.t.out = out;
  p.t.lse = lse;
  p.t.part_ml = static_cast<float*>(ws);
  return hip_status(launch_decode8(p, static_cast<hipStream_t>(stream)));
}

cobs_status_t cobs_unpack8(const cobs_config_t* cfg, const cobs_kv8_t* kv, const int32_t* seq_lens,
                           int32_t first_block, int32_t num_blocks, const cobs_kv_t* dst, void* stream) {
  cobs_status_t s = check_shape(cfg);
  if (s != COBS_OK) return s;
  if ((s = check_cache8(cfg, kv)) != COBS_OK) return s;
  if ((s = check_cache(cfg, dst)) != COBS_OK) return s;
  if (shares_memory(cfg, dst)) return COBS_ERR_INVALID_ARG;
  const int32_t nb = cfg->max_seq_len / cfg->block_size;
  if (!seq_lens || first_block < -1 || first_block > nb || num_blocks < 0 || num_blocks > nb - (first_block < 0 ? 0 : first_block))
    return COBS_ERR_INVALID_ARG;
  for (const void* x : {dst->k, dst->v})
    if (x == kv->k || x == kv->v || x == kv->k_scale || x == kv->v_scale) return COBS_ERR_INVALID_ARG;
  Unpack8Params p = {};
  p.src = view_of8(cfg, kv);
  p.dst = view_of(cfg, dst, cfg->max_seq_len);
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  p.seq_lens = seq_lens;
  p.B = cfg->batch;
  p.hkv = cfg->num_kv_heads;
  p.d = cfg->head_dim;
  p.tmax = cfg->max_seq_len;
  p.first = first_block;
  p.num = num_blocks;
  p.f32 = cfg->kv_dtype == COBS_F32;
  return hip_status(launch_unpack8(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

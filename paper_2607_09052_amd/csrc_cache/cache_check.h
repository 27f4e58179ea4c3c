// Host checks and parameter blocks that the entry points on the cache share.
#pragma once

#include <math.h>

#include "cache_kernels.h"
#include "cobs.h"

namespace cobs {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline cobs_status_t hip_status(hipError_t e) { return e == hipSuccess ? COBS_OK : COBS_ERR_HIP; }

// The fields of cobs_config_t that these calls read, with the decode path's limits.
inline cobs_status_t check_shape(const cobs_config_t* c) {
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

inline cobs_status_t check_cache(const cobs_config_t* c, const cobs_kv_t* kv) {
  if (!kv || !kv->k || !kv->v || !aligned(kv->k, 16) || !aligned(kv->v, 16)) return COBS_ERR_INVALID_ARG;
  if (kv->block_table) return kv->num_pages < 1 ? COBS_ERR_INVALID_ARG : COBS_OK;
  const int64_t vec = c->kv_dtype == COBS_F32 ? 4 : 8;      // elements of 16 bytes
  if (kv->stride_t < c->head_dim || kv->stride_h < 0 || kv->stride_b < 0) return COBS_ERR_INVALID_ARG;
  if (kv->stride_t % vec || kv->stride_h % vec || kv->stride_b % vec) return COBS_ERR_INVALID_ARG;
  if (kv->stride_t > (int64_t)1 << 22) return COBS_ERR_UNSUPPORTED;
  return COBS_OK;
}

inline int log2_of(int block_size) { return block_size == 32 ? 5 : (block_size == 64 ? 6 : 7); }

inline KvView view_of(const cobs_config_t* c, const cobs_kv_t* kv, int capacity) {
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

inline void shape_of(const cobs_config_t* c, int32_t num_queries, AttendParams* a) {
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

// The queries of a call and what they attend to; all of `a` but the cache.
inline cobs_status_t check_queries(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                                   const int32_t* seq_lens, const int32_t* draft_lens, const uint64_t* tree_mask,
                                   int32_t sparse, const int32_t* sel, AttendParams* a) {
  if (num_queries < 1) return COBS_ERR_INVALID_ARG;
  if (num_queries > kMaxQueries) return COBS_ERR_UNSUPPORTED;
  if (io_dtype != COBS_F32 && io_dtype != COBS_BF16) return COBS_ERR_INVALID_ARG;
  if (!q || !aligned(q, 16) || !seq_lens) return COBS_ERR_INVALID_ARG;
  if ((draft_lens == nullptr) != (tree_mask == nullptr) || !aligned(tree_mask, 8)) return COBS_ERR_INVALID_ARG;
  if (sparse != 0 && sparse != 1) return COBS_ERR_INVALID_ARG;
  if (sparse ? (!sel && cfg->budget > 0) : sel != nullptr) return COBS_ERR_INVALID_ARG;
  shape_of(cfg, num_queries, a);
  a->q = q;
  a->seq_lens = seq_lens;
  a->draft_lens = draft_lens;
  a->mask = tree_mask;
  a->sel = sel;
  a->sparse = sparse;
  a->io_bf16 = io_dtype == COBS_BF16;
  return COBS_OK;
}

}  // namespace cobs

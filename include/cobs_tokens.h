/*
 * cobs_tokens.h - new tokens on their way into the KV cache, and a cache of 8-bit
 * floats, part of libcobs.so beside cobs.h and cobs_cache.h: rotary positions of
 * query and key heads, the append of rotated keys and of values to a cache, the
 * same into a cache of 8-bit floats with one scale for each block and KV head,
 * attention over such a cache, and its blocks written back to a bf16 or fp32 one.
 *
 * The conventions of cobs.h and cobs_cache.h hold: device pointers that the caller
 * owns, host validation before any launch, asynchronous work on `stream` (of the
 * current device), no allocation, no state between calls, deterministic results.
 * Of cobs_config_t these calls read batch, num_q_heads, num_kv_heads, head_dim,
 * max_seq_len and block_size, cobs_append and cobs_unpack8 kv_dtype as well, and
 * cobs_decode8 budget, window and softmax_scale, with the same limits as there;
 * the other fields are ignored (but have to be valid values for a kv_dtype,
 * budget, window and scale).
 */
#ifndef COBS_TOKENS_H
#define COBS_TOKENS_H

#include "cobs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads of tokens as a projection leaves them: element (b, i, h, e) at
 *   p + b*stride_b + i*stride_n + h*stride_h + e   (strides in elements, e < d contiguous).
 * p: 16-byte aligned; strides >= 0 and multiples of 16 bytes' worth of elements (that of a dimension
 * of 1 is not used).  Of what a call writes no two elements may share memory: sorted by stride, each
 * dimension's stride has to span the ones before it, or the call is refused. */
typedef struct {
  void* p;
  int64_t stride_b, stride_n, stride_h;
} cobs_heads_t;

/* Rotary positions.  The first rotary_dim = r elements of a head are r/2 pairs; pair p of a
 * token at position t turns by the angle a = t f_p and is multiplied by `scale`:
 *   y_lo = scale (x_lo cos a - x_hi sin a),   y_hi = scale (x_hi cos a + x_lo sin a),
 * lo = p, hi = p + r/2 (interleaved = 0) or lo = 2p, hi = 2p + 1 (interleaved = 1).  The
 * elements from r on are left as they are.  The frequencies are the caller's, so that any
 * scaling of them for long contexts is a matter of this table.
 *   inv_freq: device fp32 [r/2], f_p in radians, |t f_p| <= 2^51 (all positions: |f_p| <= 2^20);
 *             a pair whose angle is past that, or not finite, becomes NaN.  t f_p is exact before
 *             it is reduced, so far positions lose nothing; the pair's products are fp32.
 *   rotary_dim: a multiple of 16, 16 <= r <= d.  scale: finite.                       */
typedef struct {
  const float* inv_freq;
  int32_t rotary_dim;
  int32_t interleaved;
  float scale;
} cobs_rope_t;

/* Rotary positions of num_heads heads of batch * num_tokens tokens.
 *   x:   in_dtype COBS_F32 or COBS_BF16, [batch, num_tokens, num_heads, head_dim] by its strides.
 *   positions: device int32 [batch, num_tokens]; negative ones turn the other way.
 *   out: out_dtype COBS_F32 or COBS_BF16, the same shape, rounded once; x itself (same type
 *        and strides), or apart in memory.
 *   head_dim 64 or 128; batch * num_tokens * num_heads <= 2^31.                       */
cobs_status_t cobs_rotate(const cobs_heads_t* x, cobs_dtype_t in_dtype, int32_t batch, int32_t num_tokens,
                          int32_t num_heads, int32_t head_dim, const cobs_rope_t* rope, const int32_t* positions,
                          const cobs_heads_t* out, cobs_dtype_t out_dtype, void* stream);

/* New tokens behind a cache's: token i < n of row b, n = new_lens[b] (clamped to [0, num_new];
 * new_lens NULL: num_new), becomes cached token T + i, T = seq_lens[b] (clamped), its key
 * rotated, its value as it is, rounded once to kv_dtype.
 *   k_new, v_new: in_dtype COBS_F32 or COBS_BF16, [B, num_new, Hkv, d] by their strides, apart from what the call writes.
 *   rope:      NULL leaves keys and queries as they are.
 *   positions: optional device int32 [B, num_new]; NULL: T + i (the place in the cache;
 *              after an eviction, or for a draft's tree, the positions are others).
 *   q, q_out:  optional, both or neither: the same tokens' queries, in_dtype [B, num_new, Hq, d],
 *              rotated beside the keys into q_out (q_dtype COBS_F32 or COBS_BF16): q itself
 *              (same type and strides), or apart from all else.  Queries i >= n are left as they were.
 *   new_seq_lens: optional device int32 [B], written: min(T + n, max_seq_len); not seq_lens itself.
 *   Tokens behind the cache's capacity, or whose page id is out of range, are dropped.
 *   1 <= num_new, batch * num_new <= 2^24.  Keys and values, and rows, heads and tokens of the cache, share no
 *   memory (one pointer for both is refused, and strides of which, sorted, one does not span the ones before it, as
 *   with cobs_heads_t; no page is in a table twice).
 * The records of the blocks that got tokens are stale afterwards (cobs_decode_step
 * refreshes the newest; cobs_build_block_stats rebuilds any).                       */
cobs_status_t cobs_append(const cobs_config_t* cfg, const cobs_heads_t* k_new, const cobs_heads_t* v_new,
                          cobs_dtype_t in_dtype, int32_t num_new, const cobs_kv_t* kv, const int32_t* seq_lens,
                          const int32_t* new_lens, const cobs_rope_t* rope, const int32_t* positions,
                          const cobs_heads_t* q, const cobs_heads_t* q_out, cobs_dtype_t q_dtype,
                          int32_t* new_seq_lens, void* stream);

/* A cache of 8-bit floats: OCP e4m3 (4 exponent bits of bias 7, 3 mantissa bits, no infinities,
 * +-448 the largest, 0x7f and 0xff NaN), and for each block of block_size tokens and KV head one
 * fp32 scale of the keys and one of the values: the element is code * scale.
 * Places are those of cobs_kv_t with one byte an element (contiguous with strides, multiples
 * of 16, or pages).  Scales, 4-byte aligned: [B, Hkv, T_max/L], or with pages [num_pages, Hkv].
 * Scales are finite and not negative.                                               */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int64_t stride_b, stride_h, stride_t;
  const int32_t* block_table;
  int64_t num_pages;
} cobs_kv8_t;

/* cobs_append into an 8-bit cache.  For each block and KV head that gets new tokens, keys and
 * values apart, with m the largest |x| among the new tokens' elements (rotated, in fp32; only finite
 * ones count): s' = the smallest power of two with m / s' <= 448, 2^-100 at least; the block's
 * scale becomes s = max(s', its scale) if it holds earlier tokens (positions below T), else s'.
 * Elements are encoded as the nearest e4m3 number to x / s, ties to even; what is not finite
 * becomes NaN.  Where a scale grows, the block's earlier tokens are encoded again at the new one
 * (exact but for the smallest numbers, as scales are powers of two).  The codes of a block
 * behind its last token are left as they were.
 * Arguments otherwise as for cobs_append.  Earlier scales have to be powers of two from 2^-100
 * on (as written here), or the quotients' rounding may be off in the last bit before it.       */
cobs_status_t cobs_append8(const cobs_config_t* cfg, const cobs_heads_t* k_new, const cobs_heads_t* v_new,
                           cobs_dtype_t in_dtype, int32_t num_new, const cobs_kv8_t* kv, const int32_t* seq_lens,
                           const int32_t* new_lens, const cobs_rope_t* rope, const int32_t* positions,
                           const cobs_heads_t* q, const cobs_heads_t* q_out, cobs_dtype_t q_dtype,
                           int32_t* new_seq_lens, void* stream);

/* Workspace bytes of cobs_decode8 (0 if invalid).  It has to be zero-filled before its first use;
 * every call leaves its arrival counters (the first 16 KB) zero again, so that later calls of cobs_decode8
 * on the same stream, of other shapes too, may use it; other operators may not, as they leave
 * what they like there.  Calls that share it must not overlap in time. */
size_t cobs_decode8_workspace_bytes(const cobs_config_t* cfg, int32_t num_queries);

/* Attention of num_queries query tokens a row (1 <= num_queries <= 64) over an 8-bit cache.
 * Arguments and attended tokens are cobs_tree_decode's: the context of C = seq_lens[b] tokens, all of
 * it or (sparse = 1) the selected blocks and the window, and with a tree mask the drafted tokens
 * behind it.  One query without a draft is a decode step.
 * A token that a query does not attend to has no effect on it, whatever its codes are.
 * Scores, softmax and sums are fp32.  The matrix cores take the codes as bf16, which is exact, an
 * fp32 query and the probabilities as three bf16 parts, which hold all their bits; with io_dtype
 * COBS_BF16 and more than 16 query rows of a KV head (num_queries * num_q_heads / num_kv_heads)
 * the probabilities enter as two (2^-17).  bf16 outputs are rounded once.                       */
cobs_status_t cobs_decode8(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                           const cobs_kv8_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                           const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, void* out, float* lse,
                           void* ws, size_t ws_bytes, void* stream);

/* Blocks of an 8-bit cache as bf16 or fp32 (kv_dtype): elements code * scale in fp32, for bf16 rounded from
 * there (both exact for scales that are powers of two), token t to token t of another cache of the same
 * configuration, for cobs_build_block_stats and whatever else reads one.
 *   first_block >= 0: the blocks first_block <= j < first_block + num_blocks that a row of
 *   T = seq_lens[b] tokens has; first_block = -1: its last num_blocks blocks.  num_blocks >= 0.
 *   dst: strides or pages of its own, apart from the source.  Tokens from T on, and those whose
 *   page is out of range in the source or in dst (so a table may have pages for the wanted
 *   blocks alone), are left as they were.  Keys, values, rows, heads and tokens of dst share no memory
 *   (refused as for cobs_append).                                                                  */
cobs_status_t cobs_unpack8(const cobs_config_t* cfg, const cobs_kv8_t* kv, const int32_t* seq_lens,
                           int32_t first_block, int32_t num_blocks, const cobs_kv_t* dst, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* COBS_TOKENS_H */

/*
 * cobs_cache.h - operators on the KV cache between decode steps, part of
 * libcobs.so beside the decode path of cobs.h: attention of several query
 * tokens a row (the tree of a speculative draft), the attention weights that
 * cached tokens receive, eviction by those weights, and the compaction of the
 * cache to the tokens that are kept (evicted to, or accepted of a draft).
 *
 * The conventions of cobs.h hold: device pointers that the caller owns, host
 * validation before any launch, asynchronous work on `stream` (of the current
 * device), no allocation, no state between calls, deterministic results (the
 * same call gives the same bits; the order in which a row's attention is summed
 * may go by the lengths of the batch's other rows).  Of
 * cobs_config_t these calls read batch, num_q_heads, num_kv_heads, head_dim,
 * max_seq_len, block_size, budget, window, kv_dtype and softmax_scale, with the
 * same limits as there; the record fields are ignored.
 *
 * The tokens a query attends to.  Row b's context is its first C = seq_lens[b]
 * cached tokens (clamped to [0, max_seq_len]).
 *   - All of it (sparse = 0), or (sparse = 1) the union that cobs_sparse_decode
 *     attends to at T = C: the tokens before the window start ws = max(0, C - w)
 *     of the selected blocks, and the last w tokens.  sel: device int32
 *     [B, Hkv, budget]; as there, its longest strictly ascending prefix of
 *     candidate ids is used.  sel is required with sparse = 1 and budget > 0,
 *     and must be NULL with sparse = 0.
 *   - A draft (tree_mask != NULL): query i is drafted token i of
 *     n = draft_lens[b] (device int32 [B], clamped to [0, min(num_queries,
 *     max_seq_len - C)]).  Drafted token j's key and value stand in the cache
 *     behind the context, at position C + j.  tree_mask: device uint64
 *     [B, num_queries]; query i attends to drafted token j (its ancestors and
 *     itself, say) iff bit j of tree_mask[b][i] is set; bits from n on are
 *     ignored.  Queries i >= n attend to nothing.
 *   - No draft (tree_mask and draft_lens both NULL): all num_queries queries
 *     attend to the context alone.  One query is then cobs_sparse_decode.
 * A token that a query does not attend to has no effect on it, whatever its key
 * and value hold; one that it attends to acts as in plain arithmetic (with a score of
 * -inf its probability is 0, an infinite value is one in the output; a query with no
 * other scores is like one that attends to nothing).  Infinities there may make a call
 * take a hundred times as long.  Tokens on a page whose id is out of range are left out.
 */
#ifndef COBS_CACHE_H
#define COBS_CACHE_H

#include "cobs.h"

#ifdef __cplusplus
extern "C" {
#endif

#define COBS_MAX_QUERIES 64 /* queries (drafted tokens) per row and call */

/* Workspace bytes of cobs_tree_decode (0 if invalid).  It needs no clearing. */
size_t cobs_tree_workspace_bytes(const cobs_config_t* cfg, int32_t num_queries);

/* Attention of num_queries query tokens a row (1 <= num_queries <= 64) over the
 * tokens above, one softmax per query and query head.
 *   q:    device io_dtype [B, num_queries, Hq, d], unscaled; io_dtype COBS_F32 or COBS_BF16.
 *   out:  device io_dtype [B, num_queries, Hq, d], written; 0 for a query that attends to nothing.
 *   lse:  optional device fp32 [B, num_queries, Hq], written: ln sum exp(c q.k_t); -inf for such a query.
 *   q, out: 16-byte aligned, apart in memory.
 *   ws:   cobs_tree_workspace_bytes(cfg, num_queries), 256-byte aligned.
 * Scores, softmax and sums are fp32.  With bf16 keys and values the matrix cores
 * take bf16 operands: an fp32 query and its probabilities enter as three bf16
 * parts, which hold all their bits; with io_dtype COBS_BF16 the probabilities enter as
 * two (2^-17) and the outputs are rounded once.                                   */
cobs_status_t cobs_tree_decode(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype, int32_t num_queries,
                               const cobs_kv_t* kv, const int32_t* seq_lens, const int32_t* draft_lens,
                               const uint64_t* tree_mask, int32_t sparse, const int32_t* sel, void* out, float* lse,
                               void* ws, size_t ws_bytes, void* stream);

/* The attention weights that every cached token receives from the queries:
 *   weights[b][h][t] = prev[b][h][t] + sum_{i, g} exp(c q_{i,g}.k_t - lse_{i,g})
 * over the queries i (and the G query heads g of KV head h) that attend to t, for
 * t < C + n; weights of later positions are left as they were.
 *   q, num_queries, io_dtype, kv, ..., sel: as for cobs_tree_decode (V is not read).
 *   lse:     device fp32 [B, num_queries, Hq]: the queries' normalisers, as cobs_tree_decode
 *            or a decode step returns them.  A query head with lse -inf or +inf adds nothing
 *            (+inf leaves a rejected drafted token out), whatever its query holds
 *            (one that is not finite makes the call some hundred times as long).
 *   prev:    optional device fp32 [B, Hkv, max_seq_len], NULL for zeros; `weights` itself, or apart.
 *   weights: device fp32 [B, Hkv, max_seq_len].                                     */
cobs_status_t cobs_attention_weights(const cobs_config_t* cfg, const void* q, cobs_dtype_t io_dtype,
                                     int32_t num_queries, const cobs_kv_t* kv, const int32_t* seq_lens,
                                     const int32_t* draft_lens, const uint64_t* tree_mask, int32_t sparse,
                                     const int32_t* sel, const float* lse, const float* prev, float* weights,
                                     void* stream);

/* Workspace bytes of cobs_evict (0 if none is needed, or cfg is invalid).  It needs
 * no clearing.                                                                    */
size_t cobs_evict_workspace_bytes(const cobs_config_t* cfg);

/* The tokens a cache keeps.  For every (batch row, KV head) with T = seq_lens[b]
 * tokens: all of them if T <= keep, else the first `sinks`, the last `recent`
 * and, of those between, the keep - sinks - recent with the largest weights (ties
 * to the lower position; a NaN weight ranks with -inf).
 *   weights:  device fp32 [B, Hkv, max_seq_len].
 *   1 <= keep <= max_seq_len; sinks, recent >= 0, sinks + recent <= keep.
 *   kept:     device int32 [B, Hkv, keep], written: positions, ascending, then -1.
 *   new_lens: optional device int32 [B], written: min(T, keep); not seq_lens itself.
 *   ws:       cobs_evict_workspace_bytes(cfg), 256-byte aligned; may be NULL if that is 0.  */
cobs_status_t cobs_evict(const cobs_config_t* cfg, const float* weights, const int32_t* seq_lens, int32_t keep,
                         int32_t sinks, int32_t recent, int32_t* kept, int32_t* new_lens, void* ws, size_t ws_bytes,
                         void* stream);

/* Move the kept tokens' keys, values and weights together: cached token
 * kept[..][j] of (b, h) becomes token first[b] + j.
 *   kept:      device int32 [B, Hkv, num_kept] (per_head = 1) or [B, num_kept], one list for
 *              all KV heads (per_head = 0).  Entries outside [0, T), T = seq_lens[b] clamped,
 *              or whose row or destination lies on a page out of range, move nothing.
 *   seq_lens:  device int32 [B]: cached tokens of each row before the move, drafted ones included.
 *   first:     optional device int32 [B] (>= 0), NULL for 0: where the moved tokens go (the
 *              context length, when the accepted tokens of a draft move up behind it).
 *   dst:       NULL: in place.  Then the entries must ascend strictly with
 *              kept[j] >= first + j (as cobs_evict's do; otherwise the moved rows' contents are
 *              unspecified).  Else another cache with the strides or pages of `dst` and a capacity
 *              of dst_max_seq_len tokens (a multiple of block_size; in place max_seq_len), apart
 *              from the first in memory: other tensors, or other pages of the same pool, given by
 *              a table of their own.  Any order, repeats allowed; tokens that would go behind the
 *              capacity are dropped.  Rows and heads of the destination share no memory (strides
 *              of 0 are refused; no page is in a table twice).
 *   weights:   optional device fp32 [B, Hkv, max_seq_len]; weights_out: device fp32
 *              [B, Hkv, dst_max_seq_len], both or neither; the same pointer exactly when in
 *              place.  weights_out of the positions first + j whose entry moves nothing, and of
 *              those from first + num_kept to T, is set to 0.
 * Other positions of the destination are left as they were.  The records of moved
 * blocks are stale afterwards: rebuild them with cobs_build_block_stats.          */
cobs_status_t cobs_compact_cache(const cobs_config_t* cfg, const cobs_kv_t* kv, const int32_t* kept, int32_t per_head,
                                 int32_t num_kept, const int32_t* seq_lens, const int32_t* first,
                                 const cobs_kv_t* dst, int32_t dst_max_seq_len, const float* weights,
                                 float* weights_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* COBS_CACHE_H */

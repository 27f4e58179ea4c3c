// The heads of new tokens on their way: queries rotated, keys rotated and appended, values appended
// (cobs_rotate, cobs_append; the queries of cobs_append8).  A copy with a few operations an element: bound by
// HBM, or for a few tokens by the launch and a chain of loads (length, page, row).
//
// A workgroup takes a few consecutive tokens and some of their heads.  Its threads first write the
// tokens' cosines and sines to LDS, a pair each, as the fp64 reduction costs as much as the copy of 8
// elements and all heads of a token share it.  Then a thread takes 16 elements of a head, both
// sides of 8 pairs, in two 16-byte pieces (bf16).
//
// Measured (d 128, bf16): 8190 tokens of 32 heads rotated in 29.6 us, 4.5 TB/s, two rounds of workgroups; 32000 in 98 us, 5.3 TB/s;
// 32749 tokens of 32 query and 8 KV heads appended in 161 us, 5.0 TB/s (a large copy: 5.0); one token of 64 rows 4.6 us.  A thread's loads form a
// chain: length, page, the argument block's strides, then its pointer and type (chosen by lane: queries, keys or values), the row's two pieces one
// after the other.  Many workgroups hide it; few tokens and the first round show it (8190 tokens of 64-element heads in pairs side by side: 19.4 us, their bytes 13.3).
#pragma once

#include "tokens_device.h"

namespace cobs {

constexpr int kHeadThreads = 256;
constexpr int kMostTokens = 8;       // tokens of a workgroup

struct HeadsShared {
  float2 turn[kMostTokens][64];
  int64_t to[kMostTokens];           // place of the token in the cache (elements, KV head 0), -1: none
  int b[kMostTokens], i[kMostTokens];  // row and token; b = -1: none there
};

// Workgroup `wg` of ceil(B N / per_wg) * slot_groups.  Heads 0 .. hq - 1 are queries, then hkv keys and hkv
// values with a cache `kv` (CACHE).
template <int D, bool CACHE>
__device__ __forceinline__ void heads_body(const NewTokens& p, const KvView* kv, bool kv_f32, int wg, int per_wg, int slots,
                                           int slot_groups, HeadsShared& s) {
  constexpr int TPR = D / 16;
  const int tid = threadIdx.x, group = wg % slot_groups;
  const uint32_t first = (uint32_t)(wg / slot_groups) * per_wg;        // (tokens of a call: below 2^31)
  const int heads = p.hq + (CACHE ? 2 * p.hkv : 0);
  const int h0 = group * slots, h1 = min(heads, h0 + slots);
  if (tid < per_wg) {
    const uint32_t token = first + tid;
    int b = -1, i = 0;
    int64_t to = -1;
    if (token < (uint32_t)p.B * p.N) {
      b = token / (uint32_t)p.N;
      i = token - (uint32_t)b * p.N;
      const NewRow r = new_row(p, b);
      if (i >= r.n) b = -1;
      else if (CACHE && r.T + i < p.tmax) to = kv_offset(*kv, b, 0, r.T + i);
    }
    s.b[tid] = b;
    s.i[tid] = i;
    s.to[tid] = to;
  }
  if (p.rope.half > 0) {
    for (int x = tid; x < per_wg * p.rope.half; x += kHeadThreads) {
      const int k = x / p.rope.half, pair = x - k * p.rope.half;
      const uint32_t token = first + k;
      if (token >= (uint32_t)p.B * p.N) break;
      const uint32_t b = token / (uint32_t)p.N;
      const int at = p.rope.positions ? p.rope.positions[token] : new_row(p, b).T + (int)(token - b * p.N);
      s.turn[k][pair] = turn_of(p.rope, at, pair);
    }
  }
  __syncthreads();
  const int piece = tid % TPR;
  const Piece e = piece_of<D>(p.rope, piece);
  const int64_t head_step = CACHE ? (kv->table ? ((int64_t)D << kv->lsh) : kv->sh) : 0;
  const int rows = per_wg * (h1 - h0);
  for (int x = tid / TPR; x < rows; x += kHeadThreads / TPR) {
    const int k = x / (h1 - h0), h = h0 + (x - k * (h1 - h0));
    const int b = s.b[k];
    if (b < 0) continue;
    const bool query = h < p.hq, key = !query && h < p.hq + p.hkv;
    const HeadsView& from = query ? p.q : (key ? p.k : p.v);
    const int hh = query ? h : (h - p.hq) - (key ? 0 : p.hkv);
    const int64_t at = b * from.sb + s.i[k] * from.sn + hh * from.sh;
    void* out = query ? p.q_out.p : nullptr;
    int64_t to = query ? b * p.q_out.sb + s.i[k] * p.q_out.sn + hh * p.q_out.sh : s.to[k];
    bool f32 = p.q_out.f32;
    if constexpr (CACHE) {
      if (!query) {
        if (to < 0) continue;
        to += hh * head_step;
        out = const_cast<void*>(key ? kv->k : kv->v);
        f32 = kv_f32;
      }
    }
    const bool turned = e.turned && (query || key);
    float y[16];
    const Raw8 r0 = load_raw8(from.p, at + e.e0, from.f32), r1 = load_raw8(from.p, at + e.e1, from.f32);
    widen8(r0, from.f32, y);
    widen8(r1, from.f32, y + 8);
    if (turned) {
      float2 cs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) cs[j] = s.turn[k][pair_of(p.rope, piece, j)];
      turn16(y, cs, p.rope.interleaved);
    }
    store8(out, to + e.e0, f32, y);
    store8(out, to + e.e1, f32, y + 8);
  }
}

// Tokens and heads of a workgroup: with tokens enough to fill the card all heads of as many tokens as are two passes
// of its threads, else one token and 256 threads' worth of heads.  (By 4 tokens, 6 passes: 32749 tokens of 32 query and 8 KV heads
// appended in 173 us, by 2 in 164; by 4, half a pass: 64000 tokens of 2 KV heads 48 us for 38.)
inline void plan_heads(int64_t tokens, int heads, int d, int* per_wg, int* slots, int* groups) {
  const bool many = tokens >= 4 * 1024;
  *per_wg = 1;
  while (many && *per_wg < kMostTokens && *per_wg * heads * (d / 16) < 2 * kHeadThreads) *per_wg *= 2;
  *slots = many ? heads : kHeadThreads / (d / 16);
  if (*slots > heads) *slots = heads;
  *groups = (heads + *slots - 1) / *slots;
}

}  // namespace cobs

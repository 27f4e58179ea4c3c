// Attention of several query tokens a row over a cache of 8-bit floats (cobs_decode8), on the matrix cores.
//
// The M = N G query rows of one (batch row, KV head) are the columns of S^T = K Q^T and O^T = V^T P^T, a tile of
// R = 16 or 32 rows by frames of 32 tokens.  Codes become bf16, which holds each e4m3 number, in registers, and no
// tile passes through LDS.  Lane l has the query row l % R and
//   K   R = 16: the tokens l % 16 and 16 more on, R = 32: the token l % 32, and of its elements the part that 64 / R lanes share,
//       8 for a k-step; the queries' operand has its elements in the same places;
//   V   8 tokens in the order in which its probabilities come out of the first product, and the D / 16 columns
//       (D / 16)(l % 16) onwards: bytes of two tokens are paired (v_perm) before they are converted, which is the transposition;
//       for R = 32 lanes l and l ^ 16 then exchange columns for tokens (v_permlane16_swap).
// A frame of 128-element heads is 4 + 4 KB, four 16-byte and eight 8-byte loads a lane; the next frame's begin where the registers
// of this one fall free.  A block's scale of the keys multiplies the scores, that of the values the probabilities, both in fp32.
//
// A workgroup's four waves take the same R rows and different frames; the frames of a row's context are split over
// workgroups as in cobs_tree_decode.  Few rows' parts are joined by the last workgroup to leave one, others by that operator's
// kernels.  More than R rows take more workgroups, next to each other on one XCD, whose L2 gives the frames again.
//
// What bounds it, d 128, bf16 queries: one token of 16 rows of 32k tokens (4 heads a KV head): 1.07 GB in 179 us, 6.0 TB/s, HBM.
// From 32 rows on the waves' instructions: a frame of 32 rows is some 270 vector instructions (80 of them conversions)
// and 24 products of 32 cycles, and two waves a SIMD overlap little of the one with the other (16 drafted tokens of 8 heads
// over 4 contexts of 16k to 32k: 43 GFLOP, 64 with the probabilities' second part, in 98 us; vector pipes busy 63 % of the time, matrix
// pipes 39 %).  Tried for that: frames shared through LDS and converted once (64 rows over 8 x 16k tokens: 115 us for 89), tiles of 16
// rows two a wave (89 for 88), both frames' codes in registers (spills), a wave's priority raised in its products (85 for 82).
//
// The codes of tokens that take no part are cleared; a NaN in a drafted token's value, which not all queries see,
// is cleared and then reaches the rows that see it by a product of flags (spread_nan).
#pragma once

#include "tokens_device.h"

namespace cobs {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kTable8 = 256;           // frames described in LDS at a time

// A tile of R query rows.
template <int D, int R>
struct Tile8 {
  using Acc = std::conditional_t<R == 16, f32x4_t, f32x16_t>;
  static constexpr int NO = D / R;                        // products of the values: one for each column of a lane
  static constexpr int KS = R == 16 ? D / 32 : D / 16;    // k-steps of the scores
  static constexpr int TT = 32 / R;                       // products of the scores: tokens of a frame by R
  static constexpr int PS = R / 16;                       // k-steps of the values
  static constexpr int NA = R * R / 64;                   // registers of an accumulator
  static constexpr int NI = TT * NA;                      // a lane's scores of a frame
};
template <int R>
__device__ __forceinline__ auto product(sbf16x8_t a, sbf16x8_t b, typename Tile8<64, R>::Acc c) {
  if constexpr (R == 16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Token of the frame that a lane's score i stands for, less 4 (l / R): the first product's rows.
template <int R>
__host__ __device__ constexpr int score_token(int i) { return (i & 3) + (R == 16 ? 16 : 8) * (i >> 2); }
// Token of the frame whose value codes a lane holds in place j < 8.
template <int R>
__device__ __forceinline__ int value_token(int lane, int j) {
  return R == 16 ? 4 * (lane >> 4) + (j & 3) + 16 * (j >> 2) : 16 * ((lane >> 4) & 1) + 4 * (lane >> 5) + (j & 3) + 8 * (j >> 2);
}
// First of the D / R columns that row m of the second product's tiles stands for (a tile for each).
template <int D, int R>
__device__ __forceinline__ int column_of(int m) { return R == 16 ? (D / 16) * m : (D / 16) * (m & 15) + (D / 32) * (m >> 4); }

// A frame in the table: place of its first row, its position, its live rows lo .. hi - 1 (relative), its scales
// (of the keys times the softmax's, for exponents of 2).
struct alignas(16) Frame8 {
  int64_t base;
  int a;
  int16_t lo, hi;
  float ks, vs;
};

// A frame's entry in scalar registers; one past the table's end is empty (place 0, no live rows).
struct ScalarFrame {
  int64_t base;
  int a, lo, hi;
  float ks, vs;
  __device__ __forceinline__ bool empty() const { return hi <= lo; }
  __device__ __forceinline__ bool whole(int C) const { return lo == 0 && hi == kFrame && a + kFrame <= C; }
  __device__ __forceinline__ uint32_t ends() const { return (hi < kFrame ? (1u << hi) - 1u : ~0u) & (~0u << lo); }
};
__device__ __forceinline__ ScalarFrame table_frame(const Frame8* table, int fi, int cnt) {
  ScalarFrame f = {0, 0, 0, 0, 0.0f, 0.0f};
  if (fi < cnt) {
    const uint4 e = *reinterpret_cast<const uint4*>(&table[fi]);
    const float2 s = *reinterpret_cast<const float2*>(&table[fi].ks);
    const uint32_t b0 = wave_uniform32((int)e.x), b1 = wave_uniform32((int)e.y), w = wave_uniform32((int)e.w);
    f.base = (int64_t)(((uint64_t)b1 << 32) | b0);
    f.a = wave_uniform32((int)e.z);
    f.lo = (int)(int16_t)(w & 0xffff);
    f.hi = (int)(int16_t)(w >> 16);
    f.ks = __int_as_float(wave_uniform32(__float_as_int(s.x)));
    f.vs = __int_as_float(wave_uniform32(__float_as_int(s.y)));
  }
  return f;
}

// Frame `f` of a row's attended ones, as it stands in the table; empty where its page is out of range.
__device__ __forceinline__ Frame8 describe_frame(const Decode8Params& p, const Attended& x, int b, int h, int f, float c2) {
  const AttendParams& a = p.t.a;
  int fa, lo, hi;
  x.frame(f, fa, lo, hi);
  const int64_t base = hi > lo ? kv_offset(a.kv, b, h, fa) : -1;
  Frame8 e = {0, fa, 0, 0, 1.0f, 0.0f};
  if (base >= 0) {
    const int64_t at = a.kv.table ? base / ((int64_t)a.d << a.lsh) : ((int64_t)b * a.hkv + h) * a.kv.nbmax + (fa >> a.lsh);
    e.base = base;
    e.lo = (int16_t)(lo - fa);
    e.hi = (int16_t)(hi - fa);
    e.ks = fmaxf(p.k_scale[at] * c2, 1.17549435e-38f);      // (0 would make NaN of masked scores)
    e.vs = p.v_scale[at];
  }
  return e;
}

// Two codes of a register, the low or the high ones, as bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t two_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

// Codes that are NaN, as bytes of 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t m = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (m >> 7) * 0xffu;
}

// A frame's codes in a lane (D / 8 registers of each).
template <int D, int R>
__device__ __forceinline__ void load_keys(const uint8_t* k, uint32_t rs, uint32_t (&y)[D / 8]) {
  const int lane = threadIdx.x & 63;
  const uint32_t off = (uint32_t)(lane % R) * rs + (D * R / 64) * (lane / R);
  constexpr int N = D * R / 64 / 16;                       // 16-byte loads of a token
#pragma unroll
  for (int tt = 0; tt < 32 / R; ++tt)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(k + (off + (uint32_t)(16 * tt) * rs + 16 * i));
      uint32_t* const to = y + 4 * (tt * N + i);
      to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
    }
}
template <int D, int R>
__device__ __forceinline__ void load_values(const uint8_t* v, uint32_t rs, uint32_t (&y)[D / 8]) {
  const int lane = threadIdx.x & 63;
  const uint32_t off = (uint32_t)value_token<R>(lane, 0) * rs + (D / 16) * (lane & 15);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint8_t* at = v + (off + (uint32_t)score_token<R>(j) * rs);
    if constexpr (D == 128) {
      const uint2 w = *reinterpret_cast<const uint2*>(at);
      y[2 * j] = w.x;
      y[2 * j + 1] = w.y;
    } else {
      y[j] = *reinterpret_cast<const uint32_t*>(at);
    }
  }
}

// Operand number `n` of the keys (k-step n % KS of the tokens' part n / KS).
__device__ __forceinline__ sbf16x8_t key_operand(const uint32_t* y, int n) {
  const u32x4v_t kk = {two_bf16<false>(y[2 * n]), two_bf16<true>(y[2 * n]), two_bf16<false>(y[2 * n + 1]), two_bf16<true>(y[2 * n + 1])};
  return __builtin_bit_cast(sbf16x8_t, kk);
}

// Two columns of 8 tokens, whose byte pairs are in w.
__device__ __forceinline__ void two_columns(const uint32_t (&w)[4], sbf16x8_t& even, sbf16x8_t& odd) {
  u32x4v_t a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = two_bf16<false>(w[i]);
    b[i] = two_bf16<true>(w[i]);
  }
  even = __builtin_bit_cast(sbf16x8_t, a);
  odd = __builtin_bit_cast(sbf16x8_t, b);
}

// The values as A operands: put(c, k-step, operand), column by column.
template <int D, int R, typename Put>
__device__ __forceinline__ void value_operands(const uint32_t (&y)[D / 8], Put put) {
  constexpr int W = D / 64;
  // byte pairs of the tokens 2 i and 2 i + 1: the columns 2 q and 2 q + 1
  auto pair = [&](int q, int i) {
    return __builtin_amdgcn_perm(y[(2 * i + 1) * W + q / 2], y[2 * i * W + q / 2], q & 1 ? 0x07030602u : 0x05010400u);
  };
  if constexpr (R == 16) {
#pragma unroll
    for (int q = 0; q < 2 * W; ++q) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pair(q, i);
      sbf16x8_t c0, c1;
      two_columns(w, c0, c1);
      put(2 * q, 0, c0);
      put(2 * q + 1, 0, c1);
    }
  } else {
    // lanes of even rows of 16 keep the first half of the columns, those of odd ones the second; of tokens they have 8 each
#pragma unroll
    for (int q = 0; q < W; ++q) {
      uint32_t w0[4], w1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto s = __builtin_amdgcn_permlane16_swap(pair(q, i), pair(q + W, i), false, false);
        w0[i] = s[0];
        w1[i] = s[1];
      }
      sbf16x8_t c0, c1;
      two_columns(w0, c0, c1);
      put(2 * q, 0, c0);
      put(2 * q + 1, 0, c1);
      two_columns(w1, c0, c1);
      put(2 * q, 1, c0);
      put(2 * q + 1, 1, c1);
    }
  }
}

// Eight elements of an fp32 query as three bf16 parts, by truncation: they hold all 24 bits, none overflows, and what
// is not finite is the first part alone (an infinity's scores are those of plain arithmetic).
__device__ __forceinline__ void split_query(const float (&x)[8], sbf16x8_t (&out)[3]) {
  u32x4v_t w[3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t part[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float v = x[2 * j + i];
      const uint32_t hi = v == v ? __float_as_uint(v) & 0xffff0000u : 0x7fc00000u;
      const float r = fabsf(v) < INFINITY ? v - __uint_as_float(hi) : 0.0f;
      const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
      part[i][0] = hi;
      part[i][1] = mid;
      part[i][2] = __float_as_uint(r - __uint_as_float(mid));
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) w[k][j] = (part[0][k] >> 16) | (part[1][k] & 0xffff0000u);
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) out[k] = __builtin_bit_cast(sbf16x8_t, w[k]);
}

// k-step ks of a query row as the B operand, in parts.
template <int D, int R, int PARTS>
__device__ __forceinline__ void load_query(const AttendParams& a, const QueryRow& q, int ks, sbf16x8_t (&out)[PARTS]) {
  const int64_t at = q.at * D + (D * R / 64) * ((threadIdx.x & 63) / R) + 8 * ks;
  if constexpr (PARTS == 1) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (q.live) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at);
    out[0] = __builtin_bit_cast(sbf16x8_t, w);
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    if (q.live) {
      const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at);
      const float4 s0 = s[0], s1 = s[1];
      v[0] = s0.x; v[1] = s0.y; v[2] = s0.z; v[3] = s0.w;
      v[4] = s1.x; v[5] = s1.y; v[6] = s1.z; v[7] = s1.w;
    }
    split_query(v, out);
  }
}

// Bits of the frame's tokens that a query row sees, the lane's at score_token(i).  to_c: tokens of the context.
template <int R>
__device__ __forceinline__ uint32_t visible_tokens(uint64_t bits, int to_c, uint32_t ends) {
  uint32_t u = to_c >= kFrame ? ~0u : (to_c > 0 ? (1u << to_c) - 1u : 0u);
  u |= to_c >= kFrame ? 0u : (uint32_t)(to_c > 0 ? bits << to_c : bits >> -to_c);
  return (u & ends) >> (4 * ((threadIdx.x & 63) / R));
}

// Values of tokens that take no part cleared, and NaN of drafted tokens (those from to_c on), as 0 times it would reach
// every row; whether there was any.
template <int D, int R>
__device__ __forceinline__ bool clear_dead(uint32_t (&y)[D / 8], uint32_t ends, int to_c) {
  uint32_t bad = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = value_token<R>(threadIdx.x & 63, j);
    const bool live = (ends >> t) & 1u;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      uint32_t& w = y[j * (D / 64) + i];
      w = live ? w : 0u;
      const uint32_t nan = t >= to_c ? nan_bytes(w) : 0u;
      w &= ~nan;
      bad |= nan;
    }
  }
  return __ballot(bad != 0) != 0;
}

// NaN among the values of drafted tokens, into the outputs of the rows that see such a token, whose number a product of
// flags gives.
template <int D, int R>
__device__ __forceinline__ void spread_nan(const uint32_t (&y)[D / 8], int to_c, uint32_t vis, typename Tile8<D, R>::Acc (&o)[D / R]) {
  using T = Tile8<D, R>;
  sbf16x8_t see[T::PS];
#pragma unroll
  for (int ks = 0; ks < T::PS; ++ks) {
    u32x4v_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = score_token<R>(8 * ks + 2 * i);
      w[i] = ((vis >> t) & 1u ? 0x3f80u : 0u) | ((vis >> (t + 1)) & 1u ? 0x3f800000u : 0u);
    }
    see[ks] = __builtin_bit_cast(sbf16x8_t, w);
  }
  uint32_t flag[D / 8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint32_t nan = value_token<R>(threadIdx.x & 63, j) >= to_c ? nan_bytes(y[j * (D / 64) + i]) : 0u;
      flag[j * (D / 64) + i] = nan & 0x38383838u;         // 1 in e4m3
    }
  value_operands<D, R>(flag, [&](int c, int ks, sbf16x8_t v) {
    typename T::Acc n;
#pragma unroll
    for (int i = 0; i < T::NA; ++i) n[i] = 0.0f;
    n = product<R>(v, see[ks], n);
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
      if (n[i] > 0.0f) o[c][i] = __uint_as_float(0x7fc00000u);
  });
}

// The maximum over the lanes that hold a row's tokens.
template <int R>
__device__ __forceinline__ float row_max(float x) {
  if constexpr (R == 16) x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, other_half(x));
}

// Streaming softmax of a tile, after its maximum: x the lane's scores of its row, m the row's maximum and l its sum (of the lane's
// own tokens) in the log2 domain; pb: the probabilities times the values' scale as the B operands.
template <int R, int PP>
__device__ __forceinline__ void softmax_tile(float (&x)[R / 2], float ks, float vs, float m, float& l, sbf16x8_t (&pb)[R / 16][PP]) {
  constexpr int NI = R / 2;
  const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < NI; ++j) x[j] = __builtin_amdgcn_exp2f(fmaf(x[j], ks, -ref));
  float sum[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
  for (int j = 4; j < NI; ++j) sum[j & 3] += x[j];
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
  for (int k = 0; k < R / 16; ++k) {
    float pv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) pv[j] = x[8 * k + j] * vs;
    split_bf16x8<PP>(pv, pb[k]);
  }
}

// A row's outputs at element d (a multiple of 4): sums, maximum mm (-inf: no score above that) and total.
template <int D>
__device__ __forceinline__ void finish_row(const TreeParams& p, const TreePart& part, int row, int d, float4 sum, float mm, float total) {
  const AttendParams& a = p.a;
  const int i = row / a.G;
  const int64_t at = ((int64_t)part.b * a.N + i) * a.hq + part.h * a.G + (row - i * a.G);
  store_row4(p.out, at * D + d, sum, total, a.io_bf16);
  if (d == 0 && p.lse)
    p.lse[at] = total != 0.0f ? (mm == -INFINITY ? 0.0f : mm) * 0.6931471805599453f + logf(total) : -INFINITY;
}

// Its part of them, written through to where any XCD reads it if the last workgroup joins the parts.
template <int D>
__device__ __forceinline__ void leave_part(const TreeParams& p, const TreePart& part, bool joined, int row, int d, float4 sum, float mm,
                                           float total) {
  const int64_t at = part_row(p, part, row);
  float* const o = p.part_o + at * D + d;
  float* const ml = p.part_ml + 2 * at;
  if (joined) {
    st_agent(o, sum.x); st_agent(o + 1, sum.y); st_agent(o + 2, sum.z); st_agent(o + 3, sum.w);
    if (d == 0) { st_agent(ml, mm); st_agent(ml + 1, total); }
  } else {
    *reinterpret_cast<float4*>(o) = sum;
    if (d == 0) *reinterpret_cast<float2*>(ml) = make_float2(mm, total);
  }
}

// The `rows` rows of a (row, KV head) out of its parts, by the workgroup that is the last to leave one: in the parts' order.
template <int D>
__device__ __forceinline__ void join_parts(const TreeParams& p, const TreePart& part, int rows) {
  constexpr int U = 8;                                   // parts whose loads are under way together
  const int M = p.a.N * p.a.G;
  const int64_t first = part.first * M;
  const __amdgpu_buffer_rsrc_t ml = coherent_view(p.part_ml + 2 * first, (uint32_t)(part.n * M * 8));
  const __amdgpu_buffer_rsrc_t o = coherent_view(p.part_o + first * D, (uint32_t)(part.n * M * D * 4));
  for (int idx = threadIdx.x; idx < rows * (D / 4); idx += kTreeThreads) {
    const int row = idx / (D / 4), d4 = idx % (D / 4);
    float top = -INFINITY, total = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k0 = 0; k0 < part.n; k0 += U) {
      float2 w[U];
      float4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t at = (uint32_t)(min(k0 + u, part.n - 1) * M + row);
        w[u] = ld_coherent2(ml, at * 8);
        y[u] = ld_coherent4(o, at * (D * 4) + d4 * 16);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k0 + u >= part.n) continue;
        const float mn = fmaxf(top, w[u].x), ref = mn == -INFINITY ? 0.0f : mn;
        const float f = __builtin_amdgcn_exp2f(top - ref), g = __builtin_amdgcn_exp2f(w[u].x - ref);
        top = mn;
        total = total * f + w[u].y * g;
        sum.x = sum.x * f + y[u].x * g; sum.y = sum.y * f + y[u].y * g;
        sum.z = sum.z * f + y[u].z * g; sum.w = sum.w * f + y[u].w * g;
      }
    }
    finish_row<D>(p, part, row, 4 * d4, sum, top, total);
  }
}

// bf16 parts of a probability: three, which hold all its bits, or two (2^-17) where the query is bf16 and the product's time counts.  Tiles of 16
// rows wait for memory, and the third part costs a percent at most (one token of 16 rows of 32k tokens 183.5 us, with two parts 182.7; of 64-element heads 99.3
// and 98.4; 1 row of 1k tokens 11.4 and 11.4);
// tiles of 32 rows wait for the waves' instructions (16 drafted tokens of 8 heads over 4 contexts of 16k to 32k: 126 us with three, 108 with two).
template <int PARTS, int R>
constexpr int kProbabilityParts = PARTS == 3 || R == 16 ? 3 : 2;

// Workgroups that a CU takes: three where they need not spill for it (64 rows over 8 x 16k tokens of 64-element heads: 54 us,
// by two 61).
template <int D, int PARTS, int R>
constexpr int kWorkgroups8 = D == 64 && (PARTS == 1 || R == 16) ? 3 : 2;

template <int D, int PARTS, int R>
__global__ __launch_bounds__(kTreeThreads, (kWorkgroups8<D, PARTS, R>)) void decode8_kernel(Decode8Params p) {
  using T = Tile8<D, R>;
  constexpr int WT = 4, KS = T::KS, NO = T::NO, PP = kProbabilityParts<PARTS, R>;
  constexpr bool SHARED = D == 128 && R == 32 && PARTS == 3;      // the queries' operands in LDS (the pool's place): in registers they spill
  __shared__ Frame8 table[kTable8];
  __shared__ __align__(16) float pool[WT * R * D];
  __shared__ float s_m[WT][R], s_l[WT][R];
  __shared__ int red[4];
  static_assert(!SHARED || PARTS * KS * 64 * 16 <= WT * R * D * 4, "room for the queries");

  const TreeParams& tp = p.t;
  const AttendParams& a = tp.a;
  // Workgroups go round-robin to the 8 XCDs; the row tiles of one part of the
  // context, which read the same keys and values, follow each other on one.
  const int slot = blockIdx.x >> 3, group = (slot / tp.mtiles) * 8 + (blockIdx.x & 7), mt = slot % tp.mtiles;
  if (group >= tp.units * tp.nsplit) return;
  TreePart part;
  if (!tree_part(tp, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane % R;

  const QueryRow q = query_row(a, b, h, mt * R + lr);
  sbf16x8_t* const q_lds = reinterpret_cast<sbf16x8_t*>(pool) + lane;      // [KS][PARTS][64]
  sbf16x8_t qb[SHARED ? 1 : KS][PARTS];
  if constexpr (SHARED) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if ((ks & 3) != wave) continue;
      load_query<D, R, PARTS>(a, q, ks, qb[0]);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) q_lds[(ks * PARTS + k) * 64] = qb[0][k];
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_query<D, R, PARTS>(a, q, ks, qb[ks]);
  }

  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (tp.nsplit == 1 || (p.counters && part.split == 0)) clear_padding<D>(tp, b, h, mt * R, R, x.nq);
  if (mt * R >= x.nq * a.G) return;                       // the tile's rows are all padding

  typename T::Acc o[NO];
#pragma unroll
  for (int c = 0; c < NO; ++c)
#pragma unroll
    for (int i = 0; i < T::NA; ++i) o[c][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  const int nf = x.frames(), all = (nf + WT - 1) / WT;
  const int f_lo = first_pass(all, part.split, part.n) * WT, f_hi = min(first_pass(all, part.split + 1, part.n) * WT, nf);
  const uint32_t rs = (uint32_t)(a.kv.table ? D : a.kv.st);      // (at most 2^22 bytes a row: 32 rows below 2^32)
  const float c2 = a.c * 1.4426950408889634f;
  const uint8_t* const kp = static_cast<const uint8_t*>(a.kv.k);
  const uint8_t* const vp = static_cast<const uint8_t*>(a.kv.v);

  bool nan = false;                                     // whether a drafted token's value was
  uint32_t ky[D / 8], vy[D / 8];
  auto scores = [&](float (&s)[T::NI]) {
#pragma unroll
    for (int tt = 0; tt < T::TT; ++tt) {
      typename T::Acc z;
#pragma unroll
      for (int i = 0; i < T::NA; ++i) z[i] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const sbf16x8_t kk = key_operand(ky, tt * KS + ks);
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k) z = product<R>(kk, SHARED ? q_lds[(ks * PARTS + k) * 64] : qb[SHARED ? 0 : ks][k], z);
      }
#pragma unroll
      for (int i = 0; i < T::NA; ++i) s[tt * T::NA + i] = z[i];
    }
  };

  for (int t0 = f_lo; t0 < f_hi; t0 += kTable8) {
    const int cnt = min(kTable8, f_hi - t0);
    __syncthreads();                                    // the table is free; the queries are there
    if (tid < cnt) table[tid] = describe_frame(p, x, b, h, t0 + tid, c2);
    __syncthreads();
    // A frame's scores are computed while the softmax of the one before runs.  Loads begin where their registers fall free, a frame's
    // keys before the values of the frame before it.  There is always a next frame (past the end at place 0, the cache's first
    // rows): were loads left out on some path, or in another order before the loop, the waits in it would be for all loads
    // under way instead of the older ones.
    ScalarFrame f = table_frame(table, wave, cnt), next = table_frame(table, wave + WT, cnt);
    float s[T::NI];
    load_keys<D, R>(kp + f.base, rs, ky);
    scores(s);
    load_keys<D, R>(kp + next.base, rs, ky);
    __builtin_amdgcn_sched_barrier(0);
    load_values<D, R>(vp + f.base, rs, vy);
    int it = wave;
    while (it < cnt) {
      float top;
      while (true) {
        if (!f.whole(x.C)) {
          asm volatile("");                             // (nothing of this is for the other frames)
          const int to_c = x.C - f.a;
          const uint32_t vis = visible_tokens<R>(q.bits, to_c, f.ends());
          nan |= clear_dead<D, R>(vy, f.ends(), to_c);
#pragma unroll
          for (int j = 0; j < T::NI; ++j) s[j] = (vis >> score_token<R>(j)) & 1u ? s[j] : -INFINITY;
        }
        // (f.ks > 0, so the largest score is the largest product)
        top = s[0];
#pragma unroll
        for (int j = 1; j < T::NI; ++j) top = fmaxf(top, s[j]);
        top *= f.ks;
        // The maximum is followed with a slack of 2^8 in the probabilities, so that few frames raise it and scale the outputs
        // anew, outside of this loop, which changes the outputs by products alone (a path that scales them in it costs
        // copies of them all in each frame).
        if (__ballot(top > m + 8.0f)) break;
        const ScalarFrame after = table_frame(table, it + 2 * WT, cnt);
        float z[T::NI];
        scores(z);
        load_keys<D, R>(kp + after.base, rs, ky);
        __builtin_amdgcn_sched_barrier(0x40f);          // (arithmetic may cross: the compiler would move the loads to the loop's end)
        sbf16x8_t pb[T::PS][PP];
        softmax_tile<R, PP>(s, f.ks, f.vs, m, l, pb);
        value_operands<D, R>(vy, [&](int c, int ks, sbf16x8_t v) {
#pragma unroll
          for (int k = PP - 1; k >= 0; --k) o[c] = product<R>(v, pb[ks][k], o[c]);
        });
        load_values<D, R>(vp + next.base, rs, vy);
#pragma unroll
        for (int j = 0; j < T::NI; ++j) s[j] = z[j];
        f = next;
        next = after;
        it += WT;
        if (it >= cnt) break;
      }
      if (it < cnt) {
        const float mn = fmaxf(m, row_max<R>(top)), alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
        m = mn;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NO; ++c) o[c] *= alpha;
      }
    }
  }

  // The frames of the draft once more (the last two or three; after the loop, as outputs that change on a rare path in it cost copies of
  // all of them in each frame).
  if (__builtin_expect(nan, 0)) {
    for (int f = f_lo + max(0, (f_hi - f_lo - 4 * WT) / WT * WT) + wave; f < f_hi; f += WT) {
      const Frame8 e = describe_frame(p, x, b, h, f, c2);
      const int to_c = x.C - e.a;
      if (e.hi <= e.lo || e.hi <= to_c) continue;
      const uint32_t ends = (e.hi < kFrame ? (1u << e.hi) - 1u : ~0u) & (~0u << e.lo);
      uint32_t y[D / 8];
      load_values<D, R>(vp + e.base, rs, y);
      spread_nan<D, R>(y, to_c, visible_tokens<R>(q.bits, to_c, ends), o);
    }
  }

  // ---- join the waves, in order
  if constexpr (R == 16) l += __shfl_xor(l, 16, 64);
  l += other_half(l);
  __syncthreads();                                      // the pool is free
  if (lane < R) {
    s_m[wave][lr] = m;
    s_l[wave][lr] = l;
  }
  __syncthreads();
  {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < WT; ++t) top = fmaxf(top, s_m[t][lr]);
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    float* const wo = pool + (wave * R + lr) * D;
    auto put = [&](int d, float y0, float y1, float y2, float y3) {
      *reinterpret_cast<float4*>(wo + 4 * ((d / 4) ^ (lane & 15))) = make_float4(y0 * f, y1 * f, y2 * f, y3 * f);
    };
    // row 4 (l / R) + score_token(i) of each tile c: the column column_of() + c
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
      const int d = column_of<D, R>(4 * (lane / R) + score_token<R>(i));
      if constexpr (NO >= 4) {
#pragma unroll
        for (int c = 0; c < NO; c += 4) put(d + c, o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]);
      } else {
        // (two columns of row m, the next two are those of row m + 16)
        if (i < 8) put(d, o[0][i], o[1][i], o[0][i + 8], o[1][i + 8]);
      }
    }
  }
  __syncthreads();
  for (int idx = tid; idx < R * (D / 4); idx += kTreeThreads) {
    const int r = idx / (D / 4), d4 = idx % (D / 4), row = mt * R + r;
    if (row >= x.nq * a.G) continue;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int t = 0; t < WT; ++t) mm = fmaxf(mm, s_m[t][r]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int t = 0; t < WT; ++t) {
      ll += __builtin_amdgcn_exp2f(s_m[t][r] - ref) * s_l[t][r];
      const float4 y = *reinterpret_cast<const float4*>(pool + (t * R + r) * D + 4 * (d4 ^ (r & 15)));
      sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
    }
    if (tp.nsplit == 1) finish_row<D>(tp, part, row, 4 * d4, sum, mm, ll);
    else leave_part<D>(tp, part, p.counters != nullptr, row, 4 * d4, sum, mm, ll);
  }
  if (p.counters && arrive_last(p.counters + b * a.hkv + h, part.n, red)) join_parts<D>(tp, part, x.nq * a.G);
}

}  // namespace cobs

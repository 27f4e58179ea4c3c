// Attention of several query tokens a row over a cache of 8-bit floats (cobs_decode8), on the matrix cores.
//
// The M = N G query rows of one (batch row, KV head) are the columns of S^T = K Q^T and O^T = V^T P^T, in tiles
// of 16 rows by frames of 32 tokens (16x16x32 products).  Codes become bf16, which holds each e4m3 number, in
// registers, and no tile passes through LDS:
//   K   lane l takes token l % 16 (and 16 more on) and elements (D / 4)(l / 16) onwards, 8 for a k-step, and Q's operand
//       has its elements in the same places;
//   V   a lane takes 8 tokens, 4 (l / 16) + 0..3 and 16 more on, as its probabilities come out of the first product, and
//       the D / 16 columns (D / 16)(l % 16) onwards: bytes of two tokens are paired (v_perm) before they are
//       converted, which is the transposition; product c has column (D / 16) m + c as its row m.
// A frame of 128-element heads is 4 + 4 KB, two or four 16-byte and eight 8-byte loads a lane, the next frame's under way.
// A block's scale of the keys multiplies the scores, that of the values the probabilities, both in fp32.
//
// Up to 32 rows are bound by the cache's bytes: a workgroup's waves take different frames (decode8_kernel).  Many rows
// are bound by the products and their softmax: the waves take different rows and share the frames (decode8_many_kernel).
// The frames of a row's context are split over workgroups as in cobs_tree_decode, whose kernels join the parts.
//
// The codes of tokens that take no part are cleared; a NaN in a drafted token's value, which not all queries see,
// is cleared and then reaches the rows that see it by a product of flags (spread_nan).
#pragma once

#include "tokens_device.h"

namespace cobs {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTable8 = 256;           // frames described in LDS at a time

// A frame in the table: place of its first row, its position, its live rows lo .. hi - 1 (relative), its scales
// (of the keys times the softmax's, for exponents of 2).
struct alignas(16) Frame8 {
  int64_t base;
  int a;
  int16_t lo, hi;
  float ks, vs;
};

// Two codes of a register, the low or the high ones, as bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t two_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

// Codes of 8 tokens in one column: of the tokens' registers x[0..7], byte pair `c` (columns 2c and 2c + 1 of 4).
// a: bytes of the even column, b: those of the odd one, each for the tokens 2i and 2i + 1 in register i.
template <bool HIGH>
__device__ __forceinline__ void columns(const uint32_t (&x)[8], sbf16x8_t& even, sbf16x8_t& odd) {
  u32x4v_t a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], HIGH ? 0x07030602u : 0x05010400u);
    a[i] = two_bf16<false>(w);
    b[i] = two_bf16<true>(w);
  }
  even = __builtin_bit_cast(sbf16x8_t, a);
  odd = __builtin_bit_cast(sbf16x8_t, b);
}

// Codes that are NaN, as bytes of 0xff (0x80 of each byte's sum, spread).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t m = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (m >> 7) * 0xffu;
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

// NaN among the values of drafted tokens (a frame's tokens from to_c on) cleared.
template <int D>
__device__ __forceinline__ void drop_nan(uint32_t (&v)[D / 8], int to_c) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
      if (4 * (int)((threadIdx.x & 63) >> 4) + (j & 3) + 16 * (j >> 2) >= to_c) v[j * (D / 64) + i] &= ~nan_bytes(v[j * (D / 64) + i]);
}

// NaN among the values of drafted tokens (a frame's tokens from to_c on): cleared, as 0 times it would reach
// every row, and put into the outputs of the rows that see such a token, whose number a product of flags gives.
template <int D, int QT>
__device__ __forceinline__ void spread_nan(uint32_t (&v)[D / 8], int to_c, const uint32_t (&vis)[QT], f32x4_t (&o)[QT][D / 16]) {
  const int g = (threadIdx.x & 63) >> 4;
  sbf16x8_t see[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    u32x4v_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = ((2 * i) & 3) + 16 * (i >> 1);
      w[i] = ((vis[qt] >> t) & 1u ? 0x3f80u : 0u) | ((vis[qt] >> (t + 1)) & 1u ? 0x3f800000u : 0u);
    }
    see[qt] = __builtin_bit_cast(sbf16x8_t, w);
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    uint32_t flag[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t nan = 4 * g + (j & 3) + 16 * (j >> 2) >= to_c ? nan_bytes(v[j * (D / 64) + i]) : 0u;
      v[j * (D / 64) + i] &= ~nan;
      flag[j] = nan & 0x38383838u;                        // 1 in e4m3
    }
    sbf16x8_t c[4];
    columns<false>(flag, c[0], c[1]);
    columns<true>(flag, c[2], c[3]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const f32x4_t n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[k], see[qt], f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n[r] > 0.0f) o[qt][4 * i + k][r] = __uint_as_float(0x7fc00000u);
      }
  }
}

// Bits of the frame's tokens that a query row sees (bit t: token t), those of the lane's 8 tokens at 0..3 and 16..19.
__device__ __forceinline__ uint32_t visible_tokens(uint64_t bits, int to_c, uint32_t ends) {
  uint32_t u = to_c >= kFrame ? ~0u : (to_c > 0 ? (1u << to_c) - 1u : 0u);      // (to_c: tokens of the context)
  u |= to_c >= kFrame ? 0u : (uint32_t)(to_c > 0 ? bits << to_c : bits >> -to_c);
  return (u & ends) >> (4 * ((threadIdx.x & 63) >> 4));
}

// Streaming softmax of a tile: scores s of 8 tokens of the row l % 16 in a lane; pb: the probabilities times the values'
// scale as the B operand.  Maximum m and sum l (of the lane's own tokens) are those of the scores in the log2 domain.  The maximum is
// followed with a slack of 2^8 in the probabilities, so that few frames exchange maxima and scale the outputs anew.
// (ks >= 0, so the largest score is the largest product.)
template <int NC, int PP>
__device__ __forceinline__ void softmax_tile(const f32x4_t (&s)[2], float ks, float vs, bool whole, uint32_t vis, float& m, float& l,
                                             f32x4_t (&o)[NC], sbf16x8_t (&pb)[PP]) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = s[j >> 2][j & 3];
  float top;
  if (whole) {
    top = fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(x[3], x[4])), fmaxf(fmaxf(x[5], x[6]), x[7]));
  } else {
    top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, (vis >> ((j & 3) + 16 * (j >> 2))) & 1u ? x[j] : -INFINITY);
  }
  top *= ks;
  if (__ballot(top > m + 8.0f)) {
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
    m = mn;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] *= alpha;
  }
  const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(fmaf(x[j], ks, -ref));
  if (!whole) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (vis >> ((j & 3) + 16 * (j >> 2))) & 1u ? x[j] : 0.0f;
  }
  l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] *= vs;
  split_bf16x8<PP>(x, pb);
}

// The queries' operand of one tile: column l % 16, elements (D / 4)(l / 16) + 8 ks + j; the row's drafted tokens.
template <int D, int PARTS>
__device__ __forceinline__ uint64_t load_queries(const AttendParams& a, int b, int h, int row, sbf16x8_t (&out)[D / 32][PARTS]) {
  const int lane = threadIdx.x & 63;
  const QueryRow q = query_row(a, b, h, row + (lane & 15));
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    const int64_t at = q.at * D + (D / 4) * (lane >> 4) + 8 * ks;
    if constexpr (PARTS == 1) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (q.live) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at);
      out[ks][0] = __builtin_bit_cast(sbf16x8_t, w);
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
      split_query(v, out[ks]);
    }
  }
  return q.bits;
}

// Frame `f` of a row's attended ones, as it stands in the table; empty where its page is out of range.
__device__ __forceinline__ Frame8 describe_frame(const Decode8Params& p, const Attended& x, int b, int h, int f, float c2) {
  const AttendParams& a = p.t.a;
  int fa, lo, hi;
  x.frame(f, fa, lo, hi);
  const int64_t base = hi > lo ? kv_offset(a.kv, b, h, fa) : -1;
  Frame8 e = {0, fa, 0, 0, 0.0f, 0.0f};
  if (base >= 0) {
    const int64_t at = a.kv.table ? base / ((int64_t)a.d << a.lsh) : ((int64_t)b * a.hkv + h) * a.kv.nbmax + (fa >> a.lsh);
    e.base = base;
    e.lo = (int16_t)(lo - fa);
    e.hi = (int16_t)(hi - fa);
    e.ks = p.k_scale[at] * c2;
    e.vs = p.v_scale[at];
  }
  return e;
}

// A frame's entry in scalar registers; one past the table's end is empty.
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

// A frame's codes in a lane: keys of tokens l % 16 (and 16 more on), or values of 8 tokens.
template <int D>
__device__ __forceinline__ void load_keys(const uint8_t* k, uint32_t rs, uint32_t (&y)[D / 8]) {
  const int lane = threadIdx.x & 63;
  const uint32_t off = (uint32_t)(lane & 15) * rs + (D / 4) * (lane >> 4);
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(k + (off + (uint32_t)(16 * tt) * rs + 16 * i));
      uint32_t* const to = y + 4 * (tt * (D / 64) + i);
      to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
    }
}
template <int D>
__device__ __forceinline__ void load_values(const uint8_t* v, uint32_t rs, uint32_t (&y)[D / 8]) {
  const int lane = threadIdx.x & 63;
  const uint32_t off = (uint32_t)(4 * (lane >> 4)) * rs + (D / 16) * (lane & 15);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint8_t* at = v + (off + (uint32_t)((j & 3) + 16 * (j >> 2)) * rs);
    if constexpr (D == 128) {
      const uint2 w = *reinterpret_cast<const uint2*>(at);
      y[2 * j] = w.x;
      y[2 * j + 1] = w.y;
    } else {
      y[j] = *reinterpret_cast<const uint32_t*>(at);
    }
  }
}

// k-step ks of the keys of tile tt as the A operand.
template <int D>
__device__ __forceinline__ sbf16x8_t key_operand(const uint32_t (&y)[D / 8], int tt, int ks) {
  const uint32_t w0 = y[tt * (D / 16) + 2 * ks], w1 = y[tt * (D / 16) + 2 * ks + 1];
  const u32x4v_t kk = {two_bf16<false>(w0), two_bf16<true>(w0), two_bf16<false>(w1), two_bf16<true>(w1)};
  return __builtin_bit_cast(sbf16x8_t, kk);
}

// The values of columns (D / 16) m + c as the A operands c, one after the other.
template <int D, typename Put>
__device__ __forceinline__ void value_operands(const uint32_t (&y)[D / 8], Put put) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = y[j * (D / 64) + i];
    sbf16x8_t c0, c1, c2, c3;
    columns<false>(w, c0, c1);
    columns<true>(w, c2, c3);
    put(4 * i, c0);
    put(4 * i + 1, c1);
    put(4 * i + 2, c2);
    put(4 * i + 3, c3);
  }
}

// Values of tokens that take no part cleared; whether a drafted one of the others is NaN.
template <int D>
__device__ __forceinline__ bool clear_dead(uint32_t (&y)[D / 8], uint32_t ends, int to_c) {
  const int g = (threadIdx.x & 63) >> 4;
  uint32_t bad = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = 4 * g + (j & 3) + 16 * (j >> 2);
    const bool live = (ends >> t) & 1u, drafted = t >= to_c;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      y[j * (D / 64) + i] = live ? y[j * (D / 64) + i] : 0u;
      bad |= drafted ? nan_bytes(y[j * (D / 64) + i]) : 0u;
    }
  }
  return __ballot(bad != 0) != 0;
}

// A row's outputs, or its part of them, at element d (a multiple of 4): sums, maximum mm (-inf: no score above that) and total.
template <int D>
__device__ __forceinline__ void leave_row(const TreeParams& p, const TreePart& part, int row, int d, float4 sum, float mm, float total) {
  const AttendParams& a = p.a;
  if (p.nsplit == 1) {
    const int i = row / a.G;
    const int64_t at = ((int64_t)part.b * a.N + i) * a.hq + part.h * a.G + (row - i * a.G);
    store_row4(p.out, at * D + d, sum, total, a.io_bf16);
    if (d == 0 && p.lse)
      p.lse[at] = total != 0.0f ? (mm == -INFINITY ? 0.0f : mm) * 0.6931471805599453f + logf(total) : -INFINITY;
  } else {
    const int64_t at = part_row(p, part, row);
    *reinterpret_cast<float4*>(p.part_o + at * D + d) = sum;
    if (d == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(mm, total);
  }
}

// The sum over the four lanes that hold a row's tokens.
__device__ __forceinline__ float row_total(float l) {
  l += __shfl_xor(l, 16, 64);
  return l + __shfl_xor(l, 32, 64);
}

// Few rows: the four waves take the same 16 QT rows and different frames, whose codes stay in registers.
template <int D, int PARTS, int QT>
__global__ __launch_bounds__(kTreeThreads, 2) void decode8_kernel(Decode8Params p) {
  constexpr int WT = 4, ROWS = 16 * QT;
  constexpr int KS = D / 32, NC = D / 16, PP = PARTS == 3 ? 3 : 2;
  __shared__ Frame8 table[kTable8];
  __shared__ __align__(16) float pool[WT * ROWS * D];
  __shared__ float s_m[WT][ROWS], s_l[WT][ROWS];
  __shared__ int red[4];

  const TreeParams& tp = p.t;
  const AttendParams& a = tp.a;
  const int slot = blockIdx.x >> 3, group = (slot / tp.mtiles) * 8 + (blockIdx.x & 7), mt = slot % tp.mtiles;
  if (group >= tp.units * tp.nsplit) return;
  TreePart part;
  if (!tree_part(tp, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;

  sbf16x8_t qb[QT][KS][PARTS];
  uint64_t bits[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) bits[qt] = load_queries<D, PARTS>(a, b, h, mt * ROWS + 16 * qt, qb[qt]);

  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (tp.nsplit == 1) clear_padding<D>(tp, b, h, mt * ROWS, ROWS, x.nq);
  if (mt * ROWS >= x.nq * a.G) return;                    // the tile's rows are all padding

  f32x4_t o[QT][NC];
  float m[QT], l[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m[qt] = -INFINITY;
    l[qt] = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[qt][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const int nf = x.frames(), all = (nf + WT - 1) / WT;
  const int f_lo = first_pass(all, part.split, part.n) * WT, f_hi = min(first_pass(all, part.split + 1, part.n) * WT, nf);
  const uint32_t rs = (uint32_t)(a.kv.table ? D : a.kv.st);      // (at most 2^22 bytes a row: 32 rows below 2^32)
  const float c2 = a.c * 1.4426950408889634f;
  const uint8_t* const kp = static_cast<const uint8_t*>(a.kv.k);
  const uint8_t* const vp = static_cast<const uint8_t*>(a.kv.v);

  uint32_t ky[D / 8], vy[D / 8];
  // A frame's codes, and the next one's, whose loads begin where its registers fall free.
  auto attend = [&](const ScalarFrame& f, const ScalarFrame& next) {
    if (f.empty()) {
      if (!next.empty()) { load_keys<D>(kp + next.base, rs, ky); load_values<D>(vp + next.base, rs, vy); }
      return;
    }
    const bool whole = f.whole(x.C);
    f32x4_t s[QT][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) s[qt][tt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const sbf16x8_t kk = key_operand<D>(ky, tt, ks);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k) s[qt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qb[qt][ks][k], s[qt][tt], 0, 0, 0);
      }
    }
    if (!next.empty()) load_keys<D>(kp + next.base, rs, ky);
    uint32_t vis[QT];
    if (!whole) {
      const int to_c = x.C - f.a;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) vis[qt] = visible_tokens(bits[qt], to_c, f.ends());
      if (__builtin_expect(clear_dead<D>(vy, f.ends(), to_c), 0)) spread_nan<D, QT>(vy, to_c, vis, o);
    }
    sbf16x8_t pb[QT][PP];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) softmax_tile<NC, PP>(s[qt], f.ks, f.vs, whole, vis[qt], m[qt], l[qt], o[qt], pb[qt]);
    value_operands<D>(vy, [&](int c, sbf16x8_t v) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int k = PP - 1; k >= 0; --k) o[qt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[qt][k], o[qt][c], 0, 0, 0);
    });
    if (!next.empty()) load_values<D>(vp + next.base, rs, vy);
  };

  for (int t0 = f_lo; t0 < f_hi; t0 += kTable8) {
    const int cnt = min(kTable8, f_hi - t0);
    __syncthreads();                                    // the table is free
    if (tid < cnt) table[tid] = describe_frame(p, x, b, h, t0 + tid, c2);
    __syncthreads();
    ScalarFrame now = table_frame(table, wave, cnt);
    if (!now.empty()) { load_keys<D>(kp + now.base, rs, ky); load_values<D>(vp + now.base, rs, vy); }
    for (int it = wave; it < cnt; it += WT) {
      const ScalarFrame next = table_frame(table, it + WT, cnt);
      attend(now, next);
      now = next;
    }
  }

  // ---- join the waves, in order
  __syncthreads();
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const float total = row_total(l[qt]);
    if (g == 0) {
      s_m[wave][16 * qt + l16] = m[qt];
      s_l[wave][16 * qt + l16] = total;
    }
  }
  __syncthreads();
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r16 = 16 * qt + l16;
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < WT; ++t) top = fmaxf(top, s_m[t][r16]);
    const float f = __builtin_amdgcn_exp2f(m[qt] - (top == -INFINITY ? 0.0f : top));
    float* const wo = pool + (wave * ROWS + r16) * D;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < NC; c += 4) {
        const int d4 = (NC * (4 * g + r) + c) / 4;
        *reinterpret_cast<float4*>(wo + 4 * (d4 ^ l16)) =
            make_float4(o[qt][c][r] * f, o[qt][c + 1][r] * f, o[qt][c + 2][r] * f, o[qt][c + 3][r] * f);
      }
  }
  __syncthreads();
  for (int idx = tid; idx < ROWS * (D / 4); idx += kTreeThreads) {
    const int r = idx / (D / 4), d4 = idx % (D / 4), row = mt * ROWS + r;
    if (row >= x.nq * a.G) continue;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int t = 0; t < WT; ++t) mm = fmaxf(mm, s_m[t][r]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int t = 0; t < WT; ++t) {
      ll += __builtin_amdgcn_exp2f(s_m[t][r] - ref) * s_l[t][r];
      const float4 y = *reinterpret_cast<const float4*>(pool + (t * ROWS + r) * D + 4 * (d4 ^ (r & 15)));
      sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
    }
    leave_row<D>(tp, part, row, 4 * d4, sum, mm, ll);
  }
}

// Many rows: the four waves take 16 QT rows each and all frames, which they share through LDS as bf16 operands, in the
// order in which the products' lanes take them (16 bytes a lane, so neither writes nor reads meet on a bank).  In
// a pass of two frames each wave stages one frame's keys or its values: loaded two passes ahead into registers, converted
// and written to LDS one pass ahead.
template <int D, int PARTS, int QT>
__global__ __launch_bounds__(kTreeThreads, 2) void decode8_many_kernel(Decode8Params p) {
  constexpr int ROWS = 64 * QT, FPP = 2;                  // frames of a pass
  constexpr int KS = D / 32, NC = D / 16, PP = PARTS == 3 ? 3 : 2;
  constexpr int OPS = 2 * KS + NC;                        // operands of a frame: keys, then values
  __shared__ Frame8 table[kTable8];
  __shared__ __align__(16) sbf16x8_t pool[2][FPP][OPS][64];
  __shared__ int s_bad[2][FPP];
  __shared__ int red[4];
  static_assert(sizeof(pool) + sizeof(table) + 64 <= 80 * 1024, "two workgroups a CU");

  const TreeParams& tp = p.t;
  const AttendParams& a = tp.a;
  const int slot = blockIdx.x >> 3, group = (slot / tp.mtiles) * 8 + (blockIdx.x & 7), mt = slot % tp.mtiles;
  if (group >= tp.units * tp.nsplit) return;
  TreePart part;
  if (!tree_part(tp, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int row0 = mt * ROWS + wave * 16 * QT;

  sbf16x8_t qb[QT][KS][PARTS];
  uint64_t bits[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) bits[qt] = load_queries<D, PARTS>(a, b, h, row0 + 16 * qt, qb[qt]);

  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (tp.nsplit == 1) clear_padding<D>(tp, b, h, mt * ROWS, ROWS, x.nq);
  if (mt * ROWS >= x.nq * a.G) return;                    // the tile's rows are all padding

  f32x4_t o[QT][NC];
  float m[QT], l[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m[qt] = -INFINITY;
    l[qt] = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[qt][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const int nf = x.frames(), all = (nf + FPP - 1) / FPP;
  const int f_lo = first_pass(all, part.split, part.n) * FPP, f_hi = min(first_pass(all, part.split + 1, part.n) * FPP, nf);
  const uint32_t rs = (uint32_t)(a.kv.table ? D : a.kv.st);
  const float c2 = a.c * 1.4426950408889634f;
  const uint8_t* const kp = static_cast<const uint8_t*>(a.kv.k);
  const uint8_t* const vp = static_cast<const uint8_t*>(a.kv.v);
  const int mine = wave >> 1;                             // the frame of a pass that the wave stages
  const bool keys = (wave & 1) == 0;                      // ... and which side of it
  const bool live_rows = row0 < x.nq * a.G;               // (a wave without rows stages all the same)

  int cnt = 0;
  uint32_t y[D / 8];
  auto fetch = [&](int pass) {
    const ScalarFrame f = table_frame(table, pass * FPP + mine, cnt);
    if (f.empty()) return;
    if (keys) load_keys<D>(kp + f.base, rs, y);
    else load_values<D>(vp + f.base, rs, y);
  };
  auto stage = [&](int pass) {
    const ScalarFrame f = table_frame(table, pass * FPP + mine, cnt);
    if (f.empty()) return;
    auto& to = pool[pass & 1][mine];
    if (keys) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) to[tt * KS + ks][lane] = key_operand<D>(y, tt, ks);
    } else {
      bool bad = false;
      if (!f.whole(x.C)) {
        bad = clear_dead<D>(y, f.ends(), x.C - f.a);
        if (bad) drop_nan<D>(y, x.C - f.a);
      }
      if (lane == 0) s_bad[pass & 1][mine] = bad;
      value_operands<D>(y, [&](int c, sbf16x8_t v) { to[2 * KS + c][lane] = v; });
    }
  };
  auto multiply = [&](int pass) {
    if (!live_rows) return;
#pragma unroll 1
    for (int fr = 0; fr < FPP; ++fr) {
      const ScalarFrame f = table_frame(table, pass * FPP + fr, cnt);
      if (f.empty()) continue;
      const auto& from = pool[pass & 1][fr];
      const bool whole = f.whole(x.C);
      f32x4_t s[QT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) s[qt][tt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const sbf16x8_t kk = from[tt * KS + ks][lane];
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k) s[qt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qb[qt][ks][k], s[qt][tt], 0, 0, 0);
        }
      }
      uint32_t vis[QT];
      if (!whole) {
        const int to_c = x.C - f.a;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) vis[qt] = visible_tokens(bits[qt], to_c, f.ends());
        if (__builtin_expect(s_bad[pass & 1][fr] != 0, 0)) {
          uint32_t v[D / 8];
          load_values<D>(vp + f.base, rs, v);
          clear_dead<D>(v, f.ends(), to_c);
          spread_nan<D, QT>(v, to_c, vis, o);
        }
      }
      sbf16x8_t pb[QT][PP];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) softmax_tile<NC, PP>(s[qt], f.ks, f.vs, whole, vis[qt], m[qt], l[qt], o[qt], pb[qt]);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const sbf16x8_t v = from[2 * KS + c][lane];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int k = PP - 1; k >= 0; --k) o[qt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[qt][k], o[qt][c], 0, 0, 0);
      }
    }
  };

  for (int t0 = f_lo; t0 < f_hi; t0 += kTable8) {
    __syncthreads();                                    // the table and the tiles are free
    cnt = min(kTable8, f_hi - t0);
    if (tid < cnt) table[tid] = describe_frame(p, x, b, h, t0 + tid, c2);
    __syncthreads();
    const int passes = (cnt + FPP - 1) / FPP;
    fetch(0);
    stage(0);
    fetch(1);
    __syncthreads();
    for (int it = 0; it < passes; ++it) {
      stage(it + 1);
      fetch(it + 2);
      multiply(it);
      __syncthreads();
    }
  }

  // lane: row l16 of each tile, elements (D / 16)(4 g + r) + c
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const float total = row_total(l[qt]);
    const int row = row0 + 16 * qt + l16;
    if (row >= x.nq * a.G) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < NC; c += 4)
        leave_row<D>(tp, part, row, NC * (4 * g + r) + c, make_float4(o[qt][c][r], o[qt][c + 1][r], o[qt][c + 2][r], o[qt][c + 3][r]), m[qt], total);
  }
}

}  // namespace cobs

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
// A workgroup is WQ x WT waves: WQ waves take 16 QT query rows each, WT groups of them different frames.  The
// frames of a row's context are split over workgroups as in cobs_tree_decode, whose kernels join the parts.
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

// NaN among the values of drafted tokens (a frame's tokens from to_c on): cleared, as 0 times it would reach
// every row, and put into the outputs of the rows that see such a token, whose number a product of flags gives.
template <int D, int QT>
__device__ __forceinline__ void spread_nan(uint32_t (&v)[8][D / 64], int to_c, const uint32_t (&vis)[QT], f32x4_t (&o)[QT][D / 16]) {
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
      const uint32_t nan = 4 * g + (j & 3) + 16 * (j >> 2) >= to_c ? nan_bytes(v[j][i]) : 0u;
      v[j][i] &= ~nan;
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

template <int D, int PARTS, int QT, int WQ>
__global__ __launch_bounds__(kTreeThreads, 2) void decode8_kernel(Decode8Params p) {
  constexpr int WT = 4 / WQ, TILE = 16 * QT, ROWS = TILE * WQ;   // frame groups; rows of a wave, of the workgroup
  constexpr int KS = D / 32;                              // k-steps of the scores, 16-byte loads a lane for 32 tokens
  constexpr int KL = D / 64;                              // 16-byte loads a lane for 16 tokens' keys
  constexpr int VW = D / 64;                              // registers of a token's values a lane
  constexpr int NC = D / 16;                              // products of the values
  constexpr int PP = PARTS == 3 ? 3 : 2;                  // bf16 parts of a probability
  __shared__ __align__(16) Frame8 table[kTable8];
  __shared__ __align__(16) float pool[WT > 1 ? 4 * TILE * D : 4];
  __shared__ float s_m[4][TILE], s_l[4][TILE];
  __shared__ int red[4];

  const TreeParams& tp = p.t;
  const AttendParams& a = tp.a;
  const int slot = blockIdx.x >> 3, group = (slot / tp.mtiles) * 8 + (blockIdx.x & 7), mt = slot % tp.mtiles;
  if (group >= tp.units * tp.nsplit) return;
  TreePart part;
  if (!tree_part(tp, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tg = wave / WQ, wq = wave % WQ, l16 = lane & 15, g = lane >> 4;
  const int row0 = mt * ROWS + wq * TILE;                 // the wave's query rows

  // ---- the query rows as the B operand: column l16, elements (D / 4) g + 8 ks + j
  sbf16x8_t qb[QT][KS][PARTS];
  uint64_t bits[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const QueryRow q = query_row(a, b, h, row0 + 16 * qt + l16);
    bits[qt] = q.bits;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int64_t at = q.at * D + (D / 4) * g + 8 * ks;
      if constexpr (PARTS == 1) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (q.live) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at);
        qb[qt][ks][0] = __builtin_bit_cast(sbf16x8_t, w);
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
        split_query(v, qb[qt][ks]);
      }
    }
  }

  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (tp.nsplit == 1) clear_padding<D>(tp, b, h, mt * ROWS, ROWS, x.nq);
  if (mt * ROWS >= x.nq * a.G) return;                    // the tile's rows are all padding

  f32x4_t o[QT][NC];
  float m[QT], l[QT];                                     // log2 domain; the lane's own tokens of the sum
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

  struct Codes {
    uint4 k[2][KL];
    uint32_t v[8][VW];
  };
  struct Frame {
    int64_t base;
    int a, lo, hi;
    float ks, vs;
  };
  // A frame's entry in scalar registers; one past the table's end is empty.
  auto entry = [&](int fi, int cnt) {
    Frame f = {0, 0, 0, 0, 0.0f, 0.0f};
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
  };
  const uint32_t koff = (uint32_t)l16 * rs + (D / 4) * g, voff = (uint32_t)(4 * g) * rs + (D / 16) * l16;
  auto load_keys = [&](const Frame& f, Codes& y) {
    if (f.hi <= f.lo) return;
    const uint8_t* kb = static_cast<const uint8_t*>(a.kv.k) + f.base;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < KL; ++i) y.k[tt][i] = *reinterpret_cast<const uint4*>(kb + (koff + (uint32_t)(16 * tt) * rs + 16 * i));
  };
  auto load_values = [&](const Frame& f, Codes& y) {
    if (f.hi <= f.lo) return;
    const uint8_t* vb = static_cast<const uint8_t*>(a.kv.v) + f.base;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint8_t* at = vb + (voff + (uint32_t)((j & 3) + 16 * (j >> 2)) * rs);
      if constexpr (VW == 2) {
        const uint2 w = *reinterpret_cast<const uint2*>(at);
        y.v[j][0] = w.x;
        y.v[j][1] = w.y;
      } else {
        y.v[j][0] = *reinterpret_cast<const uint32_t*>(at);
      }
    }
  };
  // A frame's codes in `y`, and the next one's, whose loads begin where its registers fall free.
  auto attend = [&](const Frame& f, const Frame& next, Codes& y) {
    if (f.hi <= f.lo) {
      load_keys(next, y);
      load_values(next, y);
      return;
    }
    const bool whole = f.lo == 0 && f.hi == kFrame && f.a + kFrame <= x.C;
    // ---- S^T: 32 tokens by 16 rows a tile
    f32x4_t s[QT][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) s[qt][tt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint4 w = y.k[tt][ks / 2];
        const uint32_t w0 = ks & 1 ? w.z : w.x, w1 = ks & 1 ? w.w : w.y;
        const u32x4v_t kk = {two_bf16<false>(w0), two_bf16<true>(w0), two_bf16<false>(w1), two_bf16<true>(w1)};
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k)
            s[qt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(sbf16x8_t, kk), qb[qt][ks][k], s[qt][tt], 0, 0, 0);
      }
    }
    load_keys(next, y);
    uint32_t vis[QT];                                     // bit t: whether the lane's query row sees token t of the frame
    uint32_t bad = 0;
    if (!whole) {
      const int to_c = x.C - f.a;                         // tokens of the context (32 and more: all)
      const uint32_t ends = (f.hi < kFrame ? (1u << f.hi) - 1u : ~0u) & (~0u << f.lo);
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        uint32_t u = to_c >= kFrame ? ~0u : (to_c > 0 ? (1u << to_c) - 1u : 0u);
        u |= to_c >= kFrame ? 0u : (uint32_t)(to_c > 0 ? bits[qt] << to_c : bits[qt] >> -to_c);
        vis[qt] = (u & ends) >> (4 * g);
      }
      // values of tokens that take no part, and NaN of drafted ones
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = 4 * g + (j & 3) + 16 * (j >> 2);
        const bool live = (ends >> t) & 1u, drafted = t >= to_c;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          const uint32_t nan = drafted ? nan_bytes(y.v[j][i]) : 0u;
          if (live) bad |= nan;
          y.v[j][i] = live ? y.v[j][i] : 0u;
        }
      }
    }
    // ---- streaming softmax: lane l has row l % 16 and 8 tokens of the frame.  The maximum is followed with
    // a slack of 2^8 in the probabilities, so that few frames exchange maxima and scale the outputs anew.
    sbf16x8_t pb[QT][PP];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = s[qt][j >> 2][j & 3] * f.ks;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = (vis[qt] >> ((j & 3) + 16 * (j >> 2))) & 1u ? z[j] : -INFINITY;
      }
      float top = z[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, z[j]);
      if (__ballot(top > m[qt] + 8.0f)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = fmaxf(m[qt], top), ref = mn == -INFINITY ? 0.0f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m[qt] - ref);
        m[qt] = mn;
        l[qt] *= alpha;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[qt][c] *= alpha;
      }
      const float ref = m[qt] == -INFINITY ? 0.0f : m[qt];
      float pv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f(z[j] - ref);
        l[qt] += e;
        pv[j] = e * f.vs;
      }
      split_bf16x8<PP>(pv, pb[qt]);
    }
    // ---- O^T += V^T P^T
    auto values = [&](auto put) {
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = y.v[j][i];
        sbf16x8_t c0, c1, c2, c3;
        columns<false>(w, c0, c1);
        columns<true>(w, c2, c3);
        put(4 * i, c0);
        put(4 * i + 1, c1);
        put(4 * i + 2, c2);
        put(4 * i + 3, c3);
      }
    };
    if (__builtin_expect(__ballot(bad != 0) != 0, 0)) spread_nan<D, QT>(y.v, x.C - f.a, vis, o);
    values([&](int c, sbf16x8_t v) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int k = PP - 1; k >= 0; --k) o[qt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[qt][k], o[qt][c], 0, 0, 0);
    });
    load_values(next, y);
  };

  for (int t0 = f_lo; t0 < f_hi; t0 += kTable8) {
    const int cnt = min(kTable8, f_hi - t0);
    __syncthreads();                                    // the table is free
    if (tid < cnt) {
      int fa, lo, hi;
      x.frame(t0 + tid, fa, lo, hi);
      const int64_t base = hi > lo ? kv_offset(a.kv, b, h, fa) : -1;
      Frame8 e = {0, fa, 0, 0, 0.0f, 0.0f};
      if (base >= 0) {
        const int64_t at = a.kv.table ? base / ((int64_t)D << a.lsh) : ((int64_t)b * a.hkv + h) * a.kv.nbmax + (fa >> a.lsh);
        e.base = base;
        e.lo = (int16_t)(lo - fa);
        e.hi = (int16_t)(hi - fa);
        e.ks = p.k_scale[at] * c2;
        e.vs = p.v_scale[at];
      }
      table[tid] = e;
    }
    __syncthreads();
    Frame now = entry(tg, cnt);
    Codes y;
    load_keys(now, y);
    load_values(now, y);
    for (int it = tg; it < cnt; it += WT) {
      const Frame next = entry(it + WT, cnt);
      attend(now, next, y);
      now = next;
    }
  }

  // ---- join the WT groups, in group order
  float total[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    total[qt] = l[qt] + __shfl_xor(l[qt], 16, 64);
    total[qt] += __shfl_xor(total[qt], 32, 64);
  }
  auto leave = [&](int row, int d, float4 sum, float mm, float ll) {         // (mm -inf: no score above that)
    if (row >= x.nq * a.G) return;
    if (tp.nsplit == 1) {
      const int i = row / a.G;
      const int64_t at = ((int64_t)b * a.N + i) * a.hq + h * a.G + (row - i * a.G);
      store_row4(tp.out, at * D + d, sum, ll, a.io_bf16);
      if (d == 0 && tp.lse) tp.lse[at] = ll != 0.0f ? (mm == -INFINITY ? 0.0f : mm) * 0.6931471805599453f + logf(ll) : -INFINITY;
    } else {
      const int64_t at = part_row(tp, part, row);
      *reinterpret_cast<float4*>(tp.part_o + at * D + d) = sum;
      if (d == 0) *reinterpret_cast<float2*>(tp.part_ml + 2 * at) = make_float2(mm, ll);
    }
  };
  if constexpr (WT == 1) {
    // lane: row l16, elements (D / 16)(4 g + r) + c
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; c += 4)
          leave(row0 + 16 * qt + l16, NC * (4 * g + r) + c, make_float4(o[qt][c][r], o[qt][c + 1][r], o[qt][c + 2][r], o[qt][c + 3][r]),
                m[qt], total[qt]);
    }
  } else {
    __syncthreads();
    if (g == 0) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        s_m[wave][16 * qt + l16] = m[qt];
        s_l[wave][16 * qt + l16] = total[qt];
      }
    }
    __syncthreads();
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r16 = 16 * qt + l16;
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < WT; ++t) top = fmaxf(top, s_m[t * WQ + wq][r16]);
      const float f = __builtin_amdgcn_exp2f(m[qt] - (top == -INFINITY ? 0.0f : top));
      float* const wo = pool + (wave * TILE + r16) * D;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; c += 4) {
          const int d4 = (NC * (4 * g + r) + c) / 4;
          *reinterpret_cast<float4*>(wo + 4 * (d4 ^ (l16 & (D / 4 - 1)))) =
              make_float4(o[qt][c][r] * f, o[qt][c + 1][r] * f, o[qt][c + 2][r] * f, o[qt][c + 3][r] * f);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < ROWS * (D / 4); idx += kTreeThreads) {
      const int rr = idx / (D / 4), d4 = idx % (D / 4), w = rr / TILE, r = rr % TILE;
      float mm = -INFINITY, ll = 0.0f;
#pragma unroll
      for (int t = 0; t < WT; ++t) mm = fmaxf(mm, s_m[t * WQ + w][r]);
      const float ref = mm == -INFINITY ? 0.0f : mm;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int t = 0; t < WT; ++t) {
        ll += __builtin_amdgcn_exp2f(s_m[t * WQ + w][r] - ref) * s_l[t * WQ + w][r];
        const float4 y = *reinterpret_cast<const float4*>(pool + ((t * WQ + w) * TILE + r) * D + 4 * (d4 ^ (r & 15 & (D / 4 - 1))));
        sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
      }
      leave(mt * ROWS + rr, 4 * d4, sum, mm, ll);
    }
  }
}

}  // namespace cobs

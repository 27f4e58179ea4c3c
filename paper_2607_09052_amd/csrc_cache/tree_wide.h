// Attention of many query rows (cobs_tree_decode, bf16): tree_kernel's products and
// softmax with 64 rows a wave, which read each key and value from LDS half as often.
//
// Four waves of up to 512 registers, one a SIMD: what runs beside the matrix
// instructions has to stand between them in the wave's own code.  So a frame's step
// takes the values of the frame before (beside this one's maxima) and the scores
// of the next (beside this one's probabilities), each in code without a branch; the
// next pass's keys and values go from registers to one of three LDS slots, and the
// loads of the pass after it start, among the scores.
//
// Measured: 512 rows over 8 rows of 32k tokens (0.55 TFLOP, 0.82 with the second part of the
// probabilities) in 804 us (tree_kernel 873), the matrix cores and the vector pipes busy 49 and
// 48 % of the time; 690 us are those products at the rate of a large plain one.
#pragma once

#include "tree_kernel.h"

namespace cobs {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kWideRows = 256;         // query rows of a workgroup
constexpr int kWideTable = 512;       // frame descriptors held in LDS at a time

template <int D>
__global__ __launch_bounds__(kTreeThreads, 1) void tree_wide_kernel(TreeParams p) {
  using S = TreeShape<D, 4, false>;
  constexpr int CPR = S::CPR, FPI = 2, QG = 2, NDT = D / 32, QK = D / 16, SLOTS = 3;
  constexpr int FRAME = S::KF + S::VF;
  constexpr int OUT = 4 * 32 * D * 4;                     // the waves' outputs of a tile
  __shared__ __align__(16) char pool[SLOTS * S::STAGE > OUT ? SLOTS * S::STAGE : OUT];
  __shared__ FrameEntry table[kWideTable + 3 * FPI];
  __shared__ float s_m[4][32], s_l[4][32];
  __shared__ unsigned long long s_bad;
  __shared__ int red[4];
  const AttendParams& a = p.a;
  const int slot = blockIdx.x >> 3, group = (slot / p.mtiles) * 8 + (blockIdx.x & 7), mt = slot % p.mtiles;
  if (group >= p.units * p.nsplit) return;
  TreePart part;
  if (!tree_part(p, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  QueryRow q[QG];
#pragma unroll
  for (int g = 0; g < QG; ++g) q[g] = query_row(a, b, h, mt * kWideRows + (wave * QG + g) * 32 + (lane & 31));
  const float c2 = a.c * 1.4426950408889634f, slack = max_slack(c2);
  if (tid == 0) s_bad = 0;
  sbf16x8_t qb[QG][QK];
#pragma unroll
  for (int g = 0; g < QG; ++g)
#pragma unroll
    for (int ks = 0; ks < QK; ++ks) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (q[g].live) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + q[g].at * D + 16 * ks + 8 * half);
      qb[g][ks] = __builtin_bit_cast(sbf16x8_t, w);
    }
  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (p.nsplit == 1) clear_padding<D>(p, b, h, mt * kWideRows, kWideRows, x.nq);
  if (mt * kWideRows >= x.nq * a.G) return;

  f32x16_t o[QG][NDT];
  float m[QG], l[QG];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[g][dt][i] = 0.0f;
  }
  const int nf = x.frames(), all = (nf + FPI - 1) / FPI;
  const int f_lo = first_pass(all, part.split, part.n) * FPI, f_hi = min(first_pass(all, part.split + 1, part.n) * FPI, nf);
  const uint32_t rsb = (uint32_t)((a.kv.table ? a.kv.d : a.kv.st) * 2);

  struct Frame {
    int64_t base;
    int a, lo, hi;
  };
  auto entry = [&](int fi) {
    const uint4 e = *reinterpret_cast<const uint4*>(&table[fi]);
    const uint32_t b0 = wave_uniform32((int)e.x), b1 = wave_uniform32((int)e.y), w = wave_uniform32((int)e.w);
    Frame f;
    f.base = (int64_t)(((uint64_t)b1 << 32) | b0);
    f.a = wave_uniform32((int)e.z);
    f.lo = (int)(int16_t)(w & 0xffff);
    f.hi = (int)(int16_t)(w >> 16);
    return f;
  };
  constexpr int LDF = S::LD / FPI;
  const uint32_t voff = (uint32_t)(tid / CPR) * rsb + (uint32_t)(tid % CPR) * 16;
  auto load = [&](const Frame (&f)[FPI], u32x4_t (&kr)[FPI][LDF], u32x4_t (&vr)[FPI][LDF]) {
#pragma unroll
    for (int fr = 0; fr < FPI; ++fr) {
      const char* kb = static_cast<const char*>(a.kv.k) + f[fr].base * 2;
      const char* vb = static_cast<const char*>(a.kv.v) + f[fr].base * 2;
#pragma unroll
      for (int j = 0; j < LDF; ++j) kr[fr][j] = *reinterpret_cast<const u32x4_t*>(kb + (voff + (uint32_t)(j * S::RPP) * rsb));
#pragma unroll
      for (int j = 0; j < LDF; ++j) vr[fr][j] = *reinterpret_cast<const u32x4_t*>(vb + (voff + (uint32_t)(j * S::RPP) * rsb));
    }
  };
  char* const kput = pool + (tid % CPR) * S::KSTEP + (tid / CPR) * 16;
  auto vput = [&](int j) { return ((tid / CPR + j * S::RPP) * CPR + v_chunk<CPR, false>(tid / CPR + j * S::RPP, tid % CPR)) * 16 + S::KF; };
  auto store = [&](int at, const u32x4_t (&kr)[FPI][LDF], const u32x4_t (&vr)[FPI][LDF]) {
#pragma unroll
    for (int fr = 0; fr < FPI; ++fr)
#pragma unroll
      for (int j = 0; j < LDF; ++j) {
        *reinterpret_cast<u32x4_t*>(kput + at + fr * FRAME + j * S::RPP * 16) = kr[fr][j];
        *reinterpret_cast<u32x4_t*>(pool + at + fr * FRAME + vput(j)) = vr[fr][j];
      }
  };
  // Frames that are not whole: rows that take no part become zeros, values of the draft finite.
  auto amend = [&](const Frame (&f)[FPI], u32x4_t (&kr)[FPI][LDF], u32x4_t (&vr)[FPI][LDF]) {
#pragma unroll
    for (int fr = 0; fr < FPI; ++fr) {
      if (f[fr].lo == 0 && f[fr].hi == kFrame && f[fr].a + kFrame <= x.C) continue;
#pragma unroll
      for (int j = 0; j < LDF; ++j) {
        const int r = tid / CPR + j * S::RPP;
        const bool part = r >= f[fr].lo && r < f[fr].hi;
        bool found;
        const uint4 v = finite_only<false>(__builtin_bit_cast(uint4, vr[fr][j]), found);
        if (part && f[fr].a + r >= x.C && found) {
          vr[fr][j] = __builtin_bit_cast(u32x4_t, v);
          atomicOr(&s_bad, 1ull << (f[fr].a + r - x.C));
        }
        if (!part) kr[fr][j] = vr[fr][j] = u32x4_t{0, 0, 0, 0};
      }
    }
  };

  f32x16_t s[QG];
  sbf16x8_t pb[QG][2][2];                                // operand of a step of 16 tokens, its two parts
  auto scores = [&](const char* fb, f32x16_t (&y)[QG]) {
    const char* const kf = fb + half * S::KSTEP + (lane & 31) * 16;
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[g][i] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < QK; ++ks) {
      const sbf16x8_t kk = *reinterpret_cast<const sbf16x8_t*>(kf + 2 * ks * S::KSTEP);
#pragma unroll
      for (int g = 0; g < QG; ++g) y[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, qb[g][ks], y[g], 0, 0, 0);
    }
  };
  // Operand of the values of a frame: step c / NDT of 16 tokens, columns 32 (c % NDT) + lane % 32
  auto value = [&](const char* fb, int c) {
    const int ks = c / NDT, dt = c % NDT;
    const int r = 16 * ks + 4 * half + ((lane & 15) >> 2), ch = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const char* at = fb + S::KF + (lane & 1) * 8;
    const s16x4_t v0 = tr_read(at + (r * CPR + v_chunk<CPR, false>(r, ch)) * 16);
    const s16x4_t v1 = tr_read(at + ((r + 8) * CPR + v_chunk<CPR, false>(r + 8, ch)) * 16);
    typedef short s16x8_t __attribute__((ext_vector_type(8)));
    const s16x8_t vv = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(sbf16x8_t, vv);
  };
  auto values = [&](const char* fb) {
#pragma unroll
    for (int c = 0; c < 2 * NDT; ++c) {
      const sbf16x8_t v = value(fb, c);
#pragma unroll
      for (int k = 1; k >= 0; --k)
#pragma unroll
        for (int g = 0; g < QG; ++g)
          o[g][c % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[g][c / NDT][k], o[g][c % NDT], 0, 0, 0);
    }
  };
  // One frame: the values of the frame before (`vb`), the softmax of this one, the scores of the next (`kb`).
  auto step = [&](const Frame& f, const char* vb, const char* kb, auto between, auto beside) {
    if (f.lo > 0 || f.hi < kFrame || f.a + f.hi > x.C) {
      const int to_c = x.C - f.a;
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        uint32_t vis = to_c >= kFrame ? ~0u : (to_c > 0 ? (1u << to_c) - 1u : 0u);
        vis |= to_c >= kFrame ? 0u : (uint32_t)(to_c > 0 ? q[g].bits << to_c : q[g].bits >> -to_c);
        vis &= (f.hi < kFrame ? (1u << f.hi) - 1u : ~0u) & (~0u << f.lo);
        vis >>= 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[g][i] = (vis >> (8 * (i >> 2) + (i & 3))) & 1u ? s[g][i] : -INFINITY;
      }
    }
    // ---- the values of the frame before, and this one's maxima
    float top[QG];
    {
      constexpr int NC = 2 * NDT, PER = 32 / NC;           // chunks; scores of each
      sbf16x8_t vv = value(vb, 0);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const sbf16x8_t cur = vv;
        if (c + 1 < NC) vv = value(vb, c + 1);
#pragma unroll
        for (int k = 1; k >= 0; --k)
#pragma unroll
          for (int g = 0; g < QG; ++g)
            o[g][c % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cur, pb[g][c / NDT][k], o[g][c % NDT], 0, 0, 0);
#pragma unroll
        for (int i = c * PER; i < (c + 1) * PER; ++i) top[i / 16] = i % 16 == 0 ? s[i / 16][0] : fmaxf(top[i / 16], s[i / 16][i % 16]);
      }
    }
    bool over = false;
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      top[g] = fmaxf(top[g], other_half(top[g]));
      over |= top[g] > m[g] + slack;
    }
    if (__ballot(over)) {
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        const float mn = fmaxf(m[g], top[g]), ref = mn == -INFINITY ? 0.0f : mn;
        const float alpha = __builtin_amdgcn_exp2f((m[g] - ref) * c2);
        m[g] = mn;
        l[g] *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[g][dt][i] *= alpha;
      }
    }
    between();
    // ---- the scores of the next, and this one's probabilities
    f32x16_t y[QG];
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[g][i] = 0.0f;
    const char* const kf = kb + half * S::KSTEP + (lane & 31) * 16;
    float mc[QG];
#pragma unroll
    for (int g = 0; g < QG; ++g) mc[g] = m[g] == -INFINITY ? 0.0f : m[g] * c2;
    {
      constexpr int PER = 32 / QK;
      sbf16x8_t kk = *reinterpret_cast<const sbf16x8_t*>(kf);
      float e[8];
#pragma unroll
      for (int ks = 0; ks < QK; ++ks) {
        const sbf16x8_t cur = kk;
        if (ks + 1 < QK) kk = *reinterpret_cast<const sbf16x8_t*>(kf + 2 * (ks + 1) * S::KSTEP);
#pragma unroll
        for (int g = 0; g < QG; ++g) y[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cur, qb[g][ks], y[g], 0, 0, 0);
#pragma unroll
        for (int i = ks * PER; i < (ks + 1) * PER; ++i) {
          e[i % 8] = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], c2, -mc[i / 16]));
          if (i % 4 == 3) l[i / 16] += (e[i % 8 - 3] + e[i % 8 - 2]) + (e[i % 8 - 1] + e[i % 8]);
          if (i % 8 == 7) {
            sbf16x8_t w[2];
            split_bf16x8<2>(e, w);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint4 u = __builtin_bit_cast(uint4, w[k]);
              asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));    // kept beside the products
              pb[i / 16][i % 16 / 8][k] = __builtin_bit_cast(sbf16x8_t, u);
            }
          }
        }
        if (ks == 0) {
          beside();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int g = 0; g < QG; ++g) s[g] = y[g];
  };

  auto at_slot = [&](int i) { return (i % SLOTS) * S::STAGE; };
  for (int t0 = f_lo; t0 < f_hi; t0 += kWideTable) {
    const int cnt = min(kWideTable, f_hi - t0);
    __syncthreads();
    for (int i = tid; i < cnt + 3 * FPI; i += kTreeThreads) {              // (and the empty ones after the last)
      int fa = 0, lo = 0, hi = 0;
      if (i < cnt) x.frame(t0 + i, fa, lo, hi);
      const int64_t base = hi > lo ? kv_offset(a.kv, b, h, fa) : -1;
      FrameEntry e;
      e.base = base < 0 ? 0 : base;
      e.a = fa;
      e.lo = (int16_t)(base < 0 ? 0 : lo - fa);
      e.hi = (int16_t)(base < 0 ? 0 : hi - fa);
      table[i] = e;
    }
    __syncthreads();
    const int passes = (cnt + FPI - 1) / FPI;
    auto frames_of = [&](int it, Frame (&f)[FPI]) {
#pragma unroll
      for (int fr = 0; fr < FPI; ++fr) f[fr] = entry(it * FPI + fr);
    };
    // the "values before the first frame": zeros
    for (int i = tid; i < S::VF / 16; i += kTreeThreads)
      *reinterpret_cast<uint4*>(pool + at_slot(2) + FRAME + S::KF + 16 * i) = make_uint4(0, 0, 0, 0);
    Frame now[FPI], next[FPI], after[FPI];
    u32x4_t kr[FPI][LDF], vr[FPI][LDF];
    frames_of(0, now);
    load(now, kr, vr);
    amend(now, kr, vr);
    store(at_slot(0), kr, vr);
    frames_of(1, next);
    load(next, kr, vr);
    __syncthreads();
    scores(pool + at_slot(0), s);
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) pb[g][ks][0] = pb[g][ks][1] = __builtin_bit_cast(sbf16x8_t, make_uint4(0, 0, 0, 0));
    int s0 = at_slot(0), s1 = at_slot(1), s2 = at_slot(2);              // this pass, the next, the one before
    for (int it = 0; it < passes; ++it) {
      frames_of(it + 2, after);
      step(now[0], pool + s2 + FRAME, pool + s0 + FRAME, [&] { amend(next, kr, vr); },
           [&] {
             store(s1, kr, vr);
             load(after, kr, vr);
           });
      __syncthreads();
      step(now[1], pool + s0, pool + s1, [] {}, [] {});
#pragma unroll
      for (int fr = 0; fr < FPI; ++fr) { now[fr] = next[fr]; next[fr] = after[fr]; }
      const int sx = s2;
      s2 = s0; s0 = s1; s1 = sx;
    }
    values(pool + s2 + FRAME);
  }

  __syncthreads();
  if (s_bad != 0) {
#pragma unroll
    for (int g = 0; g < QG; ++g) add_nonfinite<D, false>(a, x, b, h, q[g], s_bad, m[g] == -INFINITY ? 0.0f : m[g], c2, o[g]);
  }
  constexpr int PASSES = 4 * 32 * (D / 4) / kTreeThreads;
  static_assert(QG * PASSES <= 32, "a bit a pass");
  uint32_t nan = 0;
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    if (g > 0) __syncthreads();
    const float lsum = l[g] + other_half(l[g]);
    if (half == 0) { s_m[wave][lane] = m[g]; s_l[wave][lane] = lsum; }
    float* const wo = reinterpret_cast<float*>(pool) + wave * 32 * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int r = lane & 31, d4 = (32 * dt + 2 * i + 4 * half) / 4;
        *reinterpret_cast<float4*>(wo + r * D + 4 * (d4 ^ (r & (D / 4 - 1)))) =
            make_float4(o[g][dt][i], o[g][dt][i + 1], o[g][dt][i + 2], o[g][dt][i + 3]);
      }
    __syncthreads();
    for (int idx = tid; idx < 4 * 32 * (D / 4); idx += kTreeThreads) {
      const int rr = idx / (D / 4), d4 = idx % (D / 4), w = rr / 32, r = rr % 32;
      const int row = mt * kWideRows + (w * QG + g) * 32 + r;
      if (row >= x.nq * a.G) continue;
      const float mm = s_m[w][r], ll = s_l[w][r], rm = mm == -INFINITY ? 0.0f : mm;
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(pool) + (w * 32 + r) * D + 4 * (d4 ^ (r & (D / 4 - 1))));
      if (has_nan(y, ll)) nan |= 1u << (g * PASSES + idx / kTreeThreads);
      if (p.nsplit == 1) {
        const int i = row / a.G;
        const int64_t at = ((int64_t)b * a.N + i) * a.hq + h * a.G + (row - i * a.G);
        store_row4(p.out, at * D + 4 * d4, y, ll, a.io_bf16);
        if (d4 == 0 && p.lse) p.lse[at] = ll != 0.0f ? rm * a.c + logf(ll) : -INFINITY;
      } else {
        const int64_t at = part_row(p, part, row);
        *reinterpret_cast<float4*>(p.part_o + at * D + 4 * d4) = y;
        if (d4 == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(mm * c2, ll);
      }
    }
  }
  if (__builtin_expect(__ballot(nan != 0) != 0, 0))
    plain_rows<D>(p, x, part, f_lo, f_hi, nan, [&](int k, int t) {
      const int rr = (k % PASSES * kTreeThreads + t) / (D / 4);
      return mt * kWideRows + (rr / 32 * QG + k / PASSES) * 32 + rr % 32;
    });
}

}  // namespace cobs

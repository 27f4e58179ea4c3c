// Attention of several query tokens a row over the cache and their draft
// (cobs_tree_decode), on the matrix cores.
//
// The M = N G query rows of one (batch row, KV head) share its keys and values, so
// they are the columns of the products: S^T = K Q^T (32 tokens by 32 rows a tile)
// and O^T = V^T P^T.  With tokens as rows the probabilities that a lane holds
// after the softmax are the operand of the second product as they stand (the
// token order inside a k-step is permuted, which V's reads follow), every row's
// maximum, sum and output scale are one value a lane, and a maximum needs one
// exchange between the two halves of the wave.
//
// A workgroup is WQ x WT waves: WQ waves take 32 query rows each and share the
// frames in LDS, WT groups of them take different frames.  Few rows (M <= 32) are
// bound by HBM: four waves with a frame each in flight.  Many rows are bound by
// the matrix cores: 128 rows a workgroup read each key and value once.  The frames
// of a row's context are split over workgroups; tree.hip's kernels join the parts.
//
// Measured (d 128, bf16 cache): 16 rows of a batch of 32 over 85 selected blocks and a window of
// 512, fp32 queries: 800 MB in 168 us, 4.8 TB/s, with three products for one (150 TFLOP in them)
// near the matrix cores' bound too (busy 44 % of the time); 128 rows over 4 contexts of 8k to 32k tokens, on
// pages: 411 MB in 110 us, 3.7 TB/s, the matrix cores busy 35 %; 512 rows over 8 x 32k tokens:
// 0.55 TFLOP (0.82 with the second part of the probabilities) in 873 us, matrix instructions and
// softmax overlapping little with two waves a SIMD (tree_wide.h has the form for such calls).
// One short context: 9 us of dependent loads, barriers and one pass.
//
// Frames travel HBM -> registers (two passes ahead; WQ = 1: one) -> LDS, in 16-byte
// chunks that are swizzled by row against bank conflicts:
//   K       chunk c of row r at c (32 + 1) + r: the operand of a k-step is 32 rows of two
//           chunks, consecutive lanes at consecutive addresses, and every step at a
//           constant offset; the 33rd place keeps a row's writes on different banks;
//   bf16 V  row-major, chunk c of row r at c ^ 4 (r % 4) (64-element heads: c ^ 2 (r & 2)):
//           the transposing read (ds_read_b64_tr_b16) takes 4 tokens by 16 columns per
//           16 lanes;
//   fp32 V  by column, as stored.
// fp32 products run on 32x32x2 fp32 operands.  bf16 products take an fp32 query and
// its probabilities as three bf16 parts, which hold all 24 bits (two leave 2^-17:
// outputs 3.6e-6 off instead of 1e-6 at 32k tokens, and 4 to 20 % faster at up to
// 64 rows).  bf16 queries are one part, their probabilities two (2^-17, far below the outputs'
// rounding of 2^-8; one, which rounds them by 2^-8 as well, left outputs 2.0e-3 to 2.4e-3 off in
// relative norm instead of 1.7e-3, and took 610 us instead of 800 at 512 rows over 8 x 32k tokens,
// 108 instead of 129 at 128 rows on pages, and the same time for few rows).
//
// Drafted tokens stand in the frames behind the context; what a query's mask
// leaves out gets score -inf.  A value that is not finite would still reach every
// row of the product as 0 times it, so such elements of drafted tokens enter LDS
// as 0 and are added afterwards to the rows that see them (add_nonfinite).
// In several parts an operand gives NaN with an infinite key or value (inf - inf, 0 inf)
// where the operand itself gives an infinity: rows with NaN of a part that holds
// infinities are computed once more, without parts (plain_rows).
#pragma once

#include "cache_device.h"

namespace cobs {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kTable = 256;            // frame descriptors held in LDS at a time

template <int D, int WQ, bool F32>
struct TreeShape {
  static constexpr int WT = 4 / WQ;                       // frame groups
  static constexpr int ES = F32 ? 4 : 2;
  static constexpr int CPR = D * ES / 16;                 // 16-byte chunks of a row
  static constexpr int FPI = (WQ == 4 && !F32) ? 2 : 1;   // frames of a group's pass
  static constexpr int ROWS = FPI * kFrame;
  static constexpr int NBUF = WQ == 1 ? 1 : 2;            // wave-private frames need no second buffer
  static constexpr int KSTEP = (kFrame + 1) * 16;         // bytes from a K chunk to the next
  static constexpr int KF = CPR * KSTEP, VF = kFrame * D * ES;   // bytes of a frame's K and V tiles
  static constexpr int STAGE = FPI * (KF + VF);
  static constexpr int POOL = WT * NBUF * STAGE;          // at least 4 waves' outputs, 32 x D fp32 each
  static_assert(POOL >= 4 * 32 * D * 4 || WQ == 2, "room for the waves' outputs");
  static constexpr int LDS = POOL > 4 * 32 * D * 4 ? POOL : 4 * 32 * D * 4;
  static constexpr int NT = WQ * 64;                      // threads of a group
  static constexpr int RPP = NT / CPR;                    // rows a load instruction of the group covers
  static constexpr int LD = ROWS / RPP;                   // loads of a thread for K (as many for V)
};

// A frame in the table: element offset of its first row; its live rows lo .. hi - 1 (relative), position a.
struct FrameEntry {
  int64_t base;
  int a;
  int16_t lo, hi;
};

template <int CPR, bool F32>
__device__ __forceinline__ int v_chunk(int row, int c) {
  if constexpr (F32) return c;
  else return CPR == 16 ? c ^ ((row & 3) << 2) : c ^ ((row & 2) << 1);
}

// 16 bytes with the elements that are not finite cleared; `found`: whether there were any.
template <bool F32>
__device__ __forceinline__ uint4 finite_only(uint4 x, bool& found) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
  found = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      if ((w[i] & 0x7f800000u) == 0x7f800000u) { w[i] = 0; found = true; }
    } else {
      if ((w[i] & 0x7f80u) == 0x7f80u) { w[i] &= 0xffff0000u; found = true; }
      if ((w[i] & 0x7f800000u) == 0x7f800000u) { w[i] &= 0x0000ffffu; found = true; }
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// By how much a score may pass the running maximum: 2^8 in the probabilities.  (Finite at the smallest scales,
// where 8 / c2 overflows, as -inf + inf would let no score become the maximum.)
__device__ __forceinline__ float max_slack(float c2) { return fminf(8.0f / c2, 3.4028234e38f); }

// Sum over visible drafted tokens j in `bad` of p V[j][d] for the elements of V that are not finite,
// added to the lane's outputs.  Rare (an overflowed value), so from memory and element by element.
template <int D, bool F32>
__device__ __forceinline__ void add_nonfinite(const AttendParams& a, const Attended& x, int b, int h, const QueryRow& q,
                                           uint64_t bad, float m, float c2, f32x16_t (&o)[D / 32]) {
  const int half = (threadIdx.x & 63) >> 5;
  while (bad) {
    const int j = __builtin_ctzll(bad);
    bad &= bad - 1;
    const int64_t off = kv_offset(a.kv, b, h, x.C + j);
    if (off < 0) continue;
    const bool see = q.live && ((q.bits >> j) & 1);
    float s = 0.0f;
    if (see)
      for (int e = 0; e < D; ++e) s += load_elem(a.q, q.at * D + e, !a.io_bf16) * load_elem(a.kv.k, off + e, F32);
    const float p = see ? __builtin_amdgcn_exp2f(s * c2 - m * c2) : 0.0f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float v = load_elem(a.kv.v, off + 32 * dt + 8 * (i >> 2) + 4 * half + (i & 3), F32);
        if (see && !(fabsf(v) < INFINITY)) o[dt][i] += p * v;
      }
  }
}

// Whether one of the five is NaN (or there are infinities of both signs).
__device__ __forceinline__ bool has_nan(float4 y, float total) {
  const float z = ((y.x + y.y) + (y.z + y.w)) + total;
  return z != z;
}

// Whether one of 8 bf16 values is an infinity.
__device__ __forceinline__ bool has_infinity(uint4 x) {
  bool found = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i == 0 ? x.x : (i == 1 ? x.y : (i == 2 ? x.z : x.w));
    found |= (w & 0x7fffu) == 0x7f80u || (w & 0x7fff0000u) == 0x7f800000u;
  }
  return found;
}

// Query rows of the wave's outputs again (bit k of a lane's `nan`: its outputs of the pass k have NaN), if the
// frames f_lo .. f_hi - 1 of the part (bf16) hold an infinity: scores, softmax and sums element by
// element in fp32, from memory, a row at a time.  row_of(k, thread) is the row of a thread's outputs.
// Rare, so only right: one infinite value in one of 32 contexts of 32k tokens, 32 rows each: 2.5 ms for 0.11.
template <int D, typename RowOf>
__device__ __forceinline__ void plain_rows(const TreeParams& p, const Attended& x, const TreePart& part, int f_lo, int f_hi,
                                           uint32_t nan, RowOf row_of) {
  constexpr int CPR = D / 8, COLS = D / 64, TPR = D / 4;
  const AttendParams& a = p.a;
  const int b = part.b, h = part.h, lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t rs = a.kv.table ? a.kv.d : a.kv.st;
  const uint16_t* const kp = static_cast<const uint16_t*>(a.kv.k);
  const uint16_t* const vp = static_cast<const uint16_t*>(a.kv.v);
  bool found = false;
  for (int f = f_lo; f < f_hi; ++f) {
    int fa, lo, hi;
    x.frame(f, fa, lo, hi);
    const int64_t base = lo < hi ? kv_offset(a.kv, b, h, fa) : -1;
    if (base < 0) continue;
#pragma unroll 4
    for (int i = lane; i < (hi - lo) * CPR; i += 64) {
      const int64_t at = base + (lo - fa + i / CPR) * rs + 8 * (i % CPR);
      const uint4 k = *reinterpret_cast<const uint4*>(kp + at), v = *reinterpret_cast<const uint4*>(vp + at);
      found |= has_infinity(k);
      found |= has_infinity(v);
    }
  }
  if (!__ballot(found)) return;
  __threadfence_block();                                     // what is read back below is written
  const float c2 = a.c * 1.4426950408889634f;
  for (int w = 0; w < 32 * 64 / TPR; ++w) {                    // passes, and rows of the wave in a pass
    const int k = w / (64 / TPR), first = w % (64 / TPR) * TPR;
    if (!((__ballot((nan >> k) & 1) >> first) & (TPR == 32 ? 0xffffffffull : 0xffffull))) continue;
    const int row = wave_uniform32(row_of(k, (threadIdx.x & ~63) + first));
    const QueryRow q = query_row(a, b, h, row);
    float m = -INFINITY, l = 0.0f, o[COLS] = {}, qv[COLS];    // (element 64 j + lane of the query)
#pragma unroll
    for (int j = 0; j < COLS; ++j) qv[j] = load_elem(a.q, q.at * D + 64 * j + lane, !a.io_bf16);
    auto element = [&](int e) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(qv[COLS == 2 && e >= 64]), e % 64)); };
    for (int f = f_lo; f < f_hi; ++f) {
      int fa, lo, hi;
      x.frame(f, fa, lo, hi);
      const int64_t base = lo < hi ? kv_offset(a.kv, b, h, fa) : -1;
      if (base < 0) continue;
      // lane l: token l % 32, half the elements
      const int t = fa + (lane & 31);
      const bool see = t >= lo && t < hi && (t < x.C || ((q.bits >> (t - x.C)) & 1));
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < D / 2; e += 8) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (see) x = *reinterpret_cast<const uint4*>(kp + base + (lane & 31) * rs + half * (D / 2) + e);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float qe = half ? element(D / 2 + e + i) : element(e + i);
          s = fmaf(qe, i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]), s);
        }
      }
      s += other_half(s);
      float top = see ? s : -INFINITY;
#pragma unroll
      for (int k = 16; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
      const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.0f : mn, alpha = __builtin_amdgcn_exp2f((m - ref) * c2);
      const float pr = see ? __builtin_amdgcn_exp2f((s - ref) * c2) : 0.0f;
      m = mn;
      float sum = pr;
#pragma unroll
      for (int k = 16; k >= 1; k >>= 1) sum += __shfl_xor(sum, k, 64);
      l = fmaf(l, alpha, sum);
#pragma unroll
      for (int j = 0; j < COLS; ++j) o[j] *= alpha;
      const uint32_t seen = (uint32_t)__ballot(see);         // (both halves alike; a value that is not seen enters as 0)
      for (int k0 = 0; k0 < kFrame; k0 += 16) {
        uint32_t v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const uint16_t* at = vp + base + (k0 + k) * rs + COLS * lane;
          if constexpr (COLS == 2) v[k] = *reinterpret_cast<const uint32_t*>(at);
          else v[k] = *at;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float pk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pr), k0 + k));
          const uint32_t x = (seen >> (k0 + k)) & 1 ? v[k] : 0;
          o[0] = fmaf(pk, bf16_lo(x), o[0]);
          if constexpr (COLS == 2) o[1] = fmaf(pk, bf16_hi(x), o[1]);
        }
      }
    }
    // in the place of what is NaN (a score: all of the row; a value: its column, at the maximum that the others have)
    if (p.nsplit > 1) {
      const int64_t at = part_row(p, part, row);
      float2* const ml = reinterpret_cast<float2*>(p.part_ml + 2 * at);
      const bool all = ml->y != ml->y;
      const float f = all ? 1.0f : __builtin_amdgcn_exp2f(m * c2 - ml->x);
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        float& y = p.part_o[at * D + COLS * lane + j];
        if (all || y != y) y = o[j] * f;
      }
      if (all && lane == 0) *ml = make_float2(m * c2, l);
    } else {
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const int64_t at = q.at * D + COLS * lane + j;
        const float y = load_elem(p.out, at, !a.io_bf16);
        if (y != y) store_elem(p.out, at, l != 0.0f ? o[j] / l : 0.0f, !a.io_bf16);
      }
      if (lane == 0 && p.lse && p.lse[q.at] != p.lse[q.at]) p.lse[q.at] = l != 0.0f ? m * a.c + logf(l) : -INFINITY;
    }
  }
}

template <int D, int WQ, bool F32, int PARTS>
__global__ __launch_bounds__(kTreeThreads, F32 || (PARTS == 3 && D == 128 && WQ == 1) ? 1 : 2) void tree_kernel(TreeParams p) {
  using S = TreeShape<D, WQ, F32>;
  constexpr int WT = S::WT, CPR = S::CPR, LD = S::LD, NT = S::NT, FPI = S::FPI;
  constexpr int NDT = D / 32;
  constexpr int PP = PARTS == 3 ? 3 : 2;                  // bf16 parts of a probability
  constexpr bool JOINT = FPI == 2 && PARTS == 1;          // a pass's frames at one maximum (three parts leave no registers for it)
  constexpr int NF = JOINT ? 2 : 1;
  __shared__ __align__(16) char pool[S::LDS];
  __shared__ FrameEntry table[kTable];
  __shared__ float s_m[4][32], s_l[4][32];
  __shared__ unsigned long long s_bad[WT];
  __shared__ int red[4];
  // The third parts of the first QL k-steps' queries are read from LDS: they are the registers by
  // which two workgroups a CU would spill, and a spilled value's reload waits for the frames under way.
  constexpr int QL = PARTS == 3 && D == 128 ? (WQ == 2 ? 4 : (WQ == 4 ? 2 : 0)) : 0;
  __shared__ __align__(16) uint4 q_low[QL > 0 ? WQ * QL * 64 : 1];

  const AttendParams& a = p.a;
  // Workgroups go round-robin to the 8 XCDs; the row tiles of one part of the
  // context, which read the same keys and values, follow each other on one.
  const int slot = blockIdx.x >> 3, group = (slot / p.mtiles) * 8 + (blockIdx.x & 7), mt = slot % p.mtiles;
  if (group >= p.units * p.nsplit) return;
  TreePart part;
  if (!tree_part(p, group, part)) return;
  const int b = part.b, h = part.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tg = wave / WQ, wq = wave % WQ, half = lane >> 5, gt = tid % NT;
  const int row0 = (mt * WQ + wq) * 32;                         // the wave's query rows
  const QueryRow q = query_row(a, b, h, row0 + (lane & 31));
  const float c2 = a.c * 1.4426950408889634f, slack = max_slack(c2);
  if (tid < WT) s_bad[tid] = 0;

  // ---- the query rows as the B operand: column lane % 32, k = 8 half + j of every step
  constexpr int QR = F32 ? D / 2 : 1, QK = F32 ? 1 : D / 16;
  float qf[QR];
  sbf16x8_t qb[QK][F32 ? 1 : PARTS];          // (the parts in q_low are dropped)
  if constexpr (F32) {
#pragma unroll
    for (int u = 0; u < D / 8; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        qf[4 * u + j] = q.live ? load_elem(a.q, q.at * D + 8 * u + 4 * half + j, !a.io_bf16) : 0.0f;
  } else {
#pragma unroll
    for (int ks = 0; ks < QK; ++ks) {
      const int e = 16 * ks + 8 * half;
      if constexpr (PARTS == 1) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (q.live) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + q.at * D + e);
        qb[ks][0] = __builtin_bit_cast(sbf16x8_t, w);
      } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (q.live) {
          const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + q.at * D + e);
          const float4 s0 = s[0], s1 = s[1];
          v[0] = s0.x; v[1] = s0.y; v[2] = s0.z; v[3] = s0.w;
          v[4] = s1.x; v[5] = s1.y; v[6] = s1.z; v[7] = s1.w;
        }
        split_bf16x8<PARTS>(v, qb[ks]);
        if constexpr (PARTS == 3)
          if (ks < QL) q_low[(wq * QL + ks) * 64 + lane] = __builtin_bit_cast(uint4, qb[ks][2]);   // the groups': the same
      }
    }
  }

  const Attended x = attended<kTreeThreads>(a, b, h, red);
  if (p.nsplit == 1) clear_padding<D>(p, b, h, mt * WQ * 32, WQ * 32, x.nq);
  if (mt * WQ * 32 >= x.nq * a.G) return;                       // the tile's rows are all padding

  f32x16_t o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;          // raw units; the lane's own half of the sum

  constexpr int STEP = WT * FPI;                                // frames of a pass of the workgroup
  const int nf = x.frames(), all = (nf + STEP - 1) / STEP;
  const int f_lo = first_pass(all, part.split, part.n) * STEP, f_hi = min(first_pass(all, part.split + 1, part.n) * STEP, nf);
  const uint32_t rsb = (uint32_t)((a.kv.table ? a.kv.d : a.kv.st) * S::ES);     // 32 rows: below 2^32 bytes
  char* const mine = pool + tg * S::NBUF * S::STAGE;

  // A frame's entry in scalar registers; one past the table's end is empty.
  struct Frame {
    int64_t base;
    int a, lo, hi;
  };
  auto entry = [&](int fi, int cnt) {
    Frame f = {0, 0, 0, 0};
    if (fi < cnt) {
      const uint4 e = *reinterpret_cast<const uint4*>(&table[fi]);
      const uint32_t b0 = wave_uniform32((int)e.x), b1 = wave_uniform32((int)e.y), w = wave_uniform32((int)e.w);
      f.base = (int64_t)(((uint64_t)b1 << 32) | b0);
      f.a = wave_uniform32((int)e.z);
      f.lo = (int)(int16_t)(w & 0xffff);
      f.hi = (int)(int16_t)(w >> 16);
    }
    return f;
  };

  // K and V of a pass's frames, 16 bytes a load: row gt / CPR + RPP j of the frame, chunk gt % CPR
  constexpr int LDF = LD / FPI;
  uint4 kr[FPI][LDF], vr[FPI][LDF];
  const uint32_t voff = (uint32_t)(gt / CPR) * rsb + (uint32_t)(gt % CPR) * 16;
  auto load = [&](const Frame (&f)[FPI]) {
#pragma unroll
    for (int fr = 0; fr < FPI; ++fr) {
      if (f[fr].hi <= f[fr].lo) continue;
      const char* kb = static_cast<const char*>(a.kv.k) + f[fr].base * S::ES;
      const char* vb = static_cast<const char*>(a.kv.v) + f[fr].base * S::ES;
#pragma unroll
      for (int j = 0; j < LDF; ++j) kr[fr][j] = *reinterpret_cast<const uint4*>(kb + (voff + (uint32_t)(j * S::RPP) * rsb));
#pragma unroll
      for (int j = 0; j < LDF; ++j) vr[fr][j] = *reinterpret_cast<const uint4*>(vb + (voff + (uint32_t)(j * S::RPP) * rsb));
    }
  };
  auto store = [&](const Frame (&f)[FPI], char* buf) {
#pragma unroll
    for (int fr = 0; fr < FPI; ++fr) {
      const bool empty = f[fr].hi <= f[fr].lo;
      if (empty && !JOINT) continue;                         // not read either
      const bool whole = f[fr].lo == 0 && f[fr].hi == kFrame && f[fr].a + kFrame <= x.C;
      char* const kb = buf + fr * (S::KF + S::VF) + (gt % CPR) * S::KSTEP + (gt / CPR) * 16;
      char* const vb = buf + fr * (S::KF + S::VF) + S::KF;
#pragma unroll
      for (int j = 0; j < LDF; ++j) {
        const int r = gt / CPR + j * S::RPP, c = gt % CPR;
        uint4 k = kr[fr][j], v = vr[fr][j];
        if (!whole) {
          if (r < f[fr].lo || r >= f[fr].hi) {               // rows that take no part: whatever memory holds there
            k = make_uint4(0, 0, 0, 0);
            v = k;
          } else if (f[fr].a + r >= x.C) {
            bool found;
            v = finite_only<F32>(v, found);
            if (found) atomicOr(&s_bad[tg], 1ull << (f[fr].a + r - x.C));
          }
        }
        *reinterpret_cast<uint4*>(kb + j * S::RPP * 16) = k;
        *reinterpret_cast<uint4*>(vb + (r * CPR + v_chunk<CPR, F32>(r, c)) * 16) = v;
      }
    }
  };
  // NF frames of a pass from fr0 on, at one maximum
  auto attend_frames = [&](const Frame (&fs)[FPI], int fr0, const char* buf) {
    const char* const kt = buf + fr0 * (S::KF + S::VF) + half * S::KSTEP + (lane & 31) * 16;
    // ---- S^T: 32 tokens x 32 query rows a frame
    f32x16_t s[NF];
#pragma unroll
    for (int fr = 0; fr < NF; ++fr) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[fr][i] = 0.0f;
      const char* const kf = kt + fr * (S::KF + S::VF);
      if constexpr (F32) {
#pragma unroll
        for (int u = 0; u < D / 8; ++u) {
          const float4 kk = *reinterpret_cast<const float4*>(kf + 2 * u * S::KSTEP);
          s[fr] = __builtin_amdgcn_mfma_f32_32x32x2f32(kk.x, qf[4 * u], s[fr], 0, 0, 0);
          s[fr] = __builtin_amdgcn_mfma_f32_32x32x2f32(kk.y, qf[4 * u + 1], s[fr], 0, 0, 0);
          s[fr] = __builtin_amdgcn_mfma_f32_32x32x2f32(kk.z, qf[4 * u + 2], s[fr], 0, 0, 0);
          s[fr] = __builtin_amdgcn_mfma_f32_32x32x2f32(kk.w, qf[4 * u + 3], s[fr], 0, 0, 0);
        }
      } else {
        constexpr int KB = PARTS == 3 ? 2 : D / 16;       // operands read together
#pragma unroll
        for (int k0 = 0; k0 < D / 16; k0 += KB) {
          sbf16x8_t kk[KB];
#pragma unroll
          for (int ks = 0; ks < KB; ++ks) kk[ks] = *reinterpret_cast<const sbf16x8_t*>(kf + 2 * (k0 + ks) * S::KSTEP);
#pragma unroll
          for (int ks = 0; ks < KB; ++ks) {
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k) {
              sbf16x8_t qq = qb[k0 + ks][k];
              if (k == 2 && k0 + ks < QL) qq = *reinterpret_cast<const sbf16x8_t*>(&q_low[(wq * QL + k0 + ks) * 64 + lane]);
              s[fr] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk[ks], qq, s[fr], 0, 0, 0);
            }
          }
        }
      }
    }
#pragma unroll
    for (int fr = 0; fr < NF; ++fr) {
      const int lo = fs[fr0 + fr].lo, hi = fs[fr0 + fr].hi, ea = fs[fr0 + fr].a;
      if (lo > 0 || hi < kFrame || ea + hi > x.C) {
        // bit t of `vis`: whether the lane's query row sees token t of the frame
        const int to_c = x.C - ea;                          // tokens of the context (32 and more: all)
        uint32_t vis = to_c >= kFrame ? ~0u : (to_c > 0 ? (1u << to_c) - 1u : 0u);
        vis |= to_c >= kFrame ? 0u : (uint32_t)(to_c > 0 ? q.bits << to_c : q.bits >> -to_c);
        vis &= (hi < kFrame ? (1u << hi) - 1u : ~0u) & (~0u << lo);
        vis >>= 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[fr][i] = (vis >> (8 * (i >> 2) + (i & 3))) & 1u ? s[fr][i] : -INFINITY;
      }
    }
    // ---- streaming softmax: lane l has row l % 32, the tokens of its half.  The
    // maximum is followed with a slack of 2^8 in the probabilities, so that few
    // frames scale the outputs anew; probabilities and sums keep their precision.
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 16 * NF; ++i) top = fmaxf(top, s[i / 16][i % 16]);
    top = fmaxf(top, other_half(top));
    if (__ballot(top > m + slack)) {
      const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.0f : mn;
      const float alpha = __builtin_amdgcn_exp2f((m - ref) * c2);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
    }
    const float mc = m == -INFINITY ? 0.0f : m * c2;
#pragma unroll
    for (int fr = 0; fr < NF; ++fr) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[fr][i] = __builtin_amdgcn_exp2f(fmaf(s[fr][i], c2, -mc));
        l += s[fr][i];
      }
      // ---- O^T += V^T P^T
      const char* const vt = buf + (fr0 + fr) * (S::KF + S::VF) + S::KF;
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = 8 * (i >> 2) + 4 * half + (i & 3);
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const float v = *reinterpret_cast<const float*>(vt + r * CPR * 16 + (32 * dt + (lane & 31)) * 4);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[fr][i], o[dt], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          sbf16x8_t pb[PP];
          float pv[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) pv[j] = s[fr][8 * ks + j];
          split_bf16x8<PP>(pv, pb);
          // (not all of the frame's operands at once: four registers would spill)
          if constexpr (D == 128 && WQ == 1 && PARTS == 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            // tokens 16 ks + 4 half + 0..3 and 8 more on, columns 32 dt + lane % 32
            const int r = 16 * ks + 4 * half + ((lane & 15) >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const char* at = vt + (lane & 1) * 8;
            const s16x4_t v0 = tr_read(at + (r * CPR + v_chunk<CPR, F32>(r, c)) * 16);
            const s16x4_t v1 = tr_read(at + ((r + 8) * CPR + v_chunk<CPR, F32>(r + 8, c)) * 16);
            typedef short s16x8_t __attribute__((ext_vector_type(8)));
            const s16x8_t vv = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int k = PP - 1; k >= 0; --k)
              o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(sbf16x8_t, vv), pb[k], o[dt], 0, 0, 0);
          }
        }
      }
    }
  };
  auto attend = [&](const Frame (&fs)[FPI], const char* buf) {
#pragma unroll
    for (int fr = 0; fr < FPI; fr += NF)
      if (JOINT || fs[fr].hi > fs[fr].lo) attend_frames(fs, fr, buf);
  };

  for (int t0 = f_lo; t0 < f_hi; t0 += kTable) {
    const int cnt = min(kTable, f_hi - t0);
    __syncthreads();                                    // the table and the tiles are free
    if (tid < cnt) {
      int fa, lo, hi;
      x.frame(t0 + tid, fa, lo, hi);
      int64_t base = hi > lo ? kv_offset(a.kv, b, h, fa) : -1;
      FrameEntry e;
      e.base = base < 0 ? 0 : base;
      e.a = fa;
      e.lo = (int16_t)(base < 0 ? 0 : lo - fa);
      e.hi = (int16_t)(base < 0 ? 0 : hi - fa);
      table[tid] = e;
    }
    __syncthreads();
    const int passes = (cnt + STEP - 1) / STEP, mineoff = tg * FPI;
    auto frames_of = [&](int it, Frame (&f)[FPI]) {
#pragma unroll
      for (int fr = 0; fr < FPI; ++fr) f[fr] = entry(it * STEP + mineoff + fr, cnt);
    };
    Frame now[FPI], next[FPI];
    frames_of(0, now);
    load(now);
    if constexpr (WQ == 1) {
      for (int it = 0; it < passes; ++it) {
        store(now, mine);
        wave_lds_sync();
        frames_of(it + 1, next);
        load(next);
        attend(now, mine);
        wave_lds_sync();
#pragma unroll
        for (int fr = 0; fr < FPI; ++fr) now[fr] = next[fr];
      }
    } else {
      store(now, mine);
      frames_of(1, next);
      load(next);
      __syncthreads();
      for (int it = 0; it < passes; ++it) {
        Frame after[FPI];
        frames_of(it + 2, after);
        attend(now, mine + (it & 1) * S::STAGE);
        store(next, mine + ((it + 1) & 1) * S::STAGE);
        load(after);
        __syncthreads();
#pragma unroll
        for (int fr = 0; fr < FPI; ++fr) { now[fr] = next[fr]; next[fr] = after[fr]; }
      }
    }
  }

  __syncthreads();                                      // the pool is free; s_bad is complete
  if (s_bad[tg] != 0) add_nonfinite<D, F32>(a, x, b, h, q, s_bad[tg], m == -INFINITY ? 0.0f : m, c2, o);

  // ---- join the WT groups through LDS, in group order; the rows leave in their memory order
  l += other_half(l);
  if (half == 0) { s_m[wave][lane] = m; s_l[wave][lane] = l; }
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < WT; ++t) top = fmaxf(top, s_m[t * WQ + wq][lane & 31]);
  const float ref = top == -INFINITY ? 0.0f : top;
  const float scale = __builtin_amdgcn_exp2f((m - ref) * c2);
  float* const wo = reinterpret_cast<float*>(pool) + wave * 32 * D;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int r = lane & 31, d4 = (32 * dt + 2 * i + 4 * half) / 4;
      *reinterpret_cast<float4*>(wo + r * D + 4 * (d4 ^ (r & (D / 4 - 1)))) =
          make_float4(o[dt][i] * scale, o[dt][i + 1] * scale, o[dt][i + 2] * scale, o[dt][i + 3] * scale);
    }
  __syncthreads();
  uint32_t nan = 0;                                     // (a bit a pass)
  for (int idx = tid; idx < WQ * 32 * (D / 4); idx += kTreeThreads) {
    const int rr = idx / (D / 4), d4 = idx % (D / 4), w = rr / 32, r = rr % 32;
    const int row = mt * WQ * 32 + rr;
    if (row >= x.nq * a.G) continue;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int t = 0; t < WT; ++t) mm = fmaxf(mm, s_m[t * WQ + w][r]);
    const float rm = mm == -INFINITY ? 0.0f : mm;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int t = 0; t < WT; ++t) {
      ll += __builtin_amdgcn_exp2f((s_m[t * WQ + w][r] - rm) * c2) * s_l[t * WQ + w][r];
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(pool) + ((t * WQ + w) * 32 + r) * D +
                                                        4 * (d4 ^ (r & (D / 4 - 1))));
      sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
    }
    if (!F32 && has_nan(sum, ll)) nan |= 1u << (idx / kTreeThreads);
    if (p.nsplit == 1) {
      const int i = row / a.G;
      const int64_t at = ((int64_t)b * a.N + i) * a.hq + h * a.G + (row - i * a.G);
      store_row4(p.out, at * D + 4 * d4, sum, ll, a.io_bf16);
      if (d4 == 0 && p.lse) p.lse[at] = ll != 0.0f ? rm * a.c + logf(ll) : -INFINITY;
    } else {
      const int64_t at = part_row(p, part, row);
      *reinterpret_cast<float4*>(p.part_o + at * D + 4 * d4) = sum;
      if (d4 == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(mm * c2, ll);
    }
  }
  if constexpr (!F32) {
    if (__builtin_expect(__ballot(nan != 0) != 0, 0))
      plain_rows<D>(p, x, part, f_lo, f_hi, nan, [&](int k, int t) { return mt * WQ * 32 + (k * kTreeThreads + t) / (D / 4); });
  }
}

template <int D, bool F32>
hipError_t launch_tree_kernels(const TreeParams& p, int wq, int grid, hipStream_t st) {
  const dim3 g(grid), t(kTreeThreads);
  auto go = [&](auto parts) {
    constexpr int P = decltype(parts)::value;
    if (wq == 1) hipLaunchKernelGGL((tree_kernel<D, 1, F32, P>), g, t, 0, st, p);
    else if (wq == 2) hipLaunchKernelGGL((tree_kernel<D, 2, F32, P>), g, t, 0, st, p);
    else hipLaunchKernelGGL((tree_kernel<D, 4, F32, P>), g, t, 0, st, p);
  };
  if constexpr (F32) {
    go(std::integral_constant<int, 1>());
  } else {
    if (p.a.io_bf16) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 3>());
  }
  return hipGetLastError();
}

}  // namespace cobs

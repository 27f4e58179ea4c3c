// Attention weights that cached tokens receive (cobs_attention_weights), on the
// matrix cores.
//
// The work goes by the frames that are attended to (Attended), each of them one
// wave's, so that each weight is written once and no sum depends on an order of
// arrival; in a sparse call more workgroups copy the earlier weights of the other
// positions.  A wave
// loads the keys of its frames (TF at a time) straight into the operand layout, a
// pass ahead; the M = N G query rows of the KV head come from LDS in operand order, 64
// rows (32 of fp32 queries over bf16 keys) a step.  The first pass stages them, and
// what fits in 64 KB (256 rows of 128 bf16) stays there for the workgroup's whole
// work: 64 queries x 4 heads over 8 rows of 32k tokens in 185 us, 214 with every pass
// staging them anew.  More rotate through two buffers, their loads a step ahead.
// S = Q K^T with tokens as columns: a lane holds one token's scores against 4 rows of a tile, so the sum over
// queries and heads of exp2(c2 s - log2(e) lse) is a sum within the lane and, at the
// end, over the four lanes of a token.  16 x 16 products, because a load of their
// key operand covers 64 contiguous bytes of 16 keys; that of 32 x 32 products covers 32
// bytes of 32 keys, whose lines did not stay in the vector cache between the eight
// loads of a frame (4.5 TB/s at 4 rows of 32k tokens).
//
// Bound by HBM (each key once) for few rows: 4 rows of 32k tokens, one fp32 query each,
// 277 MB in 54 us, 5.2 TB/s.  For many, by a SIMD's issue: per 64 scores 16 cycles
// of the matrix core (one bf16 part, d 128) beside some 20 of multiply-add,
// exponential and sum: 256 rows run at 745 TFLOP/s over 8 x 32k tokens, and at 450 over
// 2 x 16k, where the launch, the first keys' loads and the last part are half the time.
#pragma once

#include "cache_device.h"

namespace cobs {

typedef float f32x4w_t __attribute__((ext_vector_type(4)));

constexpr int kWeightsThreads = 256;

template <int D, bool F32, int PARTS>
struct WeightsShape {
  static constexpr int TF = F32 ? 1 : 2;                // frames of a wave's pass
  static constexpr int TG = 2 * TF;                     // groups of 16 tokens
  static constexpr int KS = F32 ? D / 16 : D / 32;      // 16-byte pieces of a lane per row
  static constexpr int TILE = KS * 1024 * PARTS;        // bytes of a staged row tile
  static constexpr int ST = PARTS == 3 ? 2 : 4;         // row tiles of 16 in a buffer (two workgroups' fit a CU)
  static constexpr int STEP = ST * TILE;
  static constexpr int BUFS = PARTS == 1 && !F32 ? 65536 / STEP : 2;   // buffers: 64 KB at most
  static constexpr int PER = ST * KS * 64 / kWeightsThreads;   // staged pieces of a thread
  static constexpr int LPP = PARTS == 1 ? 1 : 2;        // 16-byte loads of a piece
};

constexpr int kCopySpan = 8192;             // positions of a copying workgroup

// Earlier weights (or zeros) of the positions below the window start whose blocks are not selected.
__device__ __forceinline__ void copy_weights(const WeightsParams& p, const Attended& x, int b, int h, int t0,
                                             unsigned long long* s_blocks) {
  const AttendParams& a = p.a;
  // s_blocks: a bit per block of the span
  if (threadIdx.x < kCopySpan / kFrame / 64) s_blocks[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < x.nsel; i += kWeightsThreads) {
    const int at = x.sel[i] - (t0 >> a.lsh);
    if (at >= 0 && at < (kCopySpan >> a.lsh)) atomicOr(&s_blocks[at >> 6], 1ull << (at & 63));
  }
  __syncthreads();
  const int64_t row = ((int64_t)b * a.hkv + h) * a.tmax;
  const int end = min(t0 + kCopySpan, x.ws);
  float v[kCopySpan / kWeightsThreads];
#pragma unroll
  for (int k = 0; k < kCopySpan / kWeightsThreads; ++k) {
    const int t = t0 + k * kWeightsThreads + threadIdx.x;
    v[k] = t < end && p.prev ? p.prev[row + t] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < kCopySpan / kWeightsThreads; ++k) {
    const int t = t0 + k * kWeightsThreads + threadIdx.x;
    const int at = (t - t0) >> a.lsh;
    if (t < end && !((s_blocks[at >> 6] >> (at & 63)) & 1)) p.weights[row + t] = v[k];
  }
}

// The tokens whose sums came out NaN (bit k of a lane's `again`: its token of pass k, in the frame that lane k TF of the wave
// holds), from memory and element by element.  NaN is right of a key with NaN, or of a query that adds.  But rows
// that add nothing take part in the products, with terms exp2(c2 s - inf) that are NaN where s is: with an infinity in the
// key (a row that fills a tile up is zeros) or in such a row's query; and with an infinite key the lower bf16
// parts of a query make NaN.  Rare, so only right; what it needs of the workgroup comes from memory and LDS, as
// scalar registers kept for it through the kernel cost 64 rows of fp32 queries over 8 x 32k tokens 131 us instead of 126.
struct WeightsUnit {
  int b, h, C, nq, passes;
};
template <int D, bool F32, int TF>
__device__ __forceinline__ void weigh_again(unsigned long long again, int my_a, int64_t my_base, const WeightsUnit& unit) {
  const WeightsParams& p = kernel_params<WeightsParams>();
  const AttendParams& a = p.a;
  const int b = unit.b, h = unit.h, C = unit.C, nq = unit.nq, passes = unit.passes;
  const int lane = threadIdx.x & 63;
  const float c2 = a.c * 1.4426950408889634f;
  auto row_of = [&](int r) { return ((int64_t)b * a.N + r / a.G) * a.hq + h * a.G + r % a.G; };
  bool odd = false;                                      // whether a row that adds nothing has a query that is not finite
  for (int r = lane; r < nq * a.G; r += 64)
    if (fabsf(p.lse[row_of(r)]) == INFINITY)
      for (int e = 0; e < D; ++e) odd |= !(fabsf(load_elem(a.q, row_of(r) * D + e, !a.io_bf16)) < INFINITY);
  odd = __ballot(odd) != 0;
  for (int ps = 0; ps < passes; ++ps) {
    const int mine = ps * TF + (TF == 2 ? lane >> 5 : 0);
    const int t = __shfl(my_a, mine, 64) + (lane & 31);
    const int64_t at = __shfl(my_base, mine, 64) + (lane & 31) * (a.kv.table ? (int64_t)a.kv.d : a.kv.st);
    if (!((again >> ps) & 1)) continue;
    bool infinite = false, nan = false;
    for (int e = 0; e < D; ++e) {
      const float k = load_elem(a.kv.k, at + e, F32);
      infinite |= fabsf(k) == INFINITY;
      nan |= k != k;
    }
    float sum = nan || !(infinite || odd) ? NAN : 0.0f;
    for (int r = 0; r < nq * a.G && sum == sum; ++r) {
      const int64_t row = row_of(r);
      const float z = p.lse[row];
      if (fabsf(z) == INFINITY || (t >= C && !((a.mask[(int64_t)b * a.N + r / a.G] >> (t - C)) & 1))) continue;
      float s = 0.0f;
      for (int e = 0; e < D; ++e) s = fmaf(load_elem(a.q, row * D + e, !a.io_bf16), load_elem(a.kv.k, at + e, F32), s);
      sum += __builtin_amdgcn_exp2f(fmaf(s, c2, -z * 1.4426950408889634f));
    }
    const int64_t w = ((int64_t)b * a.hkv + h) * a.tmax + t;
    p.weights[w] = (p.prev ? p.prev[w] : 0.0f) + sum;
  }
}

template <int D, bool F32, int PARTS>
__global__ __launch_bounds__(kWeightsThreads, 2) void weights_kernel(WeightsParams p) {
  using S = WeightsShape<D, F32, PARTS>;
  constexpr int TF = S::TF, TG = S::TG, KS = S::KS, PER = S::PER, kStepTiles = S::ST;
  constexpr int ES = F32 ? 4 : 2;
  __shared__ __align__(16) char tiles[S::BUFS * S::STEP];
  __shared__ __align__(16) float s_lse[S::BUFS][kStepTiles * 16];          // log2 units; +inf: adds nothing
  __shared__ __align__(16) unsigned long long s_bits[S::BUFS][kStepTiles * 16];
  __shared__ unsigned long long s_live[S::BUFS];                           // rows that add something
  __shared__ int red[4];
  __shared__ WeightsUnit s_unit;
  const AttendParams& a = p.a;
  const int h = blockIdx.x;
  int b = blockIdx.y, n_parts = p.parts;
  int part = p.parts - 1 - (int)blockIdx.z;             // the draft's frames and the longer parts first
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_uniform32(tid >> 6), quad = lane >> 4;
  if (p.even) {
    int n, before;
    row_parts(a, p.parts, 4 * TF, n, before);
    const int j = (int)blockIdx.y * p.parts + part;
    const unsigned long long mine = __ballot(j >= before && j < before + n);
    if (mine == 0) return;
    b = __builtin_ctzll(mine);
    part = j - __builtin_amdgcn_readlane(before, b);
    n_parts = __builtin_amdgcn_readlane(n, b);
  }
  const Attended x = attended<kWeightsThreads>(a, b, h, red);
  if (part < 0) {
    static_assert(kCopySpan / kFrame / 64 <= 2 * kStepTiles * 16, "the span's block bits fit s_bits");
    copy_weights(p, x, b, h, (-1 - part) * kCopySpan, &s_bits[0][0]);
    return;
  }
  const int nf = x.frames(), all = (nf + 4 * TF - 1) / (4 * TF);
  const int pass0 = first_pass(all, part, n_parts), passes = first_pass(all, part + 1, n_parts) - pass0;
  if (passes == 0) return;
  if (tid == 0) s_unit = {b, h, x.C, x.nq, passes};          // (read behind the barrier of the first rows)
  const int F0 = pass0 * 4 * TF;
  const int M = x.nq * a.G;
  const float c2 = a.c * 1.4426950408889634f;

  // lane f: the wave's frame f (pass f / TF): position, live tokens, first row
  int my_a = 0, my_lo = 0, my_hi = 0;
  int64_t my_base = 0;
  if (lane < passes * TF) {
    const int f = F0 + ((lane / TF) * 4 + wave) * TF + lane % TF;
    if (f < nf) {
      int lo, hi;
      x.frame(f, my_a, lo, hi);
      if (lo < hi) {
        my_lo = lo - my_a;
        my_hi = hi - my_a;
        my_base = kv_offset(a.kv, b, h, my_a);
      }
    }
  }
  const int64_t rs = a.kv.table ? a.kv.d : a.kv.st;
  const int64_t my_row = (int64_t)(lane & 15) * rs * ES + quad * 16;
  const int64_t wrow = ((int64_t)b * a.hkv + h) * a.tmax;

  auto base_of = [&](int at) {
    const uint32_t l32 = __builtin_amdgcn_readlane((uint32_t)my_base, at);
    const uint32_t h32 = __builtin_amdgcn_readlane((uint32_t)((uint64_t)my_base >> 32), at);
    return (int64_t)(((uint64_t)h32 << 32) | l32);
  };
  uint4 kn[TG][KS];                           // the next pass's keys
  auto load = [&](int ps) {
#pragma unroll
    for (int f = 0; f < TF; ++f) {
      const int at = ps * TF + f;
      if (__builtin_amdgcn_readlane(my_hi, at) == 0) continue;
      const int64_t base = base_of(at);
      if (base < 0) continue;                 // a page out of range
      const char* k = static_cast<const char*>(a.kv.k) + base * ES + my_row;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int s = 0; s < KS; ++s) kn[2 * f + g][s] = *reinterpret_cast<const uint4*>(k + 16 * g * rs * ES + s * 64);
    }
  };

  // ---- staging: lane l of piece s of a tile holds row l % 16, 16 bytes (fp32 queries
  // over bf16 keys: 8 values) at 4 s + l / 16
  uint4 qx[PER][S::LPP];
  float qz = INFINITY;
  unsigned long long qbits = 0;
  // (16 rows further the query is 16 / G on and the head the same: a constant stride)
  const int64_t qstride = (int64_t)(16 >> p.lg) * a.hq * D * (a.io_bf16 ? 2 : 4);
  const int r16 = lane & 15;
  const char* const qrow = static_cast<const char*>(a.q) +
                           ((((int64_t)b * a.N + (r16 >> p.lg)) * a.hq + h * a.G + (r16 & (a.G - 1))) * D +
                            (F32 ? 4 * quad : 8 * quad)) * (a.io_bf16 ? 2 : 4);
  auto fetch = [&](int step) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int piece = wave + 4 * j, tl = piece / KS, s = piece % KS;
      const int r = (step * kStepTiles + tl) * 16 + r16;
      const char* q = qrow + (step * kStepTiles + tl) * qstride + (F32 ? 16 : 32) * s * (a.io_bf16 ? 2 : 4);
#pragma unroll
      for (int k = 0; k < S::LPP; ++k) qx[j][k] = make_uint4(0, 0, 0, 0);
      if (r < M) {
        if (F32 && a.io_bf16) {
          const uint2 v = *reinterpret_cast<const uint2*>(q);
          qx[j][0] = make_uint4(v.x << 16, v.x & 0xffff0000u, v.y << 16, v.y & 0xffff0000u);
        } else {
#pragma unroll
          for (int k = 0; k < S::LPP; ++k) qx[j][k] = reinterpret_cast<const uint4*>(q)[k];
        }
      }
    }
    if (wave == 0 && lane < 16 * kStepTiles) {
      const int r = step * kStepTiles * 16 + lane, i = r >> p.lg;
      qz = INFINITY;
      qbits = 0;
      if (r < M) {
        qz = p.lse[((int64_t)b * a.N + i) * a.hq + h * a.G + (r - (i << p.lg))];
        if (a.mask) qbits = a.mask[(int64_t)b * a.N + i];
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int piece = wave + 4 * j, tl = piece / KS, s = piece % KS;
      char* dst = tiles + buf * S::STEP + tl * S::TILE + s * 1024 + lane * 16;
      if constexpr (PARTS == 1) {
        *reinterpret_cast<uint4*>(dst) = qx[j][0];
      } else {
        const float v[8] = {__uint_as_float(qx[j][0].x), __uint_as_float(qx[j][0].y), __uint_as_float(qx[j][0].z),
                            __uint_as_float(qx[j][0].w), __uint_as_float(qx[j][1].x), __uint_as_float(qx[j][1].y),
                            __uint_as_float(qx[j][1].z), __uint_as_float(qx[j][1].w)};
        sbf16x8_t w[PARTS];
        split_bf16x8<PARTS>(v, w);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) *reinterpret_cast<sbf16x8_t*>(dst + k * KS * 1024) = w[k];
      }
    }
    if (wave == 0) {
      const float z = qz == -INFINITY ? INFINITY : qz * 1.4426950408889634f;
      if (lane < 16 * kStepTiles) {
        s_lse[buf][lane] = z;
        s_bits[buf][lane] = z != INFINITY ? qbits : 0;    // (a row that adds nothing sees no draft)
      }
      const unsigned long long live = __ballot(z != INFINITY);
      if (lane == 0) s_live[buf] = live;
    }
  };
  static_assert(kStepTiles * 16 <= 64, "one wave holds a step's normalisers");

  const int steps = (M + kStepTiles * 16 - 1) / (kStepTiles * 16);
  const bool resident = steps <= S::BUFS;               // the first pass stages them all
  if (steps > 0) {
    fetch(0);
    load(0);
    put(0);
    if (steps > 1) fetch(1);
    __syncthreads();
  }
  unsigned long long again = 0;                                              // passes in which the lane's sum is NaN
  int n = 0;                                                                 // steps done
  for (int ps = 0; ps < passes; ++ps) {
    uint4 kc[TG][KS];
#pragma unroll
    for (int g = 0; g < TG; ++g)
#pragma unroll
      for (int s = 0; s < KS; ++s) kc[g][s] = kn[g][s];
    // lane l writes token l of the pass (fp32 caches: 32 tokens)
    const int mine = ps * TF + (TF == 2 ? lane >> 5 : 0), r32 = lane & 31;
    const int fa = __shfl(my_a, mine, 64), flo = __shfl(my_lo, mine, 64), fhi = __shfl(my_hi, mine, 64);
    const bool writes = lane < 32 * TF && r32 >= flo && r32 < fhi;
    float prev = 0.0f;
    if (writes && p.prev) prev = p.prev[wrow + fa + r32];
    if (steps > 0 && ps + 1 < passes) load(ps + 1);
    float sum[TG];
    bool good[TF], any = false, drafted = false;          // drafted: a frame reaches into the draft
#pragma unroll
    for (int g = 0; g < TG; ++g) sum[g] = 0.0f;
#pragma unroll
    for (int f = 0; f < TF; ++f) {
      good[f] = __builtin_amdgcn_readlane(my_hi, ps * TF + f) > 0 && base_of(ps * TF + f) >= 0;
      any |= good[f];
      drafted |= __builtin_amdgcn_readlane(my_a, ps * TF + f) + __builtin_amdgcn_readlane(my_hi, ps * TF + f) > x.C;
    }
    for (int st = 0; st < steps; ++st, ++n) {
      const int buf = resident ? st : (n & 1);
      const bool more = resident ? ps == 0 && st + 1 < steps : st + 1 < steps || ps + 1 < passes;
      if (any && s_live[buf] != 0) {
        auto scores = [&](int tl, f32x4w_t (&sc)[TG]) {
          const char* qt = tiles + buf * S::STEP + tl * S::TILE;
#pragma unroll
          for (int g = 0; g < TG; ++g) sc[g] = f32x4w_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            if constexpr (F32) {
              const float4 q = *reinterpret_cast<const float4*>(qt + s * 1024 + lane * 16);
#pragma unroll
              for (int g = 0; g < TG; ++g) {
                sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(q.x, __uint_as_float(kc[g][s].x), sc[g], 0, 0, 0);
                sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(q.y, __uint_as_float(kc[g][s].y), sc[g], 0, 0, 0);
                sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(q.z, __uint_as_float(kc[g][s].z), sc[g], 0, 0, 0);
                sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(q.w, __uint_as_float(kc[g][s].w), sc[g], 0, 0, 0);
              }
            } else {
#pragma unroll
              for (int k = PARTS - 1; k >= 0; --k) {
                const sbf16x8_t q = *reinterpret_cast<const sbf16x8_t*>(qt + (k * KS + s) * 1024 + lane * 16);
#pragma unroll
                for (int g = 0; g < TG; ++g)
                  sc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, __builtin_bit_cast(sbf16x8_t, kc[g][s]), sc[g], 0, 0, 0);
              }
            }
          }
        };
        // normalisers of rows 4 quad + i of a tile
        auto normalisers = [&](int tl, float (&z)[4]) {
          const float4 v = *reinterpret_cast<const float4*>(&s_lse[buf][tl * 16 + 4 * quad]);
          z[0] = v.x; z[1] = v.y; z[2] = v.z; z[3] = v.w;
        };
        const int nt = min(kStepTiles, (M + 15) / 16 - st * kStepTiles);      // the step's tiles that hold rows
        auto add = [&](const f32x4w_t (&sc)[TG], const float (&z)[4]) {
#pragma unroll
          for (int g = 0; g < TG; ++g) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(sc[g][i], c2, -z[i]));
            sum[g] += (e[0] + e[1]) + (e[2] + e[3]);
          }
        };
        if (PARTS == 1 && !F32 && !drafted && nt == kStepTiles) {
          // straight-line code: a tile's products among the exponentials of the tile before (more
          // parts or fp32 keys leave no registers for it: the spilled values cost a wait a pass)
          f32x4w_t sc[2][TG];
          scores(0, sc[0]);
#pragma unroll
          for (int tl = 0; tl < kStepTiles; ++tl) {
            float z[4];
            normalisers(tl, z);
            if (tl + 1 < kStepTiles) scores(tl + 1, sc[(tl + 1) & 1]);
            add(sc[tl & 1], z);
          }
        } else if (!drafted) {
#pragma unroll 1
          for (int tl = 0; tl < nt; ++tl) {
            f32x4w_t sc[TG];
            float z[4];
            scores(tl, sc);
            normalisers(tl, z);
            add(sc, z);
          }
        } else {
#pragma unroll 1
          for (int tl = 0; tl < nt; ++tl) {
            f32x4w_t sc[TG];
            float z[4];
            unsigned long long bits[4];
            normalisers(tl, z);
#pragma unroll
            for (int i = 0; i < 4; ++i) bits[i] = s_bits[buf][tl * 16 + 4 * quad + i];
            scores(tl, sc);
            // bit t of a row's word for a frame: whether the row sees token t of it (the context's: all rows)
#pragma unroll
            for (int f = 0; f < TF; ++f) {
              const int to_c = x.C - __builtin_amdgcn_readlane(my_a, ps * TF + f);
              const int left = min(max(to_c, 0), kFrame), right = min(max(-to_c, 0), 63);
              const uint32_t context = (uint32_t)((1ull << left) - 1);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t see = ((uint32_t)((bits[i] << left) >> right) | context) >> (lane & 15);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                  const float e = __builtin_amdgcn_exp2f(fmaf(sc[2 * f + g][i], c2, -z[i]));
                  sum[2 * f + g] += (see >> (16 * g)) & 1u ? e : 0.0f;
                }
              }
            }
          }
        }
      }
      if (more) {
        put(resident ? st + 1 : (n + 1) & 1);
        if (!resident || st + 2 < steps) fetch((st + 2) % steps);
        __syncthreads();
      }
    }
    float total = 0.0f;
#pragma unroll
    for (int g = 0; g < TG; ++g) {
      float v = sum[g];
      v += __shfl_xor(v, 16, 64);
      v += other_half(v);
      if (quad == g) total = good[g / 2] ? v : 0.0f;
    }
    if (total == total) {
      if (writes) p.weights[wrow + fa + r32] = prev + total;
    } else if (writes) {
      again |= 1ull << ps;
    }
  }
  if (__builtin_expect(__ballot(again != 0) != 0, 0))
    weigh_again<D, F32, TF>(again, my_a, my_base, s_unit);
}

template <int D, bool F32>
hipError_t launch_weights_kernels(WeightsParams p, hipStream_t st) {
  // a wave's lanes hold its frames: at most 64
  constexpr int TF = F32 ? 1 : 2, PASS = 4 * TF;
  const int frames = max_frames(p.a);
  // a pass of up to 64 rows is bound by HBM (2 us); each 64 of more rows take 3 us (fp32 keys or queries: 6)
  const int steps = (p.a.N * p.a.G + 63) / 64;
  // a sparse call's copies of the other positions, not needed in place, follow as more parts (each about
  // half a part's time)
  const int64_t units = (int64_t)p.a.hkv * p.a.B;
  const int copies = p.a.sparse && p.prev != p.weights ? (p.a.tmax + kCopySpan - 1) / kCopySpan : 0;
  p.parts = parts_of((frames + PASS - 1) / PASS, units, steps == 1 ? 2.0 : steps * (F32 || !p.a.io_bf16 ? 6.0 : 3.0), 64 / TF, 32768,
                     units * copies / 2);
  // (the longest row gets p.parts at least, another at least (p.parts - 1) / frames of them per frame: parts of some
  // 28 passes stay below the 64 frames of a wave with the rounding of both)
  p.even = parts_by_length(p.a, p.parts) && frames <= (int64_t)(TF == 2 ? 28 : 56) * PASS * (p.parts - 1);
  p.lg = p.a.G == 1 ? 0 : (p.a.G == 2 ? 1 : (p.a.G == 4 ? 2 : (p.a.G == 8 ? 3 : 4)));
  const dim3 grid(p.a.hkv, p.a.B, p.parts + copies), t(kWeightsThreads);
  if constexpr (F32) {
    hipLaunchKernelGGL((weights_kernel<D, true, 1>), grid, t, 0, st, p);
  } else {
    if (p.a.io_bf16) hipLaunchKernelGGL((weights_kernel<D, false, 1>), grid, t, 0, st, p);
    else hipLaunchKernelGGL((weights_kernel<D, false, 3>), grid, t, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace cobs

// Attention weights that cached tokens receive (cobs_attention_weights), on the
// matrix cores.
//
// The work goes by position, so that each weight is written once and no sum
// depends on an order of arrival.  A wave owns frames of 32 positions (TF at a
// time) whose keys it loads straight into the operand layout, a pass ahead; the
// M = N G query rows of the KV head come from LDS, staged once a workgroup in
// operand order (128 rows at a time where there are more).  S = Q K^T with tokens
// as columns: a lane holds one token's scores against 16 rows of a tile, so the sum
// over queries and heads of exp2(c2 s - log2(e) lse) is a sum within the lane and
// one exchange between the halves of the wave.
//
// Bound by HBM (each key once) up to M ~ 256, then by the exponentials: 24 cycles
// of a SIMD per 64 scores beside 32 of the matrix core's (one bf16 part).
#pragma once

#include "cache_device.h"

namespace cobs {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kWeightsThreads = 256;
constexpr int kWeightsTiles = 4;            // row tiles of 32 staged at a time

template <int D, bool F32, int PARTS>
struct WeightsShape {
  static constexpr int TF = F32 ? 1 : 2;                // frames of a wave's pass
  static constexpr int KS = F32 ? D / 8 : D / 16;       // 16-byte pieces of a lane per row
  static constexpr int TILE = KS * 1024 * PARTS;        // bytes of a staged row tile
  static constexpr int MAXP = 8;                        // passes of a workgroup: 64 blocks of 32 at most
};

template <int D, bool F32, int PARTS>
__global__ __launch_bounds__(kWeightsThreads, 2) void weights_kernel(WeightsParams p) {
  using S = WeightsShape<D, F32, PARTS>;
  constexpr int TF = S::TF, KS = S::KS;
  __shared__ __align__(16) char tiles[kWeightsTiles * S::TILE];
  __shared__ __align__(16) float s_lse[kWeightsTiles * 32];          // log2 units; +inf: adds nothing
  __shared__ __align__(16) unsigned long long s_bits[kWeightsTiles * 32];
  __shared__ unsigned long long s_blocks;
  __shared__ int red[4];
  const AttendParams& a = p.a;
  const int h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_uniform32(tid >> 6), half = lane >> 5;
  const int T0 = blockIdx.x * (p.passes * 4 * TF * kFrame);
  if (tid == 0) s_blocks = 0;
  const Attended x = attended<kWeightsThreads>(a, b, h, red);
  if (T0 >= x.E) return;
  const int M = x.nq * a.G;
  const float c2 = a.c * 1.4426950408889634f;
  // selected blocks within the workgroup's positions, one bit each
  if (a.sparse) {
    __syncthreads();
    for (int i = tid; i < x.nsel; i += kWeightsThreads) {
      const int at = x.sel[i] - (T0 >> a.lsh);
      if (at >= 0 && at < 64) atomicOr(&s_blocks, 1ull << at);
    }
    __syncthreads();
  }
  // lane f: the wave's frame f (pass f / TF)
  int my_lo = 0, my_hi = 0;
  int64_t my_base = 0;
  const int frames = p.passes * TF;
  if (lane < frames) {
    const int t0 = T0 + (((lane / TF) * 4 + wave) * TF + lane % TF) * kFrame;
    int lo = t0;
    if (a.sparse && !((s_blocks >> ((t0 >> a.lsh) - (T0 >> a.lsh))) & 1)) lo = max(t0, x.ws);
    const int hi = min(t0 + kFrame, x.E);
    if (lo < hi && M > 0) {
      const int64_t base = kv_offset(a.kv, b, h, t0);
      if (base >= 0) { my_base = base; my_lo = lo - t0; my_hi = hi - t0; }
    }
  }
  const int64_t rs = a.kv.table ? a.kv.d : a.kv.st;
  constexpr int ES = F32 ? 4 : 2;
  const int64_t my_row = (int64_t)(lane & 31) * rs * ES + half * 16;

  uint4 kn[TF][KS];                           // the next pass's keys
  auto load = [&](int ps) {
#pragma unroll
    for (int f = 0; f < TF; ++f) {
      const int at = ps * TF + f;
      const int hi = __builtin_amdgcn_readlane(my_hi, at);
      if (hi <= __builtin_amdgcn_readlane(my_lo, at)) continue;
      const uint32_t lo32 = __builtin_amdgcn_readlane((uint32_t)my_base, at);
      const uint32_t hi32 = __builtin_amdgcn_readlane((uint32_t)((uint64_t)my_base >> 32), at);
      const char* k = static_cast<const char*>(a.kv.k) + (int64_t)(((uint64_t)hi32 << 32) | lo32) * ES + my_row;
#pragma unroll
      for (int s = 0; s < KS; ++s) kn[f][s] = *reinterpret_cast<const uint4*>(k + s * 32);
    }
  };
  // rows of tile tl of the staged round: lane l of piece s holds row l % 32, 16 bytes at 2 s + l / 32
  auto stage = [&](int first, int tiles_n) {
    for (int it = tid; it < tiles_n * KS * 64; it += kWeightsThreads) {
      const int tl = it / (KS * 64), s = it / 64 % KS, ln = it & 63;
      const int r = first + tl * 32 + (ln & 31), i = r / a.G;
      const int64_t at = ((int64_t)b * a.N + i) * a.hq + h * a.G + (r - i * a.G);
      char* dst = tiles + tl * S::TILE + s * 1024 + ln * 16;
      if constexpr (F32) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const int e = 8 * s + 4 * (ln >> 5);
        if (r < M) {
          v.x = load_elem(a.q, at * D + e, !a.io_bf16);
          v.y = load_elem(a.q, at * D + e + 1, !a.io_bf16);
          v.z = load_elem(a.q, at * D + e + 2, !a.io_bf16);
          v.w = load_elem(a.q, at * D + e + 3, !a.io_bf16);
        }
        *reinterpret_cast<float4*>(dst) = v;
      } else if constexpr (PARTS == 1) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < M) v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at * D + 16 * s + 8 * (ln >> 5));
        *reinterpret_cast<uint4*>(dst) = v;
      } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (r < M) {
          const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at * D + 16 * s + 8 * (ln >> 5));
          const float4 q0 = q[0], q1 = q[1];
          v[0] = q0.x; v[1] = q0.y; v[2] = q0.z; v[3] = q0.w;
          v[4] = q1.x; v[5] = q1.y; v[6] = q1.z; v[7] = q1.w;
        }
        sbf16x8_t w[PARTS];
        split_bf16x8<PARTS>(v, w);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) *reinterpret_cast<sbf16x8_t*>(dst + k * KS * 1024) = w[k];
      }
    }
    for (int r0 = tid; r0 < tiles_n * 32; r0 += kWeightsThreads) {
      const int r = first + r0, i = r / a.G;
      float z = INFINITY;
      unsigned long long bits = 0;
      if (r < M) {
        const float v = p.lse[((int64_t)b * a.N + i) * a.hq + h * a.G + (r - i * a.G)];
        z = v == -INFINITY ? INFINITY : v * 1.4426950408889634f;
        if (a.mask) bits = a.mask[(int64_t)b * a.N + i];
      }
      s_lse[r0] = z;
      s_bits[r0] = bits;
    }
  };

  const int rounds = (M + kWeightsTiles * 32 - 1) / (kWeightsTiles * 32);
  if (rounds > 0) load(0);
  for (int ps = 0; ps < p.passes; ++ps) {
    const int p0 = T0 + (ps * 4 * TF) * kFrame;
    if (p0 >= x.E) break;                            // the same for all waves
    uint4 kc[TF][KS];
#pragma unroll
    for (int f = 0; f < TF; ++f)
#pragma unroll
      for (int s = 0; s < KS; ++s) kc[f][s] = kn[f][s];
    if (rounds > 0 && ps + 1 < p.passes) load(ps + 1);
    float sum[TF];
#pragma unroll
    for (int f = 0; f < TF; ++f) sum[f] = 0.0f;
    bool any = false;
#pragma unroll
    for (int f = 0; f < TF; ++f)
      any |= __builtin_amdgcn_readlane(my_hi, ps * TF + f) > __builtin_amdgcn_readlane(my_lo, ps * TF + f);
    for (int rd = 0; rd < rounds; ++rd) {
      const int first = rd * kWeightsTiles * 32, tiles_n = min(kWeightsTiles, (M - first + 31) / 32);
      if (rounds > 1 || ps == 0) {
        __syncthreads();                             // the staged rows are free
        stage(first, tiles_n);
        __syncthreads();
      }
      if (!any) continue;
      for (int tl = 0; tl < tiles_n; ++tl) {
        const char* qt = tiles + tl * S::TILE;
        f32x16_t sc[TF];
#pragma unroll
        for (int f = 0; f < TF; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[f][i] = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if constexpr (F32) {
            const float4 q = *reinterpret_cast<const float4*>(qt + s * 1024 + lane * 16);
#pragma unroll
            for (int f = 0; f < TF; ++f) {
              sc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(q.x, __uint_as_float(kc[f][s].x), sc[f], 0, 0, 0);
              sc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(q.y, __uint_as_float(kc[f][s].y), sc[f], 0, 0, 0);
              sc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(q.z, __uint_as_float(kc[f][s].z), sc[f], 0, 0, 0);
              sc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(q.w, __uint_as_float(kc[f][s].w), sc[f], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k) {
              const sbf16x8_t q = *reinterpret_cast<const sbf16x8_t*>(qt + (k * KS + s) * 1024 + lane * 16);
#pragma unroll
              for (int f = 0; f < TF; ++f)
                sc[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, __builtin_bit_cast(sbf16x8_t, kc[f][s]), sc[f], 0, 0, 0);
            }
          }
        }
        float z[16];                                 // rows 8 (i / 4) + 4 half + i % 4 of the tile
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 v = *reinterpret_cast<const float4*>(&s_lse[tl * 32 + 2 * i + 4 * half]);
          z[i] = v.x; z[i + 1] = v.y; z[i + 2] = v.z; z[i + 3] = v.w;
        }
        bool live = false;                           // a tile that adds nothing adds no NaN either
#pragma unroll
        for (int i = 0; i < 16; ++i) live |= z[i] != INFINITY;
        if (!__ballot(live)) continue;
#pragma unroll
        for (int f = 0; f < TF; ++f) {
          const int t0 = p0 + (wave * TF + f) * kFrame;
          if (t0 + kFrame <= x.C) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[f] += __builtin_amdgcn_exp2f(fmaf(sc[f][i], c2, -z[i]));
          } else {
            // drafted tokens: the rows that see them
            const int j = t0 + (lane & 31) - x.C;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const unsigned long long bits = s_bits[tl * 32 + 8 * (i >> 2) + 4 * half + (i & 3)];
              const bool see = (j < 0) | (((bits >> (j & 63)) & 1) != 0);
              const float e = __builtin_amdgcn_exp2f(fmaf(sc[f][i], c2, -z[i]));
              sum[f] += (see & (z[i] != INFINITY)) ? e : 0.0f;
            }
          }
        }
      }
    }
#pragma unroll
    for (int f = 0; f < TF; ++f) {
      const int at = ps * TF + f, lo = __builtin_amdgcn_readlane(my_lo, at), hi = __builtin_amdgcn_readlane(my_hi, at);
      const float total = sum[f] + other_half(sum[f]);
      const int r = lane & 31, t = p0 + (wave * TF + f) * kFrame + r;
      if (half == 0 && t < x.E) {
        const int64_t w = ((int64_t)b * a.hkv + h) * a.tmax + t;
        const bool in = r >= lo && r < hi;
        if (in || p.prev != p.weights) p.weights[w] = (p.prev ? p.prev[w] : 0.0f) + (in ? total : 0.0f);
      }
    }
  }
}

template <int D, bool F32>
hipError_t launch_weights_kernels(WeightsParams p, hipStream_t st) {
  // as many passes of a workgroup (its staged queries serve them all) as leave
  // the chip's 256 CUs two rounds of two workgroups
  constexpr int TOK = 4 * (F32 ? 1 : 2) * kFrame;
  const int64_t one = (int64_t)((p.a.tmax + TOK - 1) / TOK) * p.a.hkv * p.a.B;
  int64_t passes = one / 1024;
  passes = passes < 1 ? 1 : (passes > 8 ? 8 : passes);
  p.passes = (int)passes;
  const int64_t span = TOK * passes;
  const dim3 grid((unsigned)((p.a.tmax + span - 1) / span), p.a.hkv, p.a.B), t(kWeightsThreads);
  if constexpr (F32) {
    hipLaunchKernelGGL((weights_kernel<D, true, 1>), grid, t, 0, st, p);
  } else {
    if (p.a.io_bf16) hipLaunchKernelGGL((weights_kernel<D, false, 1>), grid, t, 0, st, p);
    else hipLaunchKernelGGL((weights_kernel<D, false, 2>), grid, t, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace cobs

// Device helpers of the token operators: rotary positions and e4m3 codes.
#pragma once

#include "cache_device.h"
#include "tokens_kernels.h"

namespace cobs {

// Cosine and sine of t f, |t f| <= 2^51 (NaN beyond): the product in two fp64 halves, as it has up to 55 bits, reduced to |x| <= pi / 4
// (n quarter turns taken off in two parts, after Cody and Waite), then power series, whose next terms are below 2^-28.
// Past 2^51 n would be no integer that kMagic's sum holds.
__device__ __forceinline__ float2 cos_sin(double t, double f) {
  constexpr double kMagic = 6755399441055744.0;                 // 1.5 * 2^52: its sum's low bits are the integer
  const double a = t * f, rest = fma(t, f, -a);
  const double turns = fma(a, 0.6366197723675814, kMagic), n = turns - kMagic;
  const double y = fma(-n, 1.5707963267948966, a) + fma(-n, 6.123233995736766e-17, rest);
  const float x = fabs(a) <= 2251799813685248.0 ? (float)y : __uint_as_float(0x7fc00000u);
  const int quarter = __double2loint(turns);
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const float u = quarter & 1 ? s : c, v = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -u : u, quarter & 2 ? -v : v);
}

// Cosine and sine, times the rotation's scale, of pair `pair` at position `t`.
__device__ __forceinline__ float2 turn_of(const RopeView& r, int t, int pair) {
  const float2 y = cos_sin((double)t, (double)r.freq[pair]);
  return make_float2(y.x * r.scale, y.y * r.scale);
}

// Sixteen elements of a D-element head that one thread holds: a run of 8 in each half of the rotated part, both sides of eight
// pairs (half layout) or four pairs each (interleaved), or in each half of what is left as it is.  So neighbours' runs are next to each
// other in memory (32000 tokens of 32 heads, interleaved: 98 us; with a thread's 16 elements in a row 106).
struct Piece {
  int e0, e1;          // first elements of the runs
  bool turned;
};
template <int D>
__device__ __forceinline__ Piece piece_of(const RopeView& r, int p) {
  Piece x;
  x.turned = 8 * p < r.half;
  x.e0 = x.turned ? 8 * p : 8 * p + r.half;
  x.e1 = x.e0 + (x.turned ? r.half : D / 2 - r.half);
  return x;
}
// The pair j < 8 of piece p.
__device__ __forceinline__ int pair_of(const RopeView& r, int p, int j) {
  return r.interleaved ? 4 * p + (j & 3) + (j >> 2) * (r.half >> 1) : 8 * p + j;
}

// Eight elements in memory, 16-byte aligned: fp32 or bf16.
struct Raw8 { uint4 a, b; };
__device__ __forceinline__ Raw8 load_raw8(const void* p, int64_t i, bool f32) {
  Raw8 x = {};
  if (f32) {
    const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
    x.a = s[0];
    x.b = s[1];
  } else {
    x.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
  }
  return x;
}
__device__ __forceinline__ void widen8(const Raw8& r, bool f32, float* x) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = f32 ? __uint_as_float(w[i]) : (i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]));
}
__device__ __forceinline__ void store8(void* p, int64_t i, bool f32, const float* x) {
  if (f32) {
    float4* s = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    s[0] = make_float4(x[0], x[1], x[2], x[3]);
    s[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) =
        make_uint4(f32x2_to_bf16x2_rne(x[0], x[1]), f32x2_to_bf16x2_rne(x[2], x[3]), f32x2_to_bf16x2_rne(x[4], x[5]),
                   f32x2_to_bf16x2_rne(x[6], x[7]));
  }
}

// The sixteen elements of a turned piece, by the (cos, sin) of its eight pairs.
__device__ __forceinline__ void turn16(float (&x)[16], const float2 (&cs)[8], bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float lo = x[2 * j], hi = x[2 * j + 1];
      x[2 * j] = lo * cs[j].x - hi * cs[j].y;
      x[2 * j + 1] = hi * cs[j].x + lo * cs[j].y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float lo = x[j], hi = x[8 + j];
      x[j] = lo * cs[j].x - hi * cs[j].y;
      x[8 + j] = hi * cs[j].x + lo * cs[j].y;
    }
  }
}

// A row's cached tokens before the call, and its new tokens.
struct NewRow {
  int T, n;
};
__device__ __forceinline__ NewRow new_row(const NewTokens& p, int b) {
  NewRow r;
  r.T = p.seq_lens ? clamp_len(p.seq_lens[b], p.tmax) : 0;
  r.n = p.new_lens ? clamp_len(p.new_lens[b], p.N) : p.N;
  return r;
}

// new_seq_lens, by the threads of one workgroup.
__device__ __forceinline__ void write_lens(const NewTokens& p) {
  if (!p.new_seq_lens) return;
  for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
    const NewRow r = new_row(p, b);
    p.new_seq_lens[b] = min(r.n, p.tmax - r.T) + r.T;
  }
}

}  // namespace cobs

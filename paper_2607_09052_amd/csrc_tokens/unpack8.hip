// cobs_unpack8: blocks of an 8-bit cache as bf16 or fp32.  A copy, bound by HBM (three times the codes' bytes for bf16).
// A thread takes 8 codes of a token's head, or 4 for fp32, 16 bytes out; a workgroup a block's keys or values.
// Measured (d 128, 8 heads): 4 rows of 32741 tokens as bf16, 805 MB, in 140 us, 5.7 TB/s (a large copy: 5.0); as fp32 236 us, 5.7 TB/s;
// the newest block of 32 rows 4.5 us.
#include "tokens_device.h"

namespace cobs {

constexpr int kUnpackThreads = 256;

// grid: (block and row, KV head, keys or values)
template <int D, bool F32>
__global__ __launch_bounds__(kUnpackThreads) void unpack8_kernel(Unpack8Params p) {
  constexpr int E = F32 ? 4 : 8, TPR = D / E, U = 4;      // elements of a thread; its loads under way together
  using Codes = std::conditional_t<F32, uint32_t, uint2>;
  const int b = p.first_row + blockIdx.x / p.num, which = blockIdx.x % p.num, h = blockIdx.y, value = blockIdx.z;
  const int T = clamp_len(p.seq_lens[b], p.tmax), lsh = p.src.lsh;
  const int blocks = blocks_of(T, lsh);
  const int j = (p.first >= 0 ? p.first : max(0, blocks - p.num)) + which;
  if (j >= blocks) return;
  const int64_t from = kv_offset(p.src, b, h, j << lsh), to = kv_offset(p.dst, b, h, j << lsh);
  if (from < 0 || to < 0) return;
  const int64_t at = p.src.table ? from / ((int64_t)D << lsh) : ((int64_t)b * p.hkv + h) * p.src.nbmax + j;
  const float scale = (value ? p.v_scale : p.k_scale)[at];
  const uint8_t* const codes = static_cast<const uint8_t*>(value ? p.src.v : p.src.k) + from;
  void* const out = const_cast<void*>(value ? p.dst.v : p.dst.k);
  const int64_t rs = p.src.table ? D : p.src.st, ws = p.dst.table ? D : p.dst.st;
  const int rows = min(1 << lsh, T - (j << lsh));
  // (stores of 16 bytes next to each other: with 16 codes a thread, whose stores lie 32 or 64 bytes apart, 154 and 389 us
  // for 140 and 236)
  for (int x0 = threadIdx.x; x0 < rows * TPR; x0 += U * kUnpackThreads) {
    Codes w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * kUnpackThreads;
      if (x < rows * TPR) w[u] = *reinterpret_cast<const Codes*>(codes + (x / TPR) * rs + E * (x % TPR));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * kUnpackThreads;
      if (x >= rows * TPR) continue;
      const int64_t at = to + (x / TPR) * ws + E * (x % TPR);
      float y[E];
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        const int c = reinterpret_cast<const int*>(&w[u])[i];
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
        y[4 * i] = lo[0] * scale;
        y[4 * i + 1] = lo[1] * scale;
        y[4 * i + 2] = hi[0] * scale;
        y[4 * i + 3] = hi[1] * scale;
      }
      if constexpr (F32) *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(y[0], y[1], y[2], y[3]);
      else store8(out, at, false, y);
    }
  }
}

hipError_t launch_unpack8(const Unpack8Params& q, hipStream_t st) {
  if (q.num == 0) return hipSuccess;
  Unpack8Params p = q;
  const int rows = (int)(kLaunchGroups / p.num);        // (num <= 2^13: 2^10 at least)
  for (p.first_row = 0; p.first_row < p.B; p.first_row += rows) {
    const int n = p.B - p.first_row < rows ? p.B - p.first_row : rows;
    const dim3 g((uint32_t)n * p.num, p.hkv, 2), t(kUnpackThreads);
    if (p.d == 64) {
      if (p.f32) hipLaunchKernelGGL((unpack8_kernel<64, true>), g, t, 0, st, p);
      else hipLaunchKernelGGL((unpack8_kernel<64, false>), g, t, 0, st, p);
    } else {
      if (p.f32) hipLaunchKernelGGL((unpack8_kernel<128, true>), g, t, 0, st, p);
      else hipLaunchKernelGGL((unpack8_kernel<128, false>), g, t, 0, st, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cobs

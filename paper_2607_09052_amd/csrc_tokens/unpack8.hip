// cobs_unpack8: blocks of an 8-bit cache as bf16 or fp32.  A copy, bound by HBM (three times the codes' bytes for bf16).
// A thread takes 16 codes of a token's head, 16 bytes in, 32 or 64 out; a workgroup a block's keys or values.
// Measured (d 128, bf16): 4 rows of 32741 tokens of 8 heads, 805 MB, in 154 us, 5.2 TB/s (a large copy: 5.0); the newest block of 32
// rows 4.5 us.
#include "tokens_device.h"

namespace cobs {

constexpr int kUnpackThreads = 256;

// grid: (block and row, KV head, keys or values)
template <int D, bool F32>
__global__ __launch_bounds__(kUnpackThreads) void unpack8_kernel(Unpack8Params p) {
  constexpr int TPR = D / 16;
  const int b = blockIdx.x / p.num, which = blockIdx.x % p.num, h = blockIdx.y, value = blockIdx.z;
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
  for (int x = threadIdx.x; x < rows * TPR; x += kUnpackThreads) {
    const int t = x / TPR, e = 16 * (x % TPR);
    const uint4 w = *reinterpret_cast<const uint4*>(codes + t * rs + e);
    const uint32_t c[4] = {w.x, w.y, w.z, w.w};
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
      y[4 * i] = lo[0] * scale;
      y[4 * i + 1] = lo[1] * scale;
      y[4 * i + 2] = hi[0] * scale;
      y[4 * i + 3] = hi[1] * scale;
    }
    store8(out, to + t * ws + e, F32, y);
    store8(out, to + t * ws + e + 8, F32, y + 8);
  }
}

hipError_t launch_unpack8(const Unpack8Params& p, hipStream_t st) {
  if (p.num == 0) return hipSuccess;
  const int64_t grid = (int64_t)p.B * p.num;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 g((uint32_t)grid, p.hkv, 2), t(kUnpackThreads);
  if (p.d == 64) {
    if (p.f32) hipLaunchKernelGGL((unpack8_kernel<64, true>), g, t, 0, st, p);
    else hipLaunchKernelGGL((unpack8_kernel<64, false>), g, t, 0, st, p);
  } else {
    if (p.f32) hipLaunchKernelGGL((unpack8_kernel<128, true>), g, t, 0, st, p);
    else hipLaunchKernelGGL((unpack8_kernel<128, false>), g, t, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace cobs

// cobs_attention_weights: its launches, and the kernels over bf16 caches.
#include "weights_kernel.h"

namespace cobs {

// Earlier weights (or zeros) of every cached token of a row, before the attended ones get their sums:
// four positions a thread (rows of max_seq_len fp32 are 16-byte aligned where the tensors are).
template <bool VEC>
__global__ __launch_bounds__(256) void weights_copy_kernel(WeightsParams p) {
  const AttendParams& a = p.a;
  const int b = blockIdx.z, h = blockIdx.y;
  const int C = clamp_len(a.seq_lens[b], a.tmax);
  const int E = C + (a.mask ? clamp_len(a.draft_lens[b], min(a.N, a.tmax - C)) : 0);
  const int64_t row = ((int64_t)b * a.hkv + h) * a.tmax;
  const int t = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (VEC && t + 4 <= E) {
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (p.prev) v = *reinterpret_cast<const float4*>(p.prev + row + t);
    *reinterpret_cast<float4*>(p.weights + row + t) = v;
  } else {
    for (int k = 0; k < 4; ++k)
      if (t + k < E) p.weights[row + t + k] = p.prev ? p.prev[row + t + k] : 0.0f;
  }
}

hipError_t launch_weights_f32(const WeightsParams& p, hipStream_t st);

hipError_t launch_weights(const WeightsParams& p, hipStream_t st) {
  if (p.a.sparse && p.prev != p.weights) {
    const dim3 grid((p.a.tmax + 1023) / 1024, p.a.hkv, p.a.B);
    const bool vec = ((reinterpret_cast<uintptr_t>(p.prev) | reinterpret_cast<uintptr_t>(p.weights)) & 15) == 0;
    if (vec) hipLaunchKernelGGL(weights_copy_kernel<true>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(weights_copy_kernel<false>, grid, dim3(256), 0, st, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (p.a.kv_f32) return launch_weights_f32(p, st);
  return p.a.d == 64 ? launch_weights_kernels<64, false>(p, st) : launch_weights_kernels<128, false>(p, st);
}

}  // namespace cobs

// Attention weights that cached tokens receive (cobs_attention_weights).  The
// work goes by position: a wave owns 32 positions, finds which of them are
// attended to, sums exp(c q.k - lse) over the queries and heads of its KV head
// and writes each position once, so no sum depends on an order of arrival.
#include "cache_device.h"

namespace cobs {

template <int D>
__global__ __launch_bounds__(256) void weights_plain_kernel(WeightsParams p) {
  __shared__ int red[4];
  const AttendParams& a = p.a;
  const int h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const Attended x = attended<256>(a, b, h, red);
  const int t0 = (blockIdx.x * 4 + wave) * kFrame, t = t0 + (lane & 31), half = lane >> 5;
  if (t0 >= x.E) return;
  bool in = t < x.E;
  if (a.sparse && t < x.ws) {
    const int blk = t >> a.lsh, at = sel_lower_bound(x, blk);
    in = at < x.nsel && x.sel[at] == blk;
  }
  const int64_t base = kv_offset(a.kv, b, h, t0);
  const int64_t rs = a.kv.table ? a.kv.d : a.kv.st;
  if (base < 0) in = false;
  float sum = 0.0f;
  if (in)
    for (int i = 0; i < x.nq; ++i) {
      if (t >= x.C && !((a.mask[(int64_t)b * a.N + i] >> (t - x.C)) & 1)) continue;
      for (int g = 0; g < a.G; ++g) {
        const int64_t row = ((int64_t)b * a.N + i) * a.hq + h * a.G + g;
        float sc = 0.0f;
        for (int e = half * (D / 2); e < (half + 1) * (D / 2); ++e)
          sc += load_elem(a.q, row * D + e, !a.io_bf16) * a.c * load_elem(a.kv.k, base + (t - t0) * rs + e, a.kv_f32);
        sc += __shfl_xor(sc, 32, 64);      // lane l ^ 32 holds the same token, so takes the same branches
        const float z = p.lse[row];
        if (fabsf(z) != INFINITY) sum += __expf(sc - z);
      }
    }
  if (half == 0 && t < x.E) {
    const int64_t at = ((int64_t)b * a.hkv + h) * a.tmax + t;
    p.weights[at] = (p.prev ? p.prev[at] : 0.0f) + sum;
  }
}

hipError_t launch_weights(const WeightsParams& p, hipStream_t st) {
  const dim3 grid((p.a.tmax + 127) / 128, p.a.hkv, p.a.B);
  if (p.a.d == 128) hipLaunchKernelGGL(weights_plain_kernel<128>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(weights_plain_kernel<64>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace cobs

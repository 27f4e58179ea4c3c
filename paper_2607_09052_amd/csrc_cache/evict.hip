// Which tokens a cache keeps (cobs_evict).  One workgroup per (batch row, KV
// head): the (keep - sinks - recent)-th largest weight between the first and the
// last tokens by four passes of a radix search over order-preserving 32-bit
// keys, then one pass that writes the kept positions in order.
#include "cache_device.h"

namespace cobs {

constexpr int kEvictThreads = 1024;

// Larger weight, larger key; NaN with -inf.  -0 and 0 are one weight.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) w = -INFINITY;
  return order_key(w + 0.0f);
}

__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictParams p) {
  __shared__ int hist[256];
  __shared__ int wsum[2][16];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int T = clamp_len(p.seq_lens[b], p.tmax);
  const float* w = p.weights + ((int64_t)b * p.hkv + h) * p.tmax;
  int32_t* out = p.kept + ((int64_t)b * p.hkv + h) * p.keep;
  if (p.new_lens && h == 0 && tid == 0) p.new_lens[b] = min(T, p.keep);
  if (T <= p.keep) {
    for (int j = tid; j < p.keep; j += kEvictThreads) out[j] = j < T ? j : -1;
    return;
  }
  const int lo = p.sinks, hi = T - p.recent;     // the tokens to choose from; T > keep >= sinks + recent
  uint32_t prefix = 0;
  int need = p.keep - p.sinks - p.recent;        // < hi - lo
  if (need > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kEvictThreads) {
        const uint32_t k = weight_key(w[t]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = need, d = 255;
        while (hist[d] < left) left -= hist[d--];
        s_prefix = prefix | ((uint32_t)d << shift);
        s_need = left;
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
    }
  // keep every key above `prefix` and the first `need` equal to it
  int done = 0, equal = 0;                       // kept tokens and equal keys before this round
  for (int t0 = 0; t0 < T; t0 += kEvictThreads) {
    const int t = t0 + tid;
    const bool mid = t >= lo && t < hi && p.keep > p.sinks + p.recent;
    const uint32_t k = mid ? weight_key(w[t]) : 0;
    const bool eq = mid && k == prefix;
    const unsigned long long eqs = __ballot(eq), below = ((1ull << lane) - 1);
    if (lane == 0) wsum[0][wave] = __popcll(eqs);
    __syncthreads();
    int rank = equal + __popcll(eqs & below), all = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) rank += wsum[0][i];
      all += wsum[0][i];
    }
    equal += all;
    const bool take = t < T && (t < lo || t >= hi || (mid && (k > prefix || (eq && rank < need))));
    const unsigned long long tk = __ballot(take);
    if (lane == 0) wsum[1][wave] = __popcll(tk);
    __syncthreads();
    int at = done + __popcll(tk & below);
    all = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) at += wsum[1][i];
      all += wsum[1][i];
    }
    done += all;
    if (take) out[at] = t;
    __syncthreads();
  }
}

hipError_t launch_evict(const EvictParams& p, hipStream_t st) {
  hipLaunchKernelGGL(evict_kernel, dim3(p.hkv, p.B), dim3(kEvictThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace cobs

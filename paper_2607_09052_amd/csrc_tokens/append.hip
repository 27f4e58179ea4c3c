// cobs_rotate and cobs_append (append_body.h).
#include "append_body.h"

namespace cobs {

template <int D, bool CACHE>
__global__ __launch_bounds__(kHeadThreads) void append_kernel(AppendParams p) {
  __shared__ HeadsShared s;
  const int wg = p.first_wg + blockIdx.x;
  if (wg == 0) write_lens(p.t);
  heads_body<D, CACHE>(p.t, &p.kv, p.kv_f32, wg, p.per_wg, p.slots, p.slot_groups, s);
}

hipError_t launch_append(const AppendParams& q, hipStream_t st) {
  AppendParams p = q;
  const bool cache = p.t.hkv > 0;
  const int64_t tokens = (int64_t)p.t.B * p.t.N;
  plan_heads(tokens, p.t.hq + 2 * p.t.hkv, p.t.d, &p.per_wg, &p.slots, &p.slot_groups);
  const int64_t grid = (tokens + p.per_wg - 1) / p.per_wg * p.slot_groups;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 t(kHeadThreads);
  for (int64_t first = 0; first < grid; first += kLaunchGroups) {
    const dim3 g((uint32_t)(grid - first < kLaunchGroups ? grid - first : kLaunchGroups));
    p.first_wg = (int)first;
    if (p.t.d == 64) {
      if (cache) hipLaunchKernelGGL((append_kernel<64, true>), g, t, 0, st, p);
      else hipLaunchKernelGGL((append_kernel<64, false>), g, t, 0, st, p);
    } else {
      if (cache) hipLaunchKernelGGL((append_kernel<128, true>), g, t, 0, st, p);
      else hipLaunchKernelGGL((append_kernel<128, false>), g, t, 0, st, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cobs

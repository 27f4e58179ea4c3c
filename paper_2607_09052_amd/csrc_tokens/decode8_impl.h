// Launches of decode8_kernel for one head dimension.
#pragma once

#include "decode8_kernel.h"

namespace cobs {

template <int D, int PARTS>
hipError_t launch_decode8_kernels(const Decode8Params& p, int tiles, int grid, hipStream_t st) {
  const dim3 g(grid), t(kTreeThreads);
  // (two tiles a wave with three parts of 128-element queries spill)
  constexpr int QT = D == 128 && PARTS == 3 ? 1 : 2;
  if (tiles == 1) hipLaunchKernelGGL((decode8_kernel<D, PARTS, 1>), g, t, 0, st, p);
  else if (tiles == 4) hipLaunchKernelGGL((decode8_many_kernel<D, PARTS, 1>), g, t, 0, st, p);
  else if constexpr (QT == 2) {
    if (tiles == 2) hipLaunchKernelGGL((decode8_kernel<D, PARTS, 2>), g, t, 0, st, p);
    else hipLaunchKernelGGL((decode8_many_kernel<D, PARTS, 2>), g, t, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace cobs

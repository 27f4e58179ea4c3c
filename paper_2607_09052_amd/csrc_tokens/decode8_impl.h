// Launches of decode8_kernel for one head dimension.
#pragma once

#include "decode8_kernel.h"

namespace cobs {

template <int D, int PARTS>
hipError_t launch_decode8_kernels(const Decode8Params& p, int rows, int grid, hipStream_t st) {
  const dim3 g(grid), t(kTreeThreads);
  if (rows == 16) hipLaunchKernelGGL((decode8_kernel<D, PARTS, 16>), g, t, 0, st, p);
  else hipLaunchKernelGGL((decode8_kernel<D, PARTS, 32>), g, t, 0, st, p);
  return hipGetLastError();
}

}  // namespace cobs

// tree_kernel and tree_wide_kernel for 128-element heads over bf16 caches.
#include "tree_wide.h"

namespace cobs {
hipError_t launch_tree_bf16_d128(const TreeParams& p, int wq, int grid, hipStream_t st) {
  if (wq == 8) {
    hipLaunchKernelGGL(tree_wide_kernel<128>, dim3(grid), dim3(kTreeThreads), 0, st, p);
    return hipGetLastError();
  }
  return launch_tree_kernels<128, false>(p, wq, grid, st);
}
}  // namespace cobs

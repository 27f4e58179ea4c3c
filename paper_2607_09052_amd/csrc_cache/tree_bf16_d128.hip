// tree_kernel for 128-element heads over bf16 caches.
#include "tree_kernel.h"

namespace cobs {
hipError_t launch_tree_bf16_d128(const TreeParams& p, int wq, int grid, hipStream_t st) {
  return launch_tree_kernels<128, false>(p, wq, grid, st);
}
}  // namespace cobs

// tree_kernel for 64-element heads over bf16 caches.
#include "tree_kernel.h"

namespace cobs {
hipError_t launch_tree_bf16_d64(const TreeParams& p, int wq, int grid, hipStream_t st) {
  return launch_tree_kernels<64, false>(p, wq, grid, st);
}
}  // namespace cobs

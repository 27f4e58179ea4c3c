// tree_kernel for 64-element heads over fp32 caches.
#include "tree_kernel.h"

namespace cobs {
hipError_t launch_tree_f32_d64(const TreeParams& p, int wq, int grid, hipStream_t st) {
  return launch_tree_kernels<64, true>(p, wq, grid, st);
}
}  // namespace cobs

// decode8_kernel for bf16 queries of 64-element heads.
#include "decode8_impl.h"

namespace cobs {
hipError_t launch_decode8_bf16_d64(const Decode8Params& p, int rows, int grid, hipStream_t st) {
  return launch_decode8_kernels<64, 1>(p, rows, grid, st);
}
}  // namespace cobs

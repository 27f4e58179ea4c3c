// cobs_attention_weights over fp32 caches.
#include "weights_kernel.h"

namespace cobs {

hipError_t launch_weights_f32(const WeightsParams& p, hipStream_t st) {
  return p.a.d == 64 ? launch_weights_kernels<64, true>(p, st) : launch_weights_kernels<128, true>(p, st);
}

}  // namespace cobs

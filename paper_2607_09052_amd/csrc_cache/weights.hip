// cobs_attention_weights over bf16 caches, and the choice between the types.
#include "weights_kernel.h"

namespace cobs {

hipError_t launch_weights_f32(const WeightsParams& p, hipStream_t st);

hipError_t launch_weights(const WeightsParams& p, hipStream_t st) {
  if (p.a.kv_f32) return launch_weights_f32(p, st);
  return p.a.d == 64 ? launch_weights_kernels<64, false>(p, st) : launch_weights_kernels<128, false>(p, st);
}

}  // namespace cobs

// The gradients of q, k, g and beta of the gated delta rule for key heads of 128 (delta_grad.h).
#include "delta_grad.h"

namespace vla {
hipError_t launch_delta_grad_128(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream) {
  return delta::launch_grad_dk<128>(a, d_v, io_dtype, stream);
}
}  // namespace vla

// The chain of the state's gradient of the gated delta rule for key heads of 16 (delta_reverse.h).
#include "delta_reverse.h"

namespace vla {
hipError_t launch_delta_reverse_16(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream) {
  return delta::launch_reverse_dk<16>(a, d_v, io_dtype, map, stream);
}
}  // namespace vla

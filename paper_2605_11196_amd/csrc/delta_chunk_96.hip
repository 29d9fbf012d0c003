// The block form of the gated delta rule for key heads of 96 (delta_chunk.h).
#include "delta_chunk.h"

namespace vla {
hipError_t launch_delta_chunk_96(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream) {
  return delta::launch_chunk_dk<96>(a, d_v, io_dtype, map, stream);
}
}  // namespace vla

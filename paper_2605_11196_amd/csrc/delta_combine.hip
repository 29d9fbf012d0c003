// The states between time segments of the gated delta rule.  A segment's map is affine in the state that it starts from, row by row:
// S_end = S_start X + Y (delta_chunk.h forms X and Y of every segment at once), so
//   seg_S[0] = S0;  seg_S[s + 1] = seg_S[s] X_s + Y_s,
// and in the backward pass from the last segment to the first.
//
// A workgroup takes 16 rows of S of one head, which need nothing of the others, and goes through the segments; a wave forms 16
// columns of the product on the FP32 matrix instruction, from the rows that the waves leave in LDS.  The product is transposed: a
// result tile (columns of S along its rows) is the right operand of the next product as it stands.  X of the next segment is
// requested before the present product.  Bound by the latency of a step, about 2 us at d_k = 128 (64 matrix
// instructions on each SIMD, the exchange through LDS and a barrier): 16 heads of 128 x 128, 15 steps 32 us; 64 heads, 3 steps 17.5 us (25.6
// with the workgroups of a head on different L2 caches).
#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace {

template <int DK>
__global__ void __launch_bounds__(4 * DK) delta_combine_kernel(DeltaArgs a, int d_v, int backward) {
  constexpr int KT = DK / 16;
  __shared__ f4 state[2][KT][64];
  // the workgroups of a head on one of the eight L2 caches, which take workgroups in turn: they all read X
  const int tiles = d_v / 16, turns = a.B * a.H_v / 8 * 8 * tiles, at = blockIdx.x;
  const int head = at < turns ? at / (8 * tiles) * 8 + at % 8 : at / tiles, row = 16 * (at < turns ? at / 8 % tiles : at % tiles);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, c = lane % 16, g = lane / 16;
  const size_t map = static_cast<size_t>(d_v + DK) * DK, one = static_cast<size_t>(d_v) * DK;
  const float* maps = a.seg_map + static_cast<size_t>(head) * a.n_slots * map;
  float* out = a.seg_S + static_cast<size_t>(head) * a.n_slots * one + static_cast<size_t>(row + c) * DK + 16 * wave + 4 * g;
  const int first = a.first_done ? 1 : 0;     // the state of this one is given
  const auto place = [&](int s) { return backward ? a.n_seg - 1 - s : s - (a.n_seg - a.n_slots); };
  f4 own = f4{0.0f, 0.0f, 0.0f, 0.0f};
  if (first > 0) own = *reinterpret_cast<const f4*>(out + place(1) * one);
  else if (a.S0 != nullptr) own = *reinterpret_cast<const f4*>(a.S0 + head * one + static_cast<size_t>(row + c) * DK + 16 * wave + 4 * g);
  float x[KT][4];
  f4 y;
  auto request = [&](int s) {
    const float* m = maps + s * map;
    y = *reinterpret_cast<const f4*>(m + static_cast<size_t>(row + c) * DK + 16 * wave + 4 * g);
    const float* X = m + one + 16 * wave + c;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int r = 0; r < 4; ++r) x[kt][r] = X[(16 * kt + 4 * g + r) * DK];
    }
  };
  if (first == 0) *reinterpret_cast<f4*>(out + place(0) * one) = own;
  request(place(first));
  for (int s = first; s + 1 < a.n_seg; ++s) {
    state[s & 1][wave][lane] = own;
    __syncthreads();
    f4 acc[2] = {y, f4{0.0f, 0.0f, 0.0f, 0.0f}};
    float now[KT][4];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int r = 0; r < 4; ++r) now[kt][r] = x[kt][r];
    }
    request(place(min(s + 1, a.n_seg - 2)));
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const f4 b = state[s & 1][kt][lane];
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[r & 1] = mfma16(now[kt][r], b[r], acc[r & 1]);
    }
    own = acc[0] + acc[1];
    *reinterpret_cast<f4*>(out + place(s + 1) * one) = own;
  }
}

template <int DK>
hipError_t launch(const DeltaArgs& a, int d_v, int backward, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args, &d_v, &backward};
  return hipLaunchKernel(reinterpret_cast<const void*>(&delta_combine_kernel<DK>), dim3(a.B * a.H_v * (d_v / 16)), dim3(4 * DK), params, 0, stream);
}

}  // namespace

hipError_t launch_delta_combine(const DeltaArgs& a, int d_k, int d_v, bool backward, hipStream_t stream) {
  switch (d_k) {
    case 16: return launch<16>(a, d_v, backward, stream);
    case 32: return launch<32>(a, d_v, backward, stream);
    case 64: return launch<64>(a, d_v, backward, stream);
    case 96: return launch<96>(a, d_v, backward, stream);
    case 128: return launch<128>(a, d_v, backward, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace vla

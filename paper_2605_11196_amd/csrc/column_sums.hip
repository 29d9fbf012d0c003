// Sums over workgroups of what each has given of a weight's gradient, always in the same order.
//
// Bound by memory and the latency of its loads: 64 columns a workgroup, 16 waves on their rows, eight loads of a wave under way.
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kRows = 16;

__global__ void __launch_bounds__(64 * kRows) column_sums_kernel(ColumnSums s) {
  __shared__ float part[kRows][64];
  const ColumnSum j = s.job[blockIdx.y];
  const int lane = threadIdx.x % 64, row = threadIdx.x / 64;
  if (static_cast<long long>(blockIdx.x) * 64 >= j.columns) return;
  const int c = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (c < j.columns) {
    const float* p = j.parts + c;
#pragma unroll 8
    for (int r = row; r < j.rows; r += kRows) sum += p[r * j.stride];
  }
  part[row][lane] = sum;
  __syncthreads();
  if (row != 0 || c >= j.columns) return;
  for (int r = 1; r < kRows; ++r) sum += part[r][lane];
  const size_t at = static_cast<size_t>(c) * j.step;
  if (j.bf16) static_cast<uint16_t*>(j.out)[at] = f32_to_bf16_rne(sum);
  else static_cast<float*>(j.out)[at] = sum;
}

}  // namespace

hipError_t launch_column_sums(const ColumnSums& s, hipStream_t stream) {
  int most = 0;
  for (int i = 0; i < s.n; ++i) most = most < s.job[i].columns ? s.job[i].columns : most;
  if (s.n == 0 || most == 0) return hipSuccess;
  ColumnSums args = s;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(&column_sums_kernel), dim3((most + 63) / 64, s.n), dim3(64 * kRows), params, 0, stream);
}

}  // namespace vla

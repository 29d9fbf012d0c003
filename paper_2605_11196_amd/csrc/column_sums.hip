// Sums over workgroups of what each has given of a weight's gradient, always in the same order.
//
// Bound by memory and the latency of its loads: 64 columns a workgroup at a time, 16 waves on their rows, eight loads of a wave under way.  A launch holds
// less than 2^32 work-items, which one workgroup for every 64 columns would reach at 2^28 columns (the rates' gradient of 2^22 channels with
// 64 states): kGroups of them at most go through the columns.
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kRows = 16, kGroups = 1 << 16;

__global__ void __launch_bounds__(64 * kRows) column_sums_kernel(ColumnSums s) {
  __shared__ float part[kRows][64];
  const ColumnSum j = s.job[blockIdx.y];
  const int lane = threadIdx.x % 64, row = threadIdx.x / 64;
  const long long step = 64LL * gridDim.x;
  for (long long first = 64LL * blockIdx.x; first < j.columns; first += step) {
    const long long c = first + lane;
    float sum = 0.0f;
    if (c < j.columns) {
      const float* p = j.parts + c;
#pragma unroll 8
      for (int r = row; r < j.rows; r += kRows) sum += p[r * j.stride];
    }
    part[row][lane] = sum;
    __syncthreads();
    if (row == 0 && c < j.columns) {
      for (int r = 1; r < kRows; ++r) sum += part[r][lane];
      const size_t at = static_cast<size_t>(c) * j.step;
      if (j.bf16) static_cast<uint16_t*>(j.out)[at] = f32_to_bf16_rne(sum);
      else static_cast<float*>(j.out)[at] = sum;
    }
    if (first + step < j.columns) __syncthreads();   // the parts have been read
  }
}

}  // namespace

hipError_t launch_column_sums(const ColumnSums& s, hipStream_t stream) {
  int most = 0;
  for (int i = 0; i < s.n; ++i) most = most < s.job[i].columns ? s.job[i].columns : most;
  if (s.n == 0 || most == 0) return hipSuccess;
  const long long groups = (most + 63LL) / 64;
  ColumnSums args = s;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(&column_sums_kernel), dim3(static_cast<unsigned>(groups < kGroups ? groups : kGroups), s.n), dim3(64 * kRows), params, 0, stream);
}

}  // namespace vla

// One token of the selective state space scan on a state that stays where it is.
//
// Bound by memory: the state is read and written once.  N / 4 lanes hold a channel, four states (16 bytes) a lane; the read-out is summed
// across them.  Everything a lane needs is asked for at once, and places are 32-bit numbers (64 sequences of 4096 channels, 16 states: 10.3 ->
// 8.8 us, 4.0 TB/s, of which 2 us are the launch and the first load's way).
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kThreads = 256;

template <typename IO> __device__ __forceinline__ float load1(const IO* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<uint16_t>(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ f4 four(const float* p) { return *reinterpret_cast<const f4*>(p); }
__device__ __forceinline__ f4 four(const uint16_t* p) {
  const u2 b = *reinterpret_cast<const u2*>(p);
  const f2 x = widen(b[0]), y = widen(b[1]);
  return f4{x[0], x[1], y[0], y[1]};
}
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = f32_to_bf16_rne(x); }

template <int N, typename IO>
__global__ void __launch_bounds__(kThreads) step_kernel(ScanArgs a) {
  constexpr int LANES = N / 4;
  const unsigned channel = blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;      // the call checks that their number fits
  if (channel >= static_cast<unsigned>(a.nb) * a.n) return;      // whole channels: LANES divides the workgroup
  const int s = 4 * (threadIdx.x % LANES);
  const unsigned seq = channel / a.n, c = channel - seq * a.n, g = a.G == 1 ? 0 : c / (a.n / a.G);
  const long long b = seq;
  f4* state = reinterpret_cast<f4*>(a.h_T + static_cast<size_t>(channel) * N + s);
  f4 h = *state;
  const f4 A = four(a.A + static_cast<size_t>(c) * N + s);
  const f4 Bt = four(static_cast<const IO*>(a.Bm) + b * a.B_b + g * a.B_g + s), Ct = four(static_cast<const IO*>(a.Cm) + b * a.C_b + g * a.C_g + s);
  const float u = load1(static_cast<const IO*>(a.u) + b * a.us.b + c);
  const float raw = load1(static_cast<const IO*>(a.delta) + b * a.ds.b + c) + (a.bias != nullptr ? a.bias[c] : 0.0f);
  // asked for with the rest, though only a channel's first lane needs them
  const float D = a.D != nullptr ? a.D[c] : 0.0f, z = a.z != nullptr ? load1(static_cast<const IO*>(a.z) + b * a.zs.b + c) : 0.0f;
  const float dt = a.softplus ? softplus(raw) : raw, x = dt * u;
  float y = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = fmaf(__builtin_amdgcn_exp2f(dt * (A[i] * kLog2e)), h[i], x * Bt[i]);
    y = fmaf(Ct[i], h[i], y);
  }
  *state = h;
  y = group_sum(y, LANES);
  if (s != 0) return;
  if (a.D != nullptr) y = fmaf(D, u, y);
  if (a.z != nullptr) y *= z * sigmoid(z);
  store1(static_cast<IO*>(a.y) + b * a.ys.b + c, y);
}

template <int N>
hipError_t launch(const ScanArgs& a, int io_dtype, hipStream_t stream) {
  const long long items = static_cast<long long>(a.nb) * a.n * (N / 4);
  ScanArgs args = a;
  void* params[] = {&args};
  const void* kernel = io_dtype == 1 ? reinterpret_cast<const void*>(&step_kernel<N, uint16_t>) : reinterpret_cast<const void*>(&step_kernel<N, float>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>((items + kThreads - 1) / kThreads)), dim3(kThreads), params, 0, stream);
}

}  // namespace

hipError_t launch_selective_step(const ScanArgs& a, int N, int io_dtype, hipStream_t stream) {
  switch (N) {
    case 8: return launch<8>(a, io_dtype, stream);
    case 16: return launch<16>(a, io_dtype, stream);
    case 32: return launch<32>(a, io_dtype, stream);
    case 64: return launch<64>(a, io_dtype, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace vla

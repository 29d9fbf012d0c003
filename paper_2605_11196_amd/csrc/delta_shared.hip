// dq and dk of key heads that several value heads share: the sum of the value heads' shares, in the order of the heads.  Four columns of a
// token a thread; each share is read once, bound by memory (64 heads of 128, 4096 tokens to 16 key heads: 52 us, 5.8 TB/s).
#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace {

__device__ __forceinline__ void put4(float* p, f4 x) { *reinterpret_cast<f4*>(p) = x; }
__device__ __forceinline__ void put4(uint16_t* p, f4 x) { *reinterpret_cast<u2*>(p) = u2{pack_rne(x[0], x[1]), pack_rne(x[2], x[3])}; }

template <typename IO>
__global__ void __launch_bounds__(256) delta_shared_kernel(DeltaArgs a, int d_k) {
  const int four = d_k / 4, share = a.H_v / a.H_k;
  const long long all = static_cast<long long>(a.B) * a.H_k * a.T * four;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<long long>(gridDim.x) * 256) {
    const int x = static_cast<int>(i % four) * 4;
    const long long row = i / four, head = row / a.T, t = row % a.T;       // head of the keys, over the batch
    const long long b = head / a.H_k, h = head % a.H_k;
    const size_t from = ((b * a.H_v + h * share) * a.T + t) * d_k + x, step = static_cast<size_t>(a.T) * d_k;
    f4 dq = f4{0.0f, 0.0f, 0.0f, 0.0f}, dk = dq;
    for (int s = 0; s < share; ++s) {
      dq += *reinterpret_cast<const f4*>(a.dq_part + from + s * step);
      dk += *reinterpret_cast<const f4*>(a.dk_part + from + s * step);
    }
    put4(static_cast<IO*>(a.dq) + b * a.dqs.b + h * a.dqs.h + t * a.dqs.t + x, dq);
    put4(static_cast<IO*>(a.dk) + b * a.dks.b + h * a.dks.h + t * a.dks.t + x, dk);
  }
}

}  // namespace

hipError_t launch_delta_shared(const DeltaArgs& a, int d_k, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args, &d_k};
  const long long all = static_cast<long long>(a.B) * a.H_k * a.T * (d_k / 4), groups = (all + 255) / 256;
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_shared_kernel<uint16_t>) : reinterpret_cast<const void*>(&delta_shared_kernel<float>);
  return hipLaunchKernel(fn, dim3(static_cast<unsigned>(groups < 16384 ? groups : 16384)), dim3(256), params, 0, stream);
}

}  // namespace vla

// The gated delta rule token by token (single tokens of generation, short sequences):
//
//   S' = exp(g) S;  e = beta (v - S' k);  S <- S' + e k^T;  o = scale S q = scale (S' q + e (k . q))
//
// A row of S needs nothing of the other rows, so a workgroup takes 16 rows of one head (four to a wave, 16 lanes and
// d_k / 16 columns a lane to a row) and there is no barrier.  One token reads and writes the state once, 8 d_k d_v bytes against
// 6 d_k d_v flop: memory bounds it (2048 heads of 128: 41 us, 6.5 TB/s, part of the states from the last-level cache).
#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace {

// The d_k / 16 columns of a lane: four at a time, 64 columns apart, and what is left in twos or ones, so that the 16 lanes of a
// row load from consecutive addresses.
template <int DK, typename IO>
__device__ __forceinline__ void load_cols(const IO* p, int c, float (&x)[DK / 16]) {
  constexpr int E = DK / 16;
#pragma unroll
  for (int e = 0; e + 4 <= E; e += 4) {
    if constexpr (sizeof(IO) == 2) {
      const u2 b = *reinterpret_cast<const u2*>(p + 16 * e + 4 * c);
      x[e] = __uint_as_float(b[0] << 16);
      x[e + 1] = __uint_as_float(b[0] & 0xffff0000u);
      x[e + 2] = __uint_as_float(b[1] << 16);
      x[e + 3] = __uint_as_float(b[1] & 0xffff0000u);
    } else {
      const f4 v = *reinterpret_cast<const f4*>(p + 16 * e + 4 * c);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[e + i] = v[i];
    }
  }
  if constexpr (E % 4 == 2) {
    constexpr int e = E - 2;
    x[e] = widen(p[16 * e + 2 * c]);
    x[e + 1] = widen(p[16 * e + 2 * c + 1]);
  } else if constexpr (E % 4 == 1) {
    x[E - 1] = widen(p[16 * (E - 1) + c]);
  }
}
template <int DK>
__device__ __forceinline__ void store_cols(float* p, int c, const float (&x)[DK / 16]) {
  constexpr int E = DK / 16;
#pragma unroll
  for (int e = 0; e + 4 <= E; e += 4) *reinterpret_cast<f4*>(p + 16 * e + 4 * c) = f4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  if constexpr (E % 4 == 2) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    *reinterpret_cast<f2*>(p + 16 * (E - 2) + 2 * c) = f2{x[E - 2], x[E - 1]};
  } else if constexpr (E % 4 == 1) {
    p[16 * (E - 1) + c] = x[E - 1];
  }
}
template <int E>
__device__ __forceinline__ float dot(const float (&x)[E], const float (&y)[E]) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) s = fmaf(x[e], y[e], s);
  return s;
}

template <int DK, typename IO>
__global__ void __launch_bounds__(256) delta_step_kernel(DeltaArgs a, int d_v) {
  constexpr int E = DK / 16;
  const int parts = d_v / 16, head = blockIdx.x / parts, b = head / a.H_v, h = head % a.H_v, hk = h / (a.H_v / a.H_k);
  const int c = threadIdx.x % 16, row = blockIdx.x % parts * 16 + threadIdx.x / 16;
  const size_t at = (static_cast<size_t>(head) * d_v + row) * DK;
  float S[E];
  if (a.S0 != nullptr) {
    load_cols<DK>(a.S0 + at, c, S);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) S[e] = 0.0f;
  }
  const int len = a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T;
  const IO* q = static_cast<const IO*>(a.q) + b * a.qs.b + hk * a.qs.h;
  const IO* k = static_cast<const IO*>(a.k) + b * a.ks.b + hk * a.ks.h;
  const IO* v = static_cast<const IO*>(a.v) + b * a.vs.b + h * a.vs.h + row;
  const float* g = a.g + b * a.gs.b + h * a.gs.h;
  const float* beta = a.beta + b * a.bs.b + h * a.bs.h;
  IO* o = static_cast<IO*>(a.o) + b * a.os.b + h * a.os.h + row;
  for (int t = 0; t < len; ++t) {
    float kk[E], qq[E];
    load_cols<DK>(k + t * a.ks.t, c, kk);
    load_cols<DK>(q + t * a.qs.t, c, qq);
    const float decay = expf(g[t * a.gs.t]);
    const float vt = widen(v[t * a.vs.t]);
    const float bt = beta[t * a.bs.t];
    const float kq = row_sum16(dot(kk, qq));
#pragma unroll
    for (int e = 0; e < E; ++e) S[e] *= decay;
    const float er = bt * (vt - row_sum16(dot(S, kk)));
    const float sq = row_sum16(dot(S, qq));
#pragma unroll
    for (int e = 0; e < E; ++e) S[e] = fmaf(er, kk[e], S[e]);
    if (c == 0) io_store(o + t * a.os.t, a.scale * fmaf(er, kq, sq));
  }
  for (int t = len; t < a.T; ++t) {
    if (c == 0) io_store(o + t * a.os.t, 0.0f);
  }
  if (a.S_T != nullptr) store_cols<DK>(a.S_T + at, c, S);
}

template <int DK>
hipError_t launch(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args, &d_v};
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_step_kernel<DK, uint16_t>)
                                 : reinterpret_cast<const void*>(&delta_step_kernel<DK, float>);
  return hipLaunchKernel(fn, dim3(a.B * a.H_v * (d_v / 16)), dim3(256), params, 0, stream);
}

}  // namespace

hipError_t launch_delta_step(const DeltaArgs& a, int d_k, int d_v, int io_dtype, hipStream_t stream) {
  switch (d_k) {
    case 16: return launch<16>(a, d_v, io_dtype, stream);
    case 32: return launch<32>(a, d_v, io_dtype, stream);
    case 64: return launch<64>(a, d_v, io_dtype, stream);
    case 96: return launch<96>(a, d_v, io_dtype, stream);
    case 128: return launch<128>(a, d_v, io_dtype, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace vla

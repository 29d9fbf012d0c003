// Norm of every query and key head and the position rotation, in one pass (forward and backward).
//
//   r = 1 / sqrt(sum x^2 inv_n + eps);  y = Rot_p(w x r)
//   Rot_p turns the pairs (i, i + rot/2) (or (2i, 2i+1)) of the first rot columns by the angle of position p
//   backward: z = Rot_p^T dy;  dx = r (w z - x r^2 inv_n (w z . x));  dw = sum over rows of z x r
//
// Bound by memory: each row is read once and written once (two reads in the backward pass).  d / 8 lanes hold a row (16
// for 96 columns, 12 of them at work), eight columns a lane, chosen so that a pair lies in one lane: with halves apart,
// four columns at the lane's place in each half; so no value crosses lanes but the sum of squares (DPP).  A group of lanes stays
// with one token and goes through its heads, which keeps the position, its cosines and sines and the weights on
// registers.  The sums are float32.  524288 rows of 64 in bf16 25 us (5.3 TB/s), 2.6 million rows of 128 with gradients
// 0.25 + 0.43 ms (5.3 and 4.7 TB/s).
#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4, kHeadsBack = 2;   // heads of a token that a lane group loads at once

// sum over the G lanes of a row, G a power of two up to 16
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
  if constexpr (G >= 2) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true));
  if constexpr (G >= 4) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true));
  if constexpr (G >= 8) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));
  if constexpr (G >= 16) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true));
  return x;
}

__device__ __forceinline__ f4 load4(const float* p) { return *reinterpret_cast<const f4*>(p); }
__device__ __forceinline__ f4 load4(const uint16_t* p) {
  const u2 b = *reinterpret_cast<const u2*>(p);
  return f4{__uint_as_float(b[0] << 16), __uint_as_float(b[0] & 0xffff0000u), __uint_as_float(b[1] << 16),
            __uint_as_float(b[1] & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float* p, f4 x) { *reinterpret_cast<f4*>(p) = x; }
__device__ __forceinline__ void store4(uint16_t* p, f4 x) {
  *reinterpret_cast<u2*>(p) = u2{pack_rne(x[0], x[1]), pack_rne(x[2], x[3])};
}

// What a lane keeps for its token: its columns, their weights for queries and keys, and the turn of its four pairs.
template <int D, bool INTER>
struct Lane {
  int lo, hi;
  f4 c, s;
  bool here;   // the position is in the tables

  __device__ __forceinline__ void columns(const NormArgs& a, int lane) {
    const int turning = a.rot / 8;
    if (INTER) {
      lo = 8 * lane;
      hi = lo + 4;
    } else if (lane < turning) {
      lo = 4 * lane;
      hi = lo + a.rot / 2;
    } else {
      lo = a.rot + 4 * (lane - turning);
      hi = lo + (D - a.rot) / 2;
    }
  }
  __device__ __forceinline__ void place(const NormArgs& a, int lane, int b, int t) {
    const long long p = a.positions ? a.positions[static_cast<size_t>(b) * a.T + t] : static_cast<long long>(a.offset) + t;
    here = p >= 0 && p < a.places;
    c = f4{1.0f, 1.0f, 1.0f, 1.0f};
    s = f4{0.0f, 0.0f, 0.0f, 0.0f};
    if (here && lane < a.rot / 8) {
      const size_t at = static_cast<size_t>(p) * (a.rot / 2) + 4 * lane;
      c = load4(a.cos + at);
      s = load4(a.sin + at);
    }
  }
  // (x0, x1) by the angle (its negative with back)
  template <bool BACK>
  __device__ __forceinline__ void turn(f4& x0, f4& x1) const {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float u = INTER ? (p < 2 ? x0[2 * p] : x1[2 * p - 4]) : x0[p];
      const float v = INTER ? (p < 2 ? x0[2 * p + 1] : x1[2 * p - 3]) : x1[p];
      const float sp = BACK ? -s[p] : s[p];
      const float m = u * c[p] - v * sp, n = u * sp + v * c[p];
      if (INTER) {
        if (p < 2) { x0[2 * p] = m; x0[2 * p + 1] = n; }
        else { x1[2 * p - 4] = m; x1[2 * p - 3] = n; }
      } else {
        x0[p] = m;
        x1[p] = n;
      }
    }
  }
};

__device__ __forceinline__ f4 weight4(const NormArgs& a, int which, int col) {
  if (a.w[which] == nullptr) return f4{1.0f, 1.0f, 1.0f, 1.0f};
  return a.w_bf16 ? load4(static_cast<const uint16_t*>(a.w[which]) + col) : load4(static_cast<const float*>(a.w[which]) + col);
}
__device__ __forceinline__ float dot4(f4 x, f4 y) { return fmaf(x[0], y[0], fmaf(x[1], y[1], fmaf(x[2], y[2], x[3] * y[3]))); }

template <int D> constexpr int kLanes = D == 96 ? 16 : D / 8;

template <int D, typename IO, bool INTER>
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a, int heads_each) {
  constexpr int G = kLanes<D>, TOK = kThreads / G;
  const int lane = threadIdx.x % G;
  const bool active = 8 * lane < D;
  const long long n = (static_cast<long long>(blockIdx.z) * gridDim.x + blockIdx.x) * TOK + threadIdx.x / G;
  if (n >= static_cast<long long>(a.B) * a.T) return;
  const int b = static_cast<int>(n / a.T), t = static_cast<int>(n % a.T);
  Lane<D, INTER> l;
  l.columns(a, active ? lane : 0);
  l.place(a, active ? lane : 0, b, t);
  const int first = blockIdx.y * heads_each, last = min(first + heads_each, a.H[0] + a.H[1]);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int h0 = which == 0 ? first : max(first, a.H[0]) - a.H[0];
    const int h1 = which == 0 ? min(last, a.H[0]) : last - a.H[0];
    if (h0 >= h1) continue;
    const IO* x = static_cast<const IO*>(a.x[which]) + b * a.xs[which].b + t * a.xs[which].t;
    IO* y = static_cast<IO*>(a.y[which]) + b * a.ys[which].b + t * a.ys[which].t;
    const f4 w0 = weight4(a, which, l.lo), w1 = weight4(a, which, l.hi);
    // several heads' loads are under way at once; past the last head the last one is loaded again and not stored
    for (int h = h0; h < h1; h += kHeads) {
      f4 x0[kHeads], x1[kHeads];
#pragma unroll
      for (int j = 0; j < kHeads; ++j) {
        const IO* row = x + min(h + j, h1 - 1) * a.xs[which].h;
        x0[j] = load4(row + l.lo);
        x1[j] = load4(row + l.hi);
      }
#pragma unroll
      for (int j = 0; j < kHeads; ++j) {
        const float own = active ? dot4(x0[j], x0[j]) + dot4(x1[j], x1[j]) : 0.0f;
        const float r = l.here ? rsqrtf(fmaf(lanes_sum<G>(own), a.inv_n, a.eps)) : __uint_as_float(0x7fc00000u);
        x0[j] *= w0 * r;
        x1[j] *= w1 * r;
        l.template turn<false>(x0[j], x1[j]);
        if (active && h + j < h1) {
          store4(y + (h + j) * a.ys[which].h + l.lo, x0[j]);
          store4(y + (h + j) * a.ys[which].h + l.hi, x1[j]);
        }
      }
    }
  }
}

// A workgroup goes through tiles of tokens and adds up its own part of dw on registers; the parts are summed in the order of
// the workgroups by dw_kernel, so that the result does not depend on timing.
template <int D, typename IO, bool INTER>
__global__ void __launch_bounds__(kThreads) norm_backward_kernel(NormArgs a, int tiles) {
  constexpr int G = kLanes<D>, TOK = kThreads / G;
  __shared__ float part[2][TOK][D];
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  const bool active = 8 * lane < D;
  const long long total = static_cast<long long>(a.B) * a.T;
  Lane<D, INTER> l;
  l.columns(a, active ? lane : 0);
  f4 dw0[2] = {}, dw1[2] = {};
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const long long n = static_cast<long long>(tile) * TOK + group;
    if (n >= total) continue;
    const int b = static_cast<int>(n / a.T), t = static_cast<int>(n % a.T);
    l.place(a, active ? lane : 0, b, t);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (a.H[which] == 0) continue;
      const IO* x = static_cast<const IO*>(a.x[which]) + b * a.xs[which].b + t * a.xs[which].t;
      const IO* dy = static_cast<const IO*>(a.dy[which]) + b * a.ys[which].b + t * a.ys[which].t;
      IO* dx = static_cast<IO*>(a.dx[which]) + b * a.dxs[which].b + t * a.dxs[which].t;
      const f4 w0 = weight4(a, which, l.lo), w1 = weight4(a, which, l.hi);
      for (int h = 0; h < a.H[which]; h += kHeadsBack) {
        f4 x0[kHeadsBack], x1[kHeadsBack], z0[kHeadsBack], z1[kHeadsBack];
#pragma unroll
        for (int j = 0; j < kHeadsBack; ++j) {
          const int at = min(h + j, a.H[which] - 1);
          x0[j] = load4(x + at * a.xs[which].h + l.lo);
          x1[j] = load4(x + at * a.xs[which].h + l.hi);
          z0[j] = load4(dy + at * a.ys[which].h + l.lo);
          z1[j] = load4(dy + at * a.ys[which].h + l.hi);
        }
#pragma unroll
        for (int j = 0; j < kHeadsBack; ++j) {
          l.template turn<true>(z0[j], z1[j]);
          const float sq = active ? dot4(x0[j], x0[j]) + dot4(x1[j], x1[j]) : 0.0f;
          const float along = active ? dot4(x0[j], w0 * z0[j]) + dot4(x1[j], w1 * z1[j]) : 0.0f;
          const float r = l.here ? rsqrtf(fmaf(lanes_sum<G>(sq), a.inv_n, a.eps)) : __uint_as_float(0x7fc00000u);
          const float f = lanes_sum<G>(along) * r * r * a.inv_n;
          if (h + j >= a.H[which]) continue;
          if (active) {
            store4(dx + (h + j) * a.dxs[which].h + l.lo, (w0 * z0[j] - x0[j] * f) * r);
            store4(dx + (h + j) * a.dxs[which].h + l.hi, (w1 * z1[j] - x1[j] * f) * r);
          }
          dw0[which] += z0[j] * (x0[j] * r);
          dw1[which] += z1[j] * (x1[j] * r);
        }
      }
    }
  }
  if (a.dw_part == nullptr) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (active) {
      store4(&part[which][group][l.lo], dw0[which]);
      store4(&part[which][group][l.hi], dw1[which]);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float s = 0.0f;
    for (int j = 0; j < TOK; ++j) s += part[i / D][j][i % D];
    a.dw_part[static_cast<size_t>(blockIdx.x) * 2 * D + i] = s;
  }
}

// dw[c] = sum of the workgroups' parts; 16 columns a workgroup, 16 threads on each
template <int D>
__global__ void __launch_bounds__(kThreads) dw_kernel(NormArgs a, int parts) {
  __shared__ float sums[16][17];
  const int col = blockIdx.x * 16 + threadIdx.x % 16, row = threadIdx.x / 16;
  float s = 0.0f;
#pragma unroll 4
  for (int p = row; p < parts; p += 16) s += a.dw_part[static_cast<size_t>(p) * 2 * D + col];
  sums[threadIdx.x % 16][row] = s;
  __syncthreads();
  if (row == 0) {
    float all = 0.0f;
    for (int j = 0; j < 16; ++j) all += sums[threadIdx.x][j];
    void* dw = a.dw[col / D];
    if (dw != nullptr && a.w_bf16) io_store(static_cast<uint16_t*>(dw) + col % D, all);
    else if (dw != nullptr) static_cast<float*>(dw)[col % D] = all;
  }
}

template <int D, typename IO, bool INTER>
hipError_t launch(const NormArgs& a, bool backward, hipStream_t stream) {
  constexpr int TOK = kThreads / kLanes<D>;
  const long long tokens = static_cast<long long>(a.B) * a.T;
  const int tiles = static_cast<int>((tokens + TOK - 1) / TOK);
  NormArgs args = a;
  if (!backward) {
    // Few tokens: the heads are shared out over workgroups until there are about four for each compute unit.
    const int heads = a.H[0] + a.H[1];
    int split = tiles >= 1024 ? 1 : (1024 + tiles - 1) / tiles;
    if (split > heads) split = heads;
    int each = (heads + split - 1) / split;
    split = (heads + each - 1) / each;
    void* params[] = {&args, &each};
    // a dimension of a launch holds less than 2^32 work-items, and the runtime does not check it
    constexpr int kMost = 1 << 23;
    const dim3 grid(tiles < kMost ? tiles : kMost, split, (tiles + kMost - 1) / kMost);
    return hipLaunchKernel(reinterpret_cast<const void*>(&norm_kernel<D, IO, INTER>), grid, dim3(kThreads), params, 0, stream);
  }
  int parts = tiles < kNormPartials ? tiles : kNormPartials, n_tiles = tiles;
  void* params[] = {&args, &n_tiles};
  hipError_t err = hipSuccess;
  if (tiles > 0) err = hipLaunchKernel(reinterpret_cast<const void*>(&norm_backward_kernel<D, IO, INTER>), dim3(parts), dim3(kThreads), params, 0, stream);
  if (err != hipSuccess || a.dw_part == nullptr) return err;
  void* sum_params[] = {&args, &parts};
  return hipLaunchKernel(reinterpret_cast<const void*>(&dw_kernel<D>), dim3(2 * D / 16), dim3(kThreads), sum_params, 0, stream);
}

template <int D>
hipError_t launch_d(const NormArgs& a, int io_dtype, bool interleaved, bool backward, hipStream_t stream) {
  if (io_dtype == 1) {
    return interleaved ? launch<D, uint16_t, true>(a, backward, stream) : launch<D, uint16_t, false>(a, backward, stream);
  }
  return interleaved ? launch<D, float, true>(a, backward, stream) : launch<D, float, false>(a, backward, stream);
}
hipError_t launch_any(const NormArgs& a, int d, int io_dtype, bool interleaved, bool backward, hipStream_t stream) {
  switch (d) {
    case 16: return launch_d<16>(a, io_dtype, interleaved, backward, stream);
    case 32: return launch_d<32>(a, io_dtype, interleaved, backward, stream);
    case 64: return launch_d<64>(a, io_dtype, interleaved, backward, stream);
    case 96: return launch_d<96>(a, io_dtype, interleaved, backward, stream);
    case 128: return launch_d<128>(a, io_dtype, interleaved, backward, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const NormArgs& a, int d, int io_dtype, bool interleaved, hipStream_t stream) {
  return launch_any(a, d, io_dtype, interleaved, false, stream);
}
hipError_t launch_qk_norm_rope_backward(const NormArgs& a, int d, int io_dtype, bool interleaved, hipStream_t stream) {
  return launch_any(a, d, io_dtype, interleaved, true, stream);
}

}  // namespace vla

// Device helpers of the operators on rows of channels: loads, stores, activations, sums across lanes.
#pragma once

#include "mixer_common.h"
#include "vla_mfma_util.h"

namespace vla {

typedef float f2 __attribute__((ext_vector_type(2)));

// V values of 16 bytes (bf16: 8, float32: 4), and pairs
template <typename IO> constexpr int kPiece = 16 / sizeof(IO);

__device__ __forceinline__ f2 widen(uint32_t b) { return f2{__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)}; }

// 16 bytes as they lie in memory, and their values
template <typename IO> struct Piece;
template <> struct Piece<float> {
  f4 raw;
  __device__ __forceinline__ float operator[](int i) const { return raw[i]; }
};
template <> struct Piece<uint16_t> {
  u4 raw;
  __device__ __forceinline__ float operator[](int i) const {
    return i & 1 ? __uint_as_float(raw[i / 2] & 0xffff0000u) : __uint_as_float(raw[i / 2] << 16);
  }
};
template <typename IO> __device__ __forceinline__ Piece<IO> load_piece(const IO* p) { return *reinterpret_cast<const Piece<IO>*>(p); }
template <int V> __device__ __forceinline__ void store_piece(float* p, const float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; i += 4) *reinterpret_cast<f4*>(p + i) = f4{x[i], x[i + 1], x[i + 2], x[i + 3]};
}
template <int V> __device__ __forceinline__ void store_piece(uint16_t* p, const float (&x)[V]) {
  static_assert(V % 4 == 0, "whole pieces");
#pragma unroll
  for (int i = 0; i < V; i += 4) *reinterpret_cast<u2*>(p + i) = u2{pack_rne(x[i], x[i + 1]), pack_rne(x[i + 2], x[i + 3])};
}

// Tokens of a sequence.
__device__ __forceinline__ int length_of(const int* lengths, int b, int T) { return lengths == nullptr ? T : min(max(lengths[b], 0), T); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

// log(1 + exp(x)) = max(x, 0) + log1p(w), w = exp(-|x|).  With u = 1 + w rounded and c = w - (u - 1), which is exact, log1p(w) = log(u) + log(1 + c / u);
// c is at most half a step of u, so that c in the place of the second term is off by c w or less: 2^-24 of the result.  The exponential's argument, rounded to
// float32, adds |x| half steps where x is negative and the result about w.
__device__ __forceinline__ float softplus(float x) {
  const float w = __builtin_amdgcn_exp2f(-kLog2e * fabsf(x)), u = 1.0f + w, c = w - (u - 1.0f);
  return fmaxf(x, 0.0f) + fmaf(__builtin_amdgcn_logf(u), kLn2, c);
}

__device__ __forceinline__ float swap32_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap16_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int CTRL> __device__ __forceinline__ float dpp_sum(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Sum over aligned groups of `lanes` lanes (a power of two up to 64, the same in the whole wave), in every one of them.
__device__ __forceinline__ float group_sum(float x, int lanes) {
  if (lanes >= 2) x = dpp_sum<0xB1>(x);
  if (lanes >= 4) x = dpp_sum<0x4E>(x);
  if (lanes >= 8) x = dpp_sum<0x141>(x);
  if (lanes >= 16) x = dpp_sum<0x140>(x);
  if (lanes >= 32) x = swap16_sum(x);
  if (lanes >= 64) x = swap32_sum(x);
  return x;
}

}  // namespace vla

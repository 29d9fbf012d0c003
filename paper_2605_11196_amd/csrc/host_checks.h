// What the host sides of the operators check alike: buffers of a call, alignment, the size of a launch.
#pragma once

#include "../../include/vla.h"

#include "layer_common.h"

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A caller's buffer as the byte range that its strides reach; `written` marks what the kernels store to.
struct Range {
  const void* p;
  size_t bytes;
  bool written;
};
inline bool overlap(const Range& a, const Range& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}
// No written buffer may overlap another buffer of the call, by the range of addresses that its strides span: slices of one buffer are refused
// also where their rows alternate.  `same` is the one pair that may be the same buffer.
inline bool disjoint(const Range* r, int n, const void* same0, const void* same1) {
  for (int i = 0; i < n; ++i) {
    if (!r[i].written) continue;
    for (int j = 0; j < n; ++j) {
      if (j == i || (r[j].written && j < i) || !overlap(r[i], r[j])) continue;
      const bool allowed = same0 != nullptr && r[i].p == r[j].p && r[i].bytes == r[j].bytes && (r[i].p == same0 || r[i].p == same1) && same0 == same1;
      if (!allowed) return false;
    }
  }
  return true;
}

// The strides of a call, the contiguous ones where none are given.  False where one is negative or not a whole number of
// 16-byte pieces.  (Whether rows lie in each other: rows_apart, tokens_apart.)
inline bool rows_of(const vla_strides& s, long long H, long long T, long long d, int per16, vla::Rows* out) {
  *out = vla::Rows{s.b, s.h, s.t};
  if (s.b == 0 && s.h == 0 && s.t == 0) *out = vla::Rows{H * T * d, T * d, d};
  if (T == 1) out->t = d;   // the step to a token that is not there: the kernels' bounds need it to be one
  return out->b >= 0 && out->h >= 0 && out->t >= 0 && out->b % per16 == 0 && out->h % per16 == 0 && out->t % per16 == 0;
}
inline size_t reach(const vla::Rows& r, long long B, long long H, long long T, long long d, size_t es) {
  if (B == 0 || H == 0 || T == 0) return 0;
  return (static_cast<size_t>(B - 1) * r.b + static_cast<size_t>(H - 1) * r.h + static_cast<size_t>(T - 1) * r.t + d) * es;
}

// whether rows of d elements at these strides are all apart: sorted by stride, each step clears what the smaller ones span
inline bool rows_apart(const vla::Rows& r, long long B, long long H, long long T, long long d) {
  long long s[3] = {r.b, r.h, r.t}, n[3] = {B, H, T};
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j) {
      if (s[j] < s[i]) {
        long long x = s[i]; s[i] = s[j]; s[j] = x;
        x = n[i]; n[i] = n[j]; n[j] = x;
      }
    }
  }
  if (B == 0 || H == 0 || T == 0) return true;
  long long span = d;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < span) return false;
    span += s[i] * (n[i] - 1);
  }
  return true;
}

// the tokens of a read tensor do not overlap either
inline bool tokens_apart(const vla::Rows& r, long long T, long long d) { return T <= 1 || r.t >= d; }

// A launch holds less than 2^32 work-items; the runtime wraps a larger grid without an error.
constexpr long long kMostItems = 0xffffffffLL;
inline bool fits_launch(long long groups, long long threads) { return groups <= kMostItems / threads; }

inline int launched(hipError_t err) {
  if (err == hipSuccess) return VLA_OK;
  fprintf(stderr, "libvla: kernel launch failed: %s (%d)\n", hipGetErrorString(err), static_cast<int>(err));
  return VLA_ERR_HIP;
}

}  // namespace

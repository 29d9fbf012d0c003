// Short causal convolution of every channel, its activation, and the window that is carried between calls (forward, one token, backward).
//
//   pre_t = bias + sum_j w_j x_{t - W + 1 + j};  y = pre or pre sigmoid(pre);  x_t for t < 0 is row W - 1 + t of the state
//   backward: e = dy act'(pre);  dx_t = sum_j w_j e_{t + W - 1 - j};  dw_j = sum_t e_t x_{t - W + 1 + j};  dbias = sum_t e_t
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written).  A thread holds 16 bytes of channels and goes
// along a run of tokens with the window on registers, eight rows' loads under way at once; the W - 1 rows before a run are read again.
// The taps of a thread's channels lie together and are loaded as fours: one by one they are 40 loads that all wait for the same unit (16384 rows
// of 2048 in bf16: 43 -> 25.5 us, one token of 64 sequences, 4096 channels: 7.6 -> 3.5).  8 x 8192 rows of 4096: 207 us forward, 5.2 TB/s; 365
// backward, 4.4 TB/s.  The weights' gradient: a sum for each run, or, where a workgroup has several runs of its channels, one of these (4 x
// 262144 rows of 64 in bf16, backward: 219 -> 127 us, most of which were the sums' way through memory).
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kThreads = kConvThreads, kStepThreads = 64;
constexpr int kAhead = 8;   // rows whose loads are under way at once

template <typename IO>
struct Weights {
  static constexpr int V = kPiece<IO>;
  float w[kConvWidth][V], bias[V];

  // the taps of V channels lie together
  template <int W> __device__ __forceinline__ void load(const ConvArgs& a, int c) {
    float taps[V * W];
    load_fours<V * W>(a, a.weight, static_cast<size_t>(c) * W, taps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = taps[i * W + j];
      bias[i] = 0.0f;
    }
    if (a.bias != nullptr) load_fours<V>(a, a.bias, c, bias);
  }
  template <int COUNT> static __device__ __forceinline__ void load_fours(const ConvArgs& a, const void* p, size_t at, float* out) {
    if (a.w_bf16) {
#pragma unroll
      for (int i = 0; i < COUNT; i += 4) {
        const ushort4 x = *reinterpret_cast<const ushort4*>(static_cast<const uint16_t*>(p) + at + i);
        out[i] = bf16_to_f32(x.x), out[i + 1] = bf16_to_f32(x.y), out[i + 2] = bf16_to_f32(x.z), out[i + 3] = bf16_to_f32(x.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at + i);
        out[i] = x.x, out[i + 1] = x.y, out[i + 2] = x.z, out[i + 3] = x.w;
      }
    }
  }
};

// Where a thread is: its channels, its sequence, its run of tokens.
struct Place {
  int c, b, run;
  bool here;
  __device__ __forceinline__ Place(const ConvArgs& a, int V, long long item) {
    const int pieces = a.n / V;
    c = static_cast<int>(item % pieces) * V;
    const long long rest = item / pieces;
    run = static_cast<int>(rest % a.runs);
    here = rest / a.runs < a.B;
    b = here ? static_cast<int>(rest / a.runs) : 0;
  }
};

// Row t of a sequence: of x, of the state before it (t < 0, at least 1 - W), zero where there is none.
template <typename IO, int W>
__device__ __forceinline__ Piece<IO> row_of(const ConvArgs& a, const IO* x, int b, int c, int t) {
  if (t >= 0) return load_piece(x + t * a.xs.t);
  if (a.state != nullptr) return load_piece(static_cast<const IO*>(a.state) + (static_cast<size_t>(b) * (W - 1) + (W - 1 + t)) * a.n + c);
  return Piece<IO>{};
}

template <int W, typename IO>
__global__ void __launch_bounds__(kThreads) conv_kernel(ConvArgs a) {
  constexpr int V = kPiece<IO>;
  const Place p(a, V, static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x);
  if (!p.here) return;
  Weights<IO> k;
  k.template load<W>(a, p.c);
  const int length = length_of(a.lengths, p.b, a.T);
  const IO* x = static_cast<const IO*>(a.x) + p.b * a.xs.b + p.c;
  IO* y = static_cast<IO*>(a.y) + p.b * a.ys.b + p.c;
  const int first = p.run * a.run, last = min(first + a.run, a.T), end = min(last, length);
  if (first < end) {
    Piece<IO> window[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) window[j] = row_of<IO, W>(a, x, p.b, p.c, first - (W - 1) + j);
    for (int t0 = first; t0 < end; t0 += kAhead) {
      Piece<IO> rows[kAhead + W - 1];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) rows[j] = window[j];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) rows[W - 1 + i] = load_piece(x + min(t0 + i, end - 1) * a.xs.t);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        float out[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float s = k.bias[v];
#pragma unroll
          for (int j = 0; j < W; ++j) s = fmaf(k.w[j][v], rows[i + j][v], s);
          out[v] = a.silu ? s * sigmoid(s) : s;
        }
        if (t0 + i < end) store_piece(y + (t0 + i) * a.ys.t, out);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) window[j] = rows[kAhead + j];
    }
  }
  for (int t = max(first, end); t < last; ++t) {
    const float zero[V] = {};
    store_piece(y + t * a.ys.t, zero);
  }
  if (p.run == 0 && a.state_T != nullptr) {
    Piece<IO> kept[W - 1];      // all of them read before one is written: the state may be the same buffer
#pragma unroll
    for (int j = 0; j < W - 1; ++j) kept[j] = row_of<IO, W>(a, x, p.b, p.c, length - (W - 1) + j);
    IO* out = static_cast<IO*>(a.state_T) + static_cast<size_t>(p.b) * (W - 1) * a.n + p.c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Piece<IO>*>(out + static_cast<size_t>(j) * a.n) = kept[j];
  }
}

template <int W, typename IO>
__global__ void __launch_bounds__(kThreads) conv_backward_kernel(ConvArgs a) {
  constexpr int V = kPiece<IO>;
  const Place p(a, V, static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x);
  if (!p.here && !a.joined) return;
  Weights<IO> k;
  k.template load<W>(a, p.c);
  const int length = length_of(a.lengths, p.b, a.T);
  const IO* x = static_cast<const IO*>(a.x) + p.b * a.xs.b + p.c;
  const IO* dy = static_cast<const IO*>(a.dy) + p.b * a.ys.b + p.c;
  IO* dx = static_cast<IO*>(a.dx) + p.b * a.dxs.b + p.c;
  const IO* dstate_T = a.dstate_T == nullptr ? nullptr : static_cast<const IO*>(a.dstate_T) + static_cast<size_t>(p.b) * (W - 1) * a.n + p.c;
  IO* dstate = a.dstate == nullptr ? nullptr : static_cast<IO*>(a.dstate) + static_cast<size_t>(p.b) * (W - 1) * a.n + p.c;
  const int first = p.run * a.run, last = min(first + a.run, a.T);
  const int own = min(last, length);          // tokens whose e counts for the weights here
  const int end = p.here ? last + W - 1 : first;   // tokens that the run's rows are read by
  float e[W][V] = {};                         // e[j] of token t - (W - 1) + j
  float dw[W][V] = {}, db[V] = {};
  Piece<IO> window[W];                        // x of the same tokens
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int t = first - (W - 1) + j;
    window[j + 1] = t < length ? row_of<IO, W>(a, x, p.b, p.c, t) : Piece<IO>{};
  }
  constexpr int kBack = 4;                    // rows whose loads are under way at once
  for (int t0 = first; t0 < end; t0 += kBack) {
    Piece<IO> rows[kBack], grads[kBack];
#pragma unroll
    for (int i = 0; i < kBack; ++i) {
      const int t = max(min(t0 + i, length - 1), 0);
      rows[i] = length > 0 ? load_piece(x + t * a.xs.t) : Piece<IO>{};
      grads[i] = length > 0 ? load_piece(dy + t * a.ys.t) : Piece<IO>{};
    }
#pragma unroll
    for (int i = 0; i < kBack; ++i) {
      const int t = t0 + i;
      const bool live = t < min(end, length);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) window[j] = window[j + 1];
      window[W - 1] = rows[i];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float s = k.bias[v];
#pragma unroll
        for (int j = 0; j < W; ++j) s = fmaf(k.w[j][v], window[j][v], s);
        float g = grads[i][v];
        if (a.silu) {
          const float sig = sigmoid(s);
          g *= sig * fmaf(s, 1.0f - sig, 1.0f);
        }
        g = live ? g : 0.0f;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) e[j][v] = e[j + 1][v];
        e[W - 1][v] = g;
        if (live && t < own) {
#pragma unroll
          for (int j = 0; j < W; ++j) dw[j][v] = fmaf(g, window[j][v], dw[j][v]);
          db[v] += g;
        }
      }
      // the row that no later token reads
      const int r = t - (W - 1);
      if (t < end && (r >= first || (first == 0 && dstate != nullptr))) {
        float out[V];
        const int j_T = r - (length - (W - 1));       // its place in the state that is carried on
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float s = 0.0f;
#pragma unroll
          for (int j = 0; j < W; ++j) s = fmaf(k.w[W - 1 - j][v], e[j][v], s);
          out[v] = s;
        }
        if (dstate_T != nullptr && j_T >= 0 && j_T < W - 1) {
          const Piece<IO> d = load_piece(dstate_T + static_cast<size_t>(j_T) * a.n);
#pragma unroll
          for (int v = 0; v < V; ++v) out[v] += d[v];
        }
        if (r >= 0) store_piece(dx + r * a.dxs.t, out);
        else store_piece(dstate + static_cast<size_t>(W - 1 + r) * a.n, out);
      }
    }
  }
  if (a.sum_part == nullptr) return;
  if (a.joined) {      // the workgroup's runs of each channel, in their order
    __shared__ __align__(16) float of_run[kThreads * V];
    const int pieces = a.n / V, at = static_cast<int>(static_cast<long long>(blockIdx.x) * kThreads % pieces);
    float* part = a.sum_part + static_cast<size_t>(blockIdx.x) * (W + 1) * a.n;
#pragma unroll
    for (int j = 0; j <= W; ++j) {
      __syncthreads();
      store_piece(of_run + threadIdx.x * V, j < W ? dw[j < W ? j : 0] : db);
      __syncthreads();
      for (int i = threadIdx.x; i < a.n; i += kThreads) {
        const int piece = i / V;
        float sum = 0.0f;
        for (int q = piece >= at ? piece - at : piece - at + pieces; q < kThreads; q += pieces) sum += of_run[q * V + i % V];
        part[static_cast<size_t>(j) * a.n + i] = sum;
      }
    }
    return;
  }
  float* part = a.sum_part + (static_cast<size_t>(p.b) * a.runs + p.run) * (W + 1) * a.n + p.c;
#pragma unroll
  for (int j = 0; j < W; ++j) store_piece(part + static_cast<size_t>(j) * a.n, dw[j]);
  store_piece(part + static_cast<size_t>(W) * a.n, db);
}

// One token: the window moves on in place.
template <int W, typename IO>
__global__ void __launch_bounds__(kStepThreads) conv_step_kernel(ConvArgs a) {
  constexpr int V = kPiece<IO>;
  const Place p(a, V, static_cast<long long>(blockIdx.x) * kStepThreads + threadIdx.x);
  if (!p.here) return;
  IO* state = static_cast<IO*>(a.state_T) + static_cast<size_t>(p.b) * (W - 1) * a.n + p.c;
  Piece<IO> window[W];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) window[j] = load_piece(state + static_cast<size_t>(j) * a.n);
  window[W - 1] = load_piece(static_cast<const IO*>(a.x) + p.b * a.xs.b + p.c);
  Weights<IO> k;
  k.template load<W>(a, p.c);
  float out[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float s = k.bias[v];
#pragma unroll
    for (int j = 0; j < W; ++j) s = fmaf(k.w[j][v], window[j][v], s);
    out[v] = a.silu ? s * sigmoid(s) : s;
  }
  store_piece(static_cast<IO*>(a.y) + p.b * a.ys.b + p.c, out);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Piece<IO>*>(state + static_cast<size_t>(j) * a.n) = window[j + 1];
}

template <int W, typename IO>
hipError_t launch(const ConvArgs& a, int what, hipStream_t stream) {
  const long long items = static_cast<long long>(a.n / kPiece<IO>) * a.B * a.runs;
  const void* kernel = what == 0   ? reinterpret_cast<const void*>(&conv_kernel<W, IO>)
                       : what == 1 ? reinterpret_cast<const void*>(&conv_step_kernel<W, IO>)
                                   : reinterpret_cast<const void*>(&conv_backward_kernel<W, IO>);
  ConvArgs args = a;
  void* params[] = {&args};
  const int threads = what == 1 ? kStepThreads : kThreads;
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>((items + threads - 1) / threads)), dim3(threads), params, 0, stream);
}
template <typename IO>
hipError_t launch_width(const ConvArgs& a, int width, int what, hipStream_t stream) {
  switch (width) {
    case 2: return launch<2, IO>(a, what, stream);
    case 3: return launch<3, IO>(a, what, stream);
    case 4: return launch<4, IO>(a, what, stream);
    default: return hipErrorInvalidValue;
  }
}
hipError_t launch_any(const ConvArgs& a, int width, int io_dtype, int what, hipStream_t stream) {
  return io_dtype == 1 ? launch_width<uint16_t>(a, width, what, stream) : launch_width<float>(a, width, what, stream);
}

}  // namespace

hipError_t launch_causal_conv(const ConvArgs& a, int width, int io_dtype, hipStream_t stream) { return launch_any(a, width, io_dtype, 0, stream); }
hipError_t launch_causal_conv_step(const ConvArgs& a, int width, int io_dtype, hipStream_t stream) { return launch_any(a, width, io_dtype, 1, stream); }
hipError_t launch_causal_conv_backward(const ConvArgs& a, int width, int io_dtype, hipStream_t stream) {
  return launch_any(a, width, io_dtype, 2, stream);
}

}  // namespace vla

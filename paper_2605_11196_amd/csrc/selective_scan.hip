// The selective state space scan: a state of N numbers for every channel, whose decay, input and read-out depend on the token (forward).
//
//   h_t[c,s] = exp(dt_t[c] A[c,s]) h_{t-1}[c,s] + dt_t[c] u_t[c] B_t[s];  y_t[c] = (sum_s C_t[s] h_t[c,s] + D[c] u_t[c]) z sigmoid(z)
//   dt = softplus(delta + bias) (or delta + bias)
//
// Bound by vector instructions: an element of the state takes a product and an exponential (8 cycles of a SIMD, the others 2 to 3), the input's
// product, the update and the read-out, and nothing of that is a matrix product, since every element has a decay of its own.  A lane holds
// eight states of two neighbouring channels, a wave eight states of 128 channels, a workgroup of N / 8 waves all states of them, and
// goes along the tokens in blocks of eight: the steps and inputs of a block, which all waves need, are formed once and shared in LDS with B and C
// as float32 (operands from vector registers take half the time of scalar ones), and the waves' parts of y are added up there.
// Few sequences of few channels are cut into time segments: a first pass gives the end of every segment from a zero start and the
// sum of its steps (its decay is exp(A sum dt)), a second kernel the states that the segments start from.
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kStates = 8;         // of a lane, for each of its two channels
constexpr int TB = kScanBlock;

// Where a workgroup is.
struct Tile {
  int b, seg, tile, group, c0, pairs;   // c0: first channel; pairs of channels that are there
  __device__ __forceinline__ explicit Tile(const ScanArgs& a) {
    const unsigned tiles = a.G * a.tiles;
    tile = blockIdx.x % tiles;
    const unsigned rest = blockIdx.x / tiles;
    seg = rest % a.n_seg;
    b = rest / a.n_seg;
    group = tile / a.tiles;
    const int of_group = a.n / a.G, first = tile % a.tiles * kScanTile;
    c0 = group * of_group + first;
    pairs = min(of_group - first, kScanTile) / 2;
  }
};
__device__ __forceinline__ int length_of(const int* lengths, int b, int T) { return lengths == nullptr ? T : min(max(lengths[b], 0), T); }

// The pair of B's or C's values that a thread stages for a block: token, place in the row, value
template <int W, typename IO>
struct Staged {
  static constexpr int N = kStates * W;
  int t, at;            // token of the block; float of the row [B | C]
  const IO* from;       // the row of token 0
  long long step;
  __device__ __forceinline__ Staged(const ScanArgs& a, const Tile& w) {
    t = threadIdx.x / N;
    at = threadIdx.x % N * 2;
    const bool is_c = at >= N;
    step = is_c ? a.C_t : a.B_t;
    from = is_c ? static_cast<const IO*>(a.Cm) + w.b * a.C_b + w.group * a.C_g + (at - N)
                : static_cast<const IO*>(a.Bm) + w.b * a.B_b + w.group * a.B_g + at;
  }
};

template <int W, typename IO, bool MAP>
__global__ void __launch_bounds__(64 * W) scan_kernel(ScanArgs a) {
  constexpr int N = kStates * W, PER = TB / W;
  __shared__ f4 steps[TB][64];        // dt, dt u of both channels of a lane
  __shared__ __align__(16) float rows[TB][2 * N];   // B, C
  __shared__ f2 part[MAP ? 1 : W][TB][64];
  const Tile w(a);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int length = length_of(a.lengths, w.b, a.T);
  const bool here = lane < w.pairs;
  const int c = w.c0 + (here ? 2 * lane : 0);
  const IO* u = static_cast<const IO*>(a.u) + w.b * a.us.b + c;
  const IO* delta = static_cast<const IO*>(a.delta) + w.b * a.ds.b + c;
  const IO* z = a.z == nullptr ? nullptr : static_cast<const IO*>(a.z) + w.b * a.zs.b + c;
  const Staged<W, IO> mine(a, w);
  const bool stage = !MAP || mine.at < N;

  float A2[2][kStates], h[2][kStates];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const size_t at = static_cast<size_t>(c + j) * N + wave * kStates;
    const float* from = a.A + at;
    const float* h0 = MAP ? nullptr
                      : a.n_seg > 1 ? a.seg_h + (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n * N + at
                      : a.h0 != nullptr ? a.h0 + static_cast<size_t>(w.b) * a.n * N + at : nullptr;
#pragma unroll
    for (int s = 0; s < kStates; ++s) {
      A2[j][s] = from[s] * kLog2e;
      h[j][s] = h0 != nullptr ? h0[s] : 0.0f;
    }
  }
  const f2 bias = a.bias != nullptr ? load2(a.bias + c) : f2{0.0f, 0.0f};
  const f2 D = a.D != nullptr ? load2(a.D + c) : f2{0.0f, 0.0f};
  f2 sum_dt = {0.0f, 0.0f};

  const int first = w.seg * a.seg_blocks, last = min(first + a.seg_blocks, (a.T + TB - 1) / TB);
  const int live = min(last, (length + TB - 1) / TB);     // blocks with a token of the sequence
  // what a block reads, on its way while the one before it is worked on
  Pair<IO> next_u[PER], next_delta[PER], next_z[PER], next_row{};
  const auto fetch = [&](int block) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const long long t = min(block * TB + wave * PER + k, length - 1);
      next_u[k] = raw2(u + t * a.us.t);
      next_delta[k] = raw2(delta + t * a.ds.t);
      if (!MAP && z != nullptr) next_z[k] = raw2(z + t * a.zs.t);
    }
    if (stage) next_row = raw2(mine.from + min(block * TB + mine.t, length - 1) * mine.step);
  };
  if (first < live) fetch(first);
  for (int block = first; block < live; ++block) {
    if (!MAP && a.kept != nullptr) {
      f4* to = reinterpret_cast<f4*>(a.kept) +
               (((static_cast<size_t>(w.b) * a.blocks + block) * (a.G * a.tiles) + w.tile) * W + wave) * 4 * 64 + lane;
#pragma unroll
      for (int j = 0; j < 4; ++j) to[64 * j] = f4{h[j / 2][j % 2 * 4], h[j / 2][j % 2 * 4 + 1], h[j / 2][j % 2 * 4 + 2], h[j / 2][j % 2 * 4 + 3]};
    }
    f2 now_u[PER], now_z[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int t = block * TB + wave * PER + k;
      const f2 x = wide2(next_u[k]), raw = wide2(next_delta[k]) + bias;
      const bool in = t < length;
      const float d0 = a.softplus ? softplus(raw[0]) : raw[0], d1 = a.softplus ? softplus(raw[1]) : raw[1];
      steps[wave * PER + k][lane] = f4{in ? d0 : 0.0f, in ? d0 * x[0] : 0.0f, in ? d1 : 0.0f, in ? d1 * x[1] : 0.0f};
      now_u[k] = x;
      if (!MAP && z != nullptr) now_z[k] = wide2(next_z[k]);
    }
    if (stage) {
      const f2 v = wide2(next_row);
      const bool in = block * TB + mine.t < length;
      *reinterpret_cast<f2*>(&rows[mine.t][mine.at]) = f2{in ? v[0] : 0.0f, in ? v[1] : 0.0f};
    }
    if (block + 1 < live) fetch(block + 1);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      const f4 s = steps[t][lane];
      const f4* Bt = reinterpret_cast<const f4*>(&rows[t][wave * kStates]);
      const f4* Ct = reinterpret_cast<const f4*>(&rows[t][N + wave * kStates]);
      const f4 b[2] = {Bt[0], Bt[1]};
      f4 cc[2] = {};
      if (!MAP) {
        cc[0] = Ct[0];
        cc[1] = Ct[1];
      }
      f2 y = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < kStates; ++i) {
          const float e = __builtin_amdgcn_exp2f(s[2 * j] * A2[j][i]);
          h[j][i] = fmaf(e, h[j][i], s[2 * j + 1] * b[i / 4][i % 4]);
          if (!MAP) y[j] = fmaf(cc[i / 4][i % 4], h[j][i], y[j]);
        }
      }
      if (MAP && wave == 0) sum_dt += f2{s[0], s[2]};
      if (!MAP) part[wave][t][lane] = y;
    }
    __syncthreads();
    if (MAP) continue;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = wave * PER + k, t = block * TB + i;
      f2 y = D * now_u[k];
#pragma unroll
      for (int v = 0; v < W; ++v) y += part[v][i][lane];
      if (z != nullptr) y *= f2{now_z[k][0] * sigmoid(now_z[k][0]), now_z[k][1] * sigmoid(now_z[k][1])};
      if (t >= length) y = f2{0.0f, 0.0f};
      if (here && t < a.T) store2(static_cast<IO*>(a.y) + w.b * a.ys.b + t * a.ys.t + c, y);
    }
  }
  if (!MAP) {
    for (int t = max(first, live) * TB + wave; t < min(last * TB, a.T); t += W) {
      if (here) store2(static_cast<IO*>(a.y) + w.b * a.ys.b + t * a.ys.t + c, f2{0.0f, 0.0f});
    }
  }
  float* to = MAP ? a.seg_h + (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n * N
              : w.seg == a.n_seg - 1 && a.h_T != nullptr ? a.h_T + static_cast<size_t>(w.b) * a.n * N : nullptr;
  if (to != nullptr && here) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float* row = to + static_cast<size_t>(c + j) * N + wave * kStates;
#pragma unroll
      for (int i = 0; i < kStates; i += 4) *reinterpret_cast<f4*>(row + i) = f4{h[j][i], h[j][i + 1], h[j][i + 2], h[j][i + 3]};
    }
  }
  if (MAP && wave == 0 && here) store2(a.seg_dt + (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n + c, sum_dt);
}

// The states that the segments start from, in the place of their maps' ends; backward: the gradients behind them, from the last one on.
constexpr int kCombine = 256;
template <bool BACK>
__global__ void __launch_bounds__(kCombine) combine_kernel(ScanArgs a, int N) {
  const long long each = static_cast<long long>(a.n) * N, i = static_cast<long long>(blockIdx.x) * kCombine + threadIdx.x;
  if (i >= each * a.nb) return;
  const long long b = i / each, at = i % each;
  const float A2 = a.A[at] * kLog2e;
  const float* start = BACK ? a.dh_T : a.h0;
  float h = start != nullptr ? start[i] : 0.0f;
  float* ends = a.seg_h + b * a.n_seg * each + at;
  const float* dt = a.seg_dt + b * a.n_seg * a.n + at / N;
  constexpr int kAhead = 8;
  for (int s0 = 0; s0 < a.n_seg; s0 += kAhead) {
    float end[kAhead], decay[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = min(s0 + k, a.n_seg - 1), seg = BACK ? a.n_seg - 1 - s : s;
      end[k] = ends[seg * each];
      decay[k] = dt[static_cast<long long>(seg) * a.n];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = s0 + k, seg = BACK ? a.n_seg - 1 - s : s;
      if (s >= a.n_seg) break;
      ends[seg * each] = h;
      h = fmaf(__builtin_amdgcn_exp2f(decay[k] * A2), h, end[k]);
    }
  }
}

template <int W, typename IO>
hipError_t launch(const ScanArgs& a, bool map, hipStream_t stream) {
  const long long groups = static_cast<long long>(a.nb) * a.n_seg * a.G * a.tiles;
  ScanArgs args = a;
  void* params[] = {&args};
  const void* kernel = map ? reinterpret_cast<const void*>(&scan_kernel<W, IO, true>) : reinterpret_cast<const void*>(&scan_kernel<W, IO, false>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>(groups)), dim3(64 * W), params, 0, stream);
}
template <typename IO>
hipError_t launch_states(const ScanArgs& a, int N, bool map, hipStream_t stream) {
  switch (N) {
    case 8: return launch<1, IO>(a, map, stream);
    case 16: return launch<2, IO>(a, map, stream);
    case 32: return launch<4, IO>(a, map, stream);
    case 64: return launch<8, IO>(a, map, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_selective_scan(const ScanArgs& a, int N, int io_dtype, bool map, hipStream_t stream) {
  return io_dtype == 1 ? launch_states<uint16_t>(a, N, map, stream) : launch_states<float>(a, N, map, stream);
}

hipError_t launch_selective_combine(const ScanArgs& a, int N, bool backward, hipStream_t stream) {
  const long long items = static_cast<long long>(a.nb) * a.n * N;
  ScanArgs args = a;
  void* params[] = {&args, &N};
  const void* kernel = backward ? reinterpret_cast<const void*>(&combine_kernel<true>) : reinterpret_cast<const void*>(&combine_kernel<false>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>((items + kCombine - 1) / kCombine)), dim3(kCombine), params, 0, stream);
}

}  // namespace vla

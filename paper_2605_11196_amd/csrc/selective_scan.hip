// The selective state space scan: a state of N numbers for every channel, whose decay, input and read-out depend on the token (forward).
//
//   h_t[c,s] = exp(dt_t[c] A[c,s]) h_{t-1}[c,s] + dt_t[c] u_t[c] B_t[s];  y_t[c] = (sum_s C_t[s] h_t[c,s] + D[c] u_t[c]) z sigmoid(z)
//   dt = softplus(delta + bias) (or delta + bias)
//
// Bound by vector instructions: an element of the state takes a product and an exponential, the input's product, the update and the
// read-out, and nothing of that is a matrix product, since every element has a decay of its own.  8 x 2048 tokens, 4096 channels of 16 states,
// bfloat16: 345 us, vector unit busy for 74 % of the cycles with 8.1 instructions an element (138 us for those five alone), two waves a SIMD, which is all that so
// many channels give; a long sequence in segments: 86 %, with six waves a SIMD at most (80 registers; float32 and 32 states five, 64 states four; 8 states five
// and four).
// Few sequences of few channels are cut into time segments: a first pass gives the end of every segment from a zero start and the
// sum of its steps (its decay is exp(A sum dt)), a second kernel the states that the segments start from.
#include "selective_lanes.h"

namespace vla {
namespace {

template <int N, typename IO, bool MAP>
__global__ void __launch_bounds__(64 * scan_waves(N)) scan_kernel(ScanArgs a) {
  typedef ScanPlace<N> P;
  constexpr int LN = P::LN, OWN = P::OWN, TURNS = kTurns<LN>;
  __shared__ __align__(16) f2 steps[scan_waves(N)][2][TB][P::CW];       // dt, dt u
  __shared__ __align__(16) float staged[scan_waves(N)][2][TB][2 * N];   // B, C
  __shared__ __align__(8) float outs[MAP ? 1 : scan_waves(N)][TB][P::CW];            // sums of the read-out
  const P w(a);
  if (MAP && w.seg == a.n_seg - 1) return;      // nothing starts from its end
  const size_t state = (static_cast<size_t>(w.b) * a.n + w.c) * N + 4 * w.q, of_seg = (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n + w.c;
  const bool gated = !MAP && a.z != nullptr;
  const ScanRows<N, IO> u(w, a.u, a.us), delta(w, a.delta, a.ds), z(w, gated ? a.z : a.u, gated ? a.zs : a.us), out(w, MAP ? a.u : a.y, MAP ? a.us : a.ys);
  char *next_row_u = u.row(w.first), *next_row_delta = delta.row(w.first), *next_row_z = z.row(w.first), *row_out = out.row(w.first);
  ScanStage<N, IO> rows(w, a, w.first);

  const f4 A2 = *reinterpret_cast<const f4*>(a.A + static_cast<size_t>(w.c) * N + 4 * w.q) * kLog2e;
  f4 h = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!MAP && a.n_seg > 1) h = *reinterpret_cast<const f4*>(a.seg_h + of_seg * N + 4 * w.q);
  if (!MAP && a.n_seg == 1 && a.h0 != nullptr) h = *reinterpret_cast<const f4*>(a.h0 + state);
  const f2 bias = pair_of(a.bias, w.c2), D = pair_of(a.D, w.c2);
  float sum_dt = 0.0f;

  // What a block reads is on its way while the one before the one before it is worked on, and its steps are formed while the one before it
  // is: neither the loads' latency nor that of the transcendental instructions stands between the states' tokens.  Loads and stores are counted
  // together and in order, so that a wait for loads is one for the stores before it: a block's results are stored a block later, between the
  // wait for one block's rows and the loads of the next one's.
  Pair<IO> next_u[OWN] = {}, next_delta[OWN] = {}, next_z[OWN] = {};
  f2 x[OWN], v[OWN], now_x[OWN], now_v[OWN];
  const auto fetch = [&](int t0) {      // the blocks one after the other
    if (t0 + TB <= a.T) {
      u.load(next_row_u, next_u);
      delta.load(next_row_delta, next_delta);
      if (gated) z.load(next_row_z, next_z);
      rows.load(TB);
    } else {
      const int tokens = a.T - t0;
      u.load(next_row_u, next_u, w, tokens);
      delta.load(next_row_delta, next_delta, w, tokens);
      if (gated) z.load(next_row_z, next_z, w, tokens);
      rows.load(tokens);
      asm volatile("" ::: "memory");      // two ways with loads of their own, and no choice of addresses for one
    }
    next_row_u += TB * u.step;
    next_row_delta += TB * delta.step;
    next_row_z += TB * z.step;
    rows.template go<false>();
  };
  const auto form = [&](int t0, int buffer) {
    f2 dt[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) dt[k] = wide2(next_delta[k]) + bias;
    if (a.softplus) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) dt[k] = f2{softplus(dt[k][0]), softplus(dt[k][1])};
    }
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      const bool in = t0 + w.own(k) < w.length;
      x[k] = wide2(or_zero(in, next_u[k]));
      v[k] = wide2(next_z[k]);
      const f2 d = or_zero(in, dt[k]);
      *reinterpret_cast<f4*>(&steps[w.wave][buffer][w.own(k)][2 * w.pair]) = f4{d[0], d[0] * x[k][0], d[1], d[1] * x[k][1]};
    }
    rows.put(staged[w.wave][buffer][0], t0 + rows.t < w.length);
  };
  if (w.first < w.live) {
    fetch(w.first);
    form(w.first, 0);
    if (w.first + TB < w.live) fetch(w.first + TB);
  }
  Pair<IO> done[OWN] = {};
  const auto put = [&](int t0) {
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      if (w.here2 && t0 + w.own(k) < w.last) out.store(row_out, k, done[k]);
    }
    row_out += TB * out.step;
  };
  const size_t kept_step = static_cast<size_t>(a.n) * N;
  float* kept = a.kept + (static_cast<size_t>(w.b) * a.blocks + w.first / TB) * kept_step + static_cast<size_t>(w.c) * N + 4 * w.q;
  int now = 0;
  for (int t0 = w.first; t0 < w.live; t0 += TB) {
    wave_fence();
    const f2* const step = steps[w.wave][now][0];
    const float* const mine = staged[w.wave][now][0];
    f2 s_[2];
    f4 B_[2], C_[2] = {};
    const auto operands = [&](int t) {
      s_[t % 2] = step[t * P::CW + w.in_wave];
      B_[t % 2] = *reinterpret_cast<const f4*>(mine + t * 2 * N + 4 * w.q);
      if (!MAP) C_[t % 2] = *reinterpret_cast<const f4*>(mine + t * 2 * N + N + 4 * w.q);
    };
    operands(0);
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      now_x[k] = x[k];
      now_v[k] = v[k];
    }
    now ^= 1;
    form(t0 + TB, now);
    if (!MAP && a.kept != nullptr) {
      if (w.here) *reinterpret_cast<f4*>(kept) = h;
      kept += kept_step;
    }
    if (!MAP && t0 > w.first) put(t0 - TB);
    if (t0 + 2 * TB < w.live) fetch(t0 + 2 * TB);
    float some[4], y[TURNS] = {};
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      if (t + 1 < TB) operands(t + 1);
      const f2 s = s_[t % 2];
      const f4 B = B_[t % 2], C = C_[t % 2];
      float read = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = fmaf(__builtin_amdgcn_exp2f(s[0] * A2[i]), h[i], s[1] * B[i]);
        if (!MAP) read = i == 0 ? C[0] * h[0] : fmaf(C[i], h[i], read);
      }
      if (MAP) sum_dt += s[0];
      else keep_sum<LN>(read, some, y, t, t % LN == LN - 1, w.q);
    }
    if (MAP) continue;
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
      if (LN <= TB || w.q < TB) outs[w.wave][LN * k + w.q][w.in_wave] = y[k];
    }
    wave_fence();
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      const int t = t0 + w.own(k);
      f2 r = *reinterpret_cast<const f2*>(&outs[w.wave][w.own(k)][2 * w.pair]);
      if (a.D != nullptr) r += D * now_x[k];      // without D nothing is added: 0 times an infinite input would be no number
      if (gated) r *= f2{now_v[k][0] * sigmoid(now_v[k][0]), now_v[k][1] * sigmoid(now_v[k][1])};
      done[k] = or_zero(t < w.length, narrow2<IO>(r));
    }
  }
  if (!MAP) {
    const int gone = w.live > w.first ? w.first + (w.live - w.first + TB - 1) / TB * TB : w.first;
    if (gone > w.first) put(gone - TB);
    for (int t0 = gone; t0 < w.last; t0 += TB) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        if (w.here2 && t0 + w.own(k) < w.last) out.store(row_out, k, Pair<IO>{});
      }
      row_out += TB * out.step;
    }
  }
  if (!w.here) return;
  if (MAP) {
    *reinterpret_cast<f4*>(a.seg_h + of_seg * N + 4 * w.q) = h;
    if (w.q == 0) a.seg_dt[of_seg] = sum_dt;
  } else if (w.seg == a.n_seg - 1 && a.h_T != nullptr) {
    *reinterpret_cast<f4*>(a.h_T + state) = h;
  }
}

// The states that the segments start from, in the place of their maps' ends; backward: the gradients behind them, from the last one on.  (The segment
// that comes last has no map: what is read for it goes nowhere.)
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
      // nothing of nothing is left, also where A > 0 has made the factor infinite
      h = h == 0.0f ? end[k] : fmaf(__builtin_amdgcn_exp2f(decay[k] * A2), h, end[k]);
    }
  }
}

template <int N, typename IO>
hipError_t launch(const ScanArgs& a, bool map, hipStream_t stream) {
  const long long groups = static_cast<long long>(a.nb) * a.n_seg * a.G * a.tiles;
  ScanArgs args = a;
  void* params[] = {&args};
  const void* kernel = map ? reinterpret_cast<const void*>(&scan_kernel<N, IO, true>) : reinterpret_cast<const void*>(&scan_kernel<N, IO, false>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>(groups)), dim3(64 * scan_waves(N)), params, 0, stream);
}
template <typename IO>
hipError_t launch_states(const ScanArgs& a, int N, bool map, hipStream_t stream) {
  switch (N) {
    case 8: return launch<8, IO>(a, map, stream);
    case 16: return launch<16, IO>(a, map, stream);
    case 32: return launch<32, IO>(a, map, stream);
    case 64: return launch<64, IO>(a, map, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int selective_tile(int N) { return scan_tile(N); }

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

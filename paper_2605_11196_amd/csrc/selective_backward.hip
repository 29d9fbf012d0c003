// Gradients of the selective state space scan.
//
//   e = dy z sigmoid(z);  g_t[c,s] = e_t[c] C_t[s] + a_{t+1}[c,s] g_{t+1}[c,s], a = exp(dt A), behind the last token dh_T
//   dC_t[s] = sum_c e_t[c] h_t[c,s];  dB_t[s] = sum_c g_t[c,s] dt_t[c] u_t[c];  with p = sum_s g B:  du = D e + dt p
//   ddt = sum_s g a h_{t-1} A + u p;  dA[c,s] = sum_t g a h_{t-1} dt;  dD = sum e u;  dh0 = a_1 g_1;  dz from y before the gate
//
// Bound by vector instructions, as the forward pass, whose layout this has.  Blocks of eight tokens from the last to the first: from the state that
// the forward pass has kept before the block the decays a and the products a h_{t-1} of its tokens are formed again and stay on registers, then g goes
// back through them.  dB and dC are sums over channels: those of a wave by lane swaps and DPP, eight numbers at a time, those of the
// waves of a workgroup through LDS (one barrier a block, the place changes), those of the workgroups by a second kernel.  Time segments
// as in the forward pass, from the last to the first.  8 x 2048 tokens, 4096 channels of 16 states, bfloat16: 930 us, vector unit busy for 77 %
// of the cycles with 23 instructions an element, 4 of them and a fifth of the time for the sums over channels; of the LDS's cycles, a third of all, a quarter are
// bank conflicts (4.2e7 of 1.7e8).  (The sums through the float32 matrix
// instruction, by a matrix of zeros and ones: 1309 us, it does not run beside vector instructions.)
//
// The kernel keeps to registers that no copy has to stand in for (the tests hold it to that): with more live values than fit, the compiler keeps addresses in
// accumulation registers over the loop, and writes them behind a divergent branch before it has turned the lanes on again.
#include "selective_lanes.h"

namespace vla {
namespace {

__device__ __forceinline__ void swap32(float& a, float& b) {   // a: the lower half's a and b; b: the upper half's
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap16(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
// p[4 j + i], tokens 2 pair + j and states i of a lane, summed over the wave's channels, into rows[token][4 q + i] (step: floats from row to row): lane
// bits 5, 4 and 3 (LN = 16: 5 and 4) come to say which of the numbers a lane has.  LN = 4: bit 2 too, for the two pairs of four tokens, of which the
// first one's numbers wait in `half` for the last one's.  A rotation by four lanes takes bit 3 along for one half of the lanes, which does not matter as
// long as the sum over bit 3 is still to come.
template <int LN>
__device__ __forceinline__ void wave_sums(const float (&p)[8], float (&half)[2], bool last, int pair, float* rows, int step, int lane) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = p[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    swap32(x[i], x[i + 4]);
    x[i] += x[i + 4];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    swap16(x[i], x[i + 2]);
    x[i] += x[i + 2];
  }
  const int q = lane % LN;
  const bool odd = lane & 8;
  if constexpr (LN == 4) {
    if (!last) {
      half[0] = x[0];
      half[1] = x[1];
      return;
    }
    const bool second = lane & 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float a = pair % 2 ? half[i] : x[i], b = pair % 2 ? x[i] : half[i], keep = second ? b : a, send = second ? a : b;
      x[i] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), 0x124, 0xf, 0xf, true));
    }
    const float keep = odd ? x[1] : x[0], send = odd ? x[0] : x[1];
    const float sum = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), 0x128, 0xf, 0xf, true));
    float* to = rows + (lane / 4 % 2 * 2 + lane / 32) * step + 4 * q + lane / 16 % 2 * 2 + lane / 8 % 2;
    to[pair / 2 * 4 * step] = sum;
    return;
  }
  float* to = rows + (2 * pair + lane / 32) * step + 4 * q + (lane / 16 % 2) * 2;
  if constexpr (LN == 16) {
    *reinterpret_cast<f2*>(to) = f2{x[0], x[1]};
  } else if constexpr (LN != 4) {
    const float keep = odd ? x[1] : x[0], send = odd ? x[0] : x[1];
    float sum = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), 0x128, 0xf, 0xf, true));
    if constexpr (LN == 2) {
      sum += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(sum), 0x104, 0xf, 0xf, true));   // from four lanes on
      sum = dpp_sum<0x4E>(sum);
    }
    if (LN == 8 || (lane & 7 & ~(LN - 1)) == 0) to[odd ? 1 : 0] = sum;
  }
}

template <int N, typename IO, bool MAP>
__global__ void __launch_bounds__(64 * scan_waves(N)) __attribute__((amdgpu_waves_per_eu(2))) backward_kernel(ScanArgs a) {
  typedef ScanPlace<N> P;
  constexpr int LN = P::LN, OWN = P::OWN, TURNS = kTurns<LN>, W = scan_waves(N);
  __shared__ f4 steps[W][TB][P::CW];                     // dt, dt u, e; then the sums over the states: y, p, sum g a h A
  __shared__ __align__(16) float staged[W][TB][2 * N];   // B, C
  __shared__ __align__(16) float sums[2][MAP ? 1 : W][TB][2 * N];
  const P w(a);
  if (MAP && w.seg == 0) return;      // nothing ends at its start
  const size_t state = (static_cast<size_t>(w.b) * a.n + w.c) * N + 4 * w.q, of_seg = (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n + w.c;
  const bool gated = a.z != nullptr;
  float* const mine = staged[w.wave][0];
  f4* const step = steps[w.wave][0];

  const f4 A2 = *reinterpret_cast<const f4*>(a.A + static_cast<size_t>(w.c) * N + 4 * w.q) * kLog2e;
  f4 g = {0.0f, 0.0f, 0.0f, 0.0f}, dA = g;
  if (!MAP && a.n_seg > 1) g = *reinterpret_cast<const f4*>(a.seg_h + of_seg * N + 4 * w.q);
  if (!MAP && a.n_seg == 1 && a.dh_T != nullptr) g = *reinterpret_cast<const f4*>(a.dh_T + state);
  const f2 bias = pair_of(a.bias, w.c2), D = pair_of(a.D, w.c2);
  float sum_dt = 0.0f;
  f2 dD = {0.0f, 0.0f}, dbias = dD;

  const int last = w.live > w.first ? w.first + (w.live - 1 - w.first) / TB * TB : w.first - TB;   // block
  // Tokens that the last block has not: it is gone through as the eight tokens up to the sequence's end, whose first `skip` count for nothing.  (Behind the end
  // they would meet the last state, and an infinite one times their step of 0 is no number.)
  const int skip_last = last >= w.first ? last + TB - w.live : 0;
  ScanStage<N, IO> rows(w, a, last);
  const ScanRows<N, IO> u(w, a.u, a.us), delta(w, a.delta, a.ds), z(w, gated ? a.z : a.u, gated ? a.zs : a.us), dy(w, a.dy, a.ys);
  const ScanRows<N, IO> du_(w, MAP ? a.u : a.du, MAP ? a.us : a.dus), ddelta_(w, MAP ? a.u : a.ddelta, MAP ? a.us : a.dds),
      dz_(w, MAP || !gated ? a.u : a.dz, MAP || !gated ? a.us : a.dzs);
  // what a block reads is on its way while the one behind it is worked on
  Pair<IO> next_u[OWN] = {}, next_delta[OWN] = {}, next_z[OWN] = {}, next_dy[OWN] = {};
  f4 next_h = {};
  const auto fetch = [&](int t0, int skip) {      // the blocks one after the other
    u.load(next_u, w, t0, skip);
    delta.load(next_delta, w, t0, skip);
    dy.load(next_dy, w, t0, skip);
    if (gated) z.load(next_z, w, t0, skip);
    rows.load_behind(skip);
    rows.template go<true>();
    if (!MAP) next_h = *reinterpret_cast<const f4*>(a.kept + ((static_cast<size_t>(w.b) * a.blocks + t0 / TB) * a.n + w.c) * N + 4 * w.q);
  };
  if (last >= w.first) fetch(last, skip_last);
  // (Results stored a block later, as in the forward pass, gain nothing here: backward pass of 8 x 2048 tokens of 4096 channels of 16 states 879 -> 896 us, of
  // 2048 of 32 960 -> 968, of 1024 of 64 1107 -> 1112.)
  constexpr int PARTS = (TB * 2 * N + 64 * W - 1) / (64 * W);
  int turn = 0, skip = skip_last;
  for (int t0 = last; t0 >= w.first; t0 -= TB) {
    f2 x[OWN], raw[OWN], v[OWN], sig[OWN], d[OWN], dt_[OWN], e_[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      const bool in = w.own(k) >= skip && w.here2;
      x[k] = wide2(next_u[k]);
      raw[k] = wide2(next_delta[k]) + bias;
      v[k] = wide2(next_z[k]);
      d[k] = wide2(next_dy[k]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sig[k][j] = sigmoid(v[k][j]);
        const float dt = a.softplus ? softplus(raw[k][j]) : raw[k][j], e = gated ? d[k][j] * v[k][j] * sig[k][j] : d[k][j];
        dt_[k][j] = in ? dt : 0.0f;
        e_[k][j] = in ? e : 0.0f;
        if (w.lane < TB * P::PAIRS) steps[w.wave][w.own(k)][2 * w.pair + j] = f4{dt_[k][j], in ? dt * x[k][j] : 0.0f, e_[k][j], 0.0f};
      }
    }
    rows.put(mine, rows.t >= skip);
    f4 h = next_h;
    if (t0 - TB >= w.first) fetch(t0 - TB, 0);
    wave_fence();
    if constexpr (MAP) {
#pragma unroll
      for (int t = TB - 1; t >= 0; --t) {
        const f4 s = step[t * P::CW + w.in_wave];
        const f4 C = *reinterpret_cast<const f4*>(mine + t * 2 * N + N + 4 * w.q);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = fmaf(s[2], C[i], g[i]) * __builtin_amdgcn_exp2f(s[0] * A2[i]);
        sum_dt += s[0];
      }
      wave_fence();
    } else {
      float* const own_sums = sums[turn][w.wave][0];
      f4 decay[TB], decayed[TB];   // a, a h_{t-1}
      float p[2][8], half[2], some[2][4], y[TURNS] = {}, through[TURNS] = {}, rate[TURNS] = {};
      // the operands of a token are on their way from LDS while the one before it is worked on; more of them would not fit
      f4 s_[2], B_[2], C_[2];
      const auto operands = [&](int t) {
        s_[t % 2] = step[t * P::CW + w.in_wave];
        B_[t % 2] = *reinterpret_cast<const f4*>(mine + t * 2 * N + 4 * w.q);
        C_[t % 2] = *reinterpret_cast<const f4*>(mine + t * 2 * N + N + 4 * w.q);
      };
      operands(0);
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        if (t + 1 < TB) operands(t + 1);
        const f4 s = s_[t % 2], B = B_[t % 2], C = C_[t % 2];
        float read = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          decay[t][i] = __builtin_amdgcn_exp2f(s[0] * A2[i]);
          decayed[t][i] = decay[t][i] * h[i];
          h[i] = fmaf(s[1], B[i], decayed[t][i]);
          read = i == 0 ? C[0] * h[0] : fmaf(C[i], h[i], read);
          p[t / 2 % 2][t % 2 * 4 + i] = s[2] * h[i];
        }
        keep_sum<LN>(read, some[0], y, t, t % LN == LN - 1, w.q);
        // the sums of the pair of tokens before lie between the work on this one
        if (t % 2 == 0 && t > 0) wave_sums<LN>(p[(t / 2 - 1) % 2], half, t / 2 % 2 == 0, t / 2 - 1, own_sums + N, 2 * N, w.lane);
        if (t % 2) __builtin_amdgcn_sched_barrier(0);
      }
      wave_sums<LN>(p[1], half, true, TB / 2 - 1, own_sums + N, 2 * N, w.lane);
#pragma unroll
      for (int t = TB - 1; t >= 0; --t) {
        if (t > 0) operands(t - 1);
        const f4 s = s_[t % 2], B = B_[t % 2], C = C_[t % 2];
        float sum_p = 0.0f, sum_r = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[i] = fmaf(s[2], C[i], g[i]);
          sum_p = i == 0 ? g[0] * B[0] : fmaf(g[i], B[i], sum_p);
          p[t / 2 % 2][t % 2 * 4 + i] = g[i] * s[1];
          const float m = g[i] * decayed[t][i];
          sum_r = i == 0 ? m * A2[0] : fmaf(m, A2[i], sum_r);
          dA[i] = fmaf(m, s[0], dA[i]);
          g[i] *= decay[t][i];
        }
        keep_sum<LN>(sum_p, some[0], through, t, t % LN == 0, w.q);
        keep_sum<LN>(sum_r, some[1], rate, t, t % LN == 0, w.q);
        if (t % 2 && t < TB - 1) wave_sums<LN>(p[(t / 2 + 1) % 2], half, t / 2 % 2 == 1, t / 2 + 1, own_sums, 2 * N, w.lane);
        if (t % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      }
      wave_sums<LN>(p[0], half, true, 0, own_sums, 2 * N, w.lane);
      wave_fence();
#pragma unroll
      for (int k = 0; k < TURNS; ++k) {
        if (LN <= TB || w.q < TB) step[(LN * k + w.q) * P::CW + w.in_wave] = f4{y[k], through[k], rate[k], 0.0f};
      }
      wave_fence();
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        const bool in = w.own(k) >= skip;
        f2 du, ddelta, dz;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f4 sum = step[w.own(k) * P::CW + 2 * w.pair + j];
          // (without D its terms are left out: 0 times an infinite number would be none)
          const float inner = a.D != nullptr ? fmaf(D[j], x[k][j], sum[0]) : sum[0], slope = a.softplus ? sigmoid(raw[k][j]) : 1.0f;
          du[j] = dt_[k][j] * sum[1];
          if (a.D != nullptr) du[j] = fmaf(D[j], e_[k][j], du[j]);
          du[j] = in ? du[j] : 0.0f;
          ddelta[j] = in ? fmaf(x[k][j], sum[1], kLn2 * sum[2]) * slope : 0.0f;
          dz[j] = in ? d[k][j] * inner * sig[k][j] * fmaf(v[k][j], 1.0f - sig[k][j], 1.0f) : 0.0f;
          dD[j] += in ? e_[k][j] * x[k][j] : 0.0f;
          dbias[j] += ddelta[j];
        }
        if (w.here2 && in) {
          du_.store(du_.row(t0 - skip), k, narrow2<IO>(du));
          ddelta_.store(ddelta_.row(t0 - skip), k, narrow2<IO>(ddelta));
          if (gated) dz_.store(dz_.row(t0 - skip), k, narrow2<IO>(dz));
        }
      }
      // dB and dC of the workgroup's channels: the waves in their order
      __syncthreads();
      float of_all[PARTS];
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int i = threadIdx.x + j * 64 * W;
        of_all[j] = 0.0f;
        if (TB * 2 * N >= 64 * W || i < TB * 2 * N) {
#pragma unroll
          for (int o = 0; o < W; ++o) of_all[j] += sums[turn][o][i / (2 * N)][i % (2 * N)];
        }
      }
      float* const to = a.dBC_part + ((static_cast<long long>(w.tile) * a.nb + w.b) * a.T + t0 - skip) * 2 * N;
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int i = threadIdx.x + j * 64 * W;
        if (i < TB * 2 * N && i / (2 * N) >= skip) to[i] = of_all[j];
      }
      turn ^= 1;
    }
    skip = 0;
  }
  if constexpr (MAP) {
    if (!w.here) return;
    *reinterpret_cast<f4*>(a.seg_h + of_seg * N + 4 * w.q) = g;
    if (w.q == 0) a.seg_dt[of_seg] = sum_dt;
  } else {
    for (int t0 = max(w.live, w.first); t0 < w.last; t0 += TB) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        if (w.here2 && t0 + w.own(k) < w.last) {
          const Pair<IO> zero = {};
          du_.store(du_.row(t0), k, zero);
          ddelta_.store(ddelta_.row(t0), k, zero);
          if (gated) dz_.store(dz_.row(t0), k, zero);
        }
      }
    }
    if (w.here) {
      *reinterpret_cast<f4*>(a.dA_part + of_seg * N + 4 * w.q) = dA;
      if (w.seg == 0 && a.dh0 != nullptr) *reinterpret_cast<f4*>(a.dh0 + state) = g;
    }
    // the lanes of a pair of channels: every PAIRS-th one
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float* const all = sums[0][w.wave][0];      // room for two numbers a lane: 16 N
      __syncthreads();
      all[w.lane] = w.here2 ? dD[j] : 0.0f;
      all[64 + w.lane] = w.here2 ? dbias[j] : 0.0f;
      wave_fence();
      if (w.lane < P::PAIRS && w.here2) {
        float total_D = 0.0f, total_bias = 0.0f;
        for (int l = w.lane; l < 64 && l < TB * P::PAIRS; l += P::PAIRS) {
          total_D += all[l];
          total_bias += all[64 + l];
        }
        const size_t at = (static_cast<size_t>(w.b) * a.n_seg + w.seg) * a.n + w.c2 + j;
        a.dD_part[at] = total_D;
        a.dbias_part[at] = total_bias;
      }
    }
  }
}

// dB and dC: the sums over a group's tiles, in their order.  Bound by memory; four states a thread.
constexpr int kThreads = 256;
template <typename IO>
__global__ void __launch_bounds__(kThreads) shared_kernel(ScanArgs a, int N) {
  const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, pieces = N / 4;
  const long long rest = i / pieces, s = i % pieces * 4, row = rest / a.G, g = rest % a.G;
  if (row >= static_cast<long long>(a.nb) * a.T) return;
  const int b = static_cast<int>(row / a.T), t = static_cast<int>(row % a.T);
  f4 B = {0.0f, 0.0f, 0.0f, 0.0f}, C = B;
  if (t < (a.lengths == nullptr ? a.T : min(a.lengths[b], a.T))) {
    const float* from = a.dBC_part + ((g * a.tiles * a.nb + b) * a.T + t) * 2 * N + s;
#pragma unroll 4
    for (int k = 0; k < a.tiles; ++k) {
      const float* p = from + static_cast<size_t>(k) * a.nb * a.T * 2 * N;
      B += *reinterpret_cast<const f4*>(p);
      C += *reinterpret_cast<const f4*>(p + N);
    }
  }
  const size_t at = (static_cast<size_t>(row) * a.G + g) * N + s;
  const float x[4] = {B[0], B[1], B[2], B[3]}, y[4] = {C[0], C[1], C[2], C[3]};
  store_piece(static_cast<IO*>(a.dB) + at, x);
  store_piece(static_cast<IO*>(a.dC) + at, y);
}

template <int N, typename IO>
hipError_t launch(const ScanArgs& a, bool map, hipStream_t stream) {
  const long long groups = static_cast<long long>(a.nb) * a.n_seg * a.G * a.tiles;
  ScanArgs args = a;
  void* params[] = {&args};
  const void* kernel = map ? reinterpret_cast<const void*>(&backward_kernel<N, IO, true>) : reinterpret_cast<const void*>(&backward_kernel<N, IO, false>);
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

hipError_t launch_selective_backward(const ScanArgs& a, int N, int io_dtype, bool map, hipStream_t stream) {
  return io_dtype == 1 ? launch_states<uint16_t>(a, N, map, stream) : launch_states<float>(a, N, map, stream);
}

hipError_t launch_selective_shared(const ScanArgs& a, int N, int io_dtype, hipStream_t stream) {
  const long long items = static_cast<long long>(a.nb) * a.T * a.G * (N / 4);
  if (items == 0) return hipSuccess;
  ScanArgs args = a;
  void* params[] = {&args, &N};
  const void* kernel = io_dtype == 1 ? reinterpret_cast<const void*>(&shared_kernel<uint16_t>) : reinterpret_cast<const void*>(&shared_kernel<float>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>((items + kThreads - 1) / kThreads)), dim3(kThreads), params, 0, stream);
}

}  // namespace vla

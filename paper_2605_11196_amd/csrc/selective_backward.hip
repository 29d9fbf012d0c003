// Gradients of the selective state space scan.
//
//   e = dy z sigmoid(z);  g_t[c,s] = e_t[c] C_t[s] + a_{t+1}[c,s] g_{t+1}[c,s], a = exp(dt A), behind the last token dh_T
//   dC_t[s] = sum_c e_t[c] h_t[c,s];  dB_t[s] = sum_c g_t[c,s] dt_t[c] u_t[c];  with p = sum_s g B:  du = D e + dt p
//   ddt = sum_s g a h_{t-1} A + u p;  dA[c,s] = sum_t g a h_{t-1} dt;  dD = sum e u;  dh0 = a_1 g_1;  dz from y before the gate
//
// Bound by vector instructions, as the forward pass.  A lane holds NS states of CH neighbouring channels, a workgroup of N / NS waves all states of 64 CH
// channels (four states of two channels; for N = 64, where that would be 16 waves, eight of one).  Blocks of eight tokens from the last to the
// first: from the state that the forward pass has kept before the block the products a h_{t-1} of its tokens are formed again and stay on registers,
// then g goes back through them.  dB and dC are sums over channels: the two of a lane are added on the way, those of a wave by a
// transposition in LDS, eight numbers at a time, and those of the tiles by a second kernel; sums over states are added up over the waves in LDS.
// Time segments as in the forward pass, from the last to the first.
//
// The kernel keeps to registers that no copy has to stand in for (the tests hold it to that): with more live values than fit, the compiler keeps addresses in
// accumulation registers over the loop, and writes them behind a divergent branch before it has turned the lanes on again.  So there is no divergent
// branch between the loads of a block and its end, and the tokens' work is kept apart (sched_barrier), without which their loads are drawn together.
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int TB = kScanBlock;
constexpr int kAtOnce = 8;         // numbers of a lane that are summed over the lanes together
constexpr int kRow = kAtOnce + 4;   // floats of a lane's row of the transposition: 16-byte aligned, rows of eight lanes on different banks

__device__ __forceinline__ int length_of(const int* lengths, int b, int T) { return lengths == nullptr ? T : min(max(lengths[b], 0), T); }

// Sums of p[0..7] over the lanes; lane l gets that of p[l % 8].
__device__ __forceinline__ float lane_sums(const float (&p)[kAtOnce], float* rows, int lane) {
  *reinterpret_cast<f4*>(rows + lane * kRow) = f4{p[0], p[1], p[2], p[3]};
  *reinterpret_cast<f4*>(rows + lane * kRow + 4) = f4{p[4], p[5], p[6], p[7]};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const float* from = rows + (lane / 8) * kRow + lane % 8;
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) s += from[8 * k * kRow];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return swap32_sum(swap16_sum(dpp_sum<0x128>(s)));
}

// A lane's channels as they lie in memory and as numbers
template <int CH, typename IO> struct Lanes;
template <typename IO> struct Lanes<2, IO> {
  typedef Pair<IO> raw;
  static __device__ __forceinline__ raw load(const IO* p) { return raw2(p); }
  static __device__ __forceinline__ void widen(raw x, float (&v)[2]) {
    const f2 w = wide2(x);
    v[0] = w[0];
    v[1] = w[1];
  }
  static __device__ __forceinline__ void store(IO* p, const float (&v)[2]) { store2(p, f2{v[0], v[1]}); }
};
template <typename IO> struct Lanes<1, IO> {
  typedef IO raw;
  static __device__ __forceinline__ raw load(const IO* p) { return *p; }
  static __device__ __forceinline__ void widen(float x, float (&v)[1]) { v[0] = x; }
  static __device__ __forceinline__ void widen(uint16_t x, float (&v)[1]) { v[0] = bf16_to_f32(x); }
  static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[1]) { *p = f32_to_bf16_rne(v[0]); }
};
template <int CH> struct Vec { float v[CH]; };

template <int N, int NS, int CH, typename IO, bool MAP>
__global__ void __launch_bounds__(64 * (N / NS)) __attribute__((amdgpu_waves_per_eu(2))) backward_kernel(ScanArgs a) {
  constexpr int W = N / NS, PER = TB / W, TILE = 64 * CH;
  static_assert(PER >= 1, "every wave has tokens of a block");
  typedef Lanes<CH, IO> L;
  __shared__ Vec<2 * CH> steps[TB][64];         // dt, dt u of a lane's channels
  __shared__ Vec<CH> grads[TB][64];             // e
  __shared__ __align__(16) float rows[TB][2 * N];   // B, C
  __shared__ Vec<2 * CH> part[MAP ? 1 : W][TB][64];   // p, sum_s g a h A of the channels
  __shared__ Vec<CH> part_y[MAP ? 1 : W][TB][64];
  __shared__ __align__(16) float turned[MAP ? 1 : W][64 * kRow];
  const unsigned tiles = a.G * a.tiles;
  const int tile = blockIdx.x % tiles;
  const unsigned rest = blockIdx.x / tiles;
  const int seg = rest % a.n_seg, b = rest / a.n_seg, group = tile / a.tiles;
  const int of_group = a.n / a.G, c_first = tile % a.tiles * TILE, there = min(of_group - c_first, TILE) / CH;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int length = length_of(a.lengths, b, a.T);
  const bool here = lane < there;
  const int c = group * of_group + c_first + (here ? CH * lane : 0);
  const IO* u = static_cast<const IO*>(a.u) + b * a.us.b + c;
  const IO* delta = static_cast<const IO*>(a.delta) + b * a.ds.b + c;
  const bool gated = a.z != nullptr;
  const IO* z = gated ? static_cast<const IO*>(a.z) + b * a.zs.b + c : u;     // without a gate something that can be read
  const long long z_t = gated ? a.zs.t : a.us.t;
  const IO* dy = static_cast<const IO*>(a.dy) + b * a.ys.b + c;
  // the values of B and C that this thread stages for a block
  constexpr int STAGE = TB * 2 * N / (64 * W);
  static_assert(STAGE * 64 * W == TB * 2 * N, "as many for each");

  float A2[CH][NS], g[CH][NS], dA[CH][NS];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const size_t at = static_cast<size_t>(c + j) * N + wave * NS;
    const float* behind = MAP ? nullptr
                          : a.n_seg > 1 ? a.seg_h + (static_cast<size_t>(b) * a.n_seg + seg) * a.n * N + at
                          : a.dh_T != nullptr ? a.dh_T + static_cast<size_t>(b) * a.n * N + at : nullptr;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      A2[j][i] = a.A[at + i] * kLog2e;
      g[j][i] = behind != nullptr ? behind[i] : 0.0f;
      dA[j][i] = 0.0f;
    }
  }
  float bias[CH], D[CH], sum_dt[CH], dD[CH], dbias[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    bias[j] = a.bias != nullptr ? a.bias[c + j] : 0.0f;
    D[j] = a.D != nullptr ? a.D[c + j] : 0.0f;
    sum_dt[j] = dD[j] = dbias[j] = 0.0f;
  }

  const int first = seg * a.seg_blocks, last = min(first + a.seg_blocks, (a.T + TB - 1) / TB);
  const int live = min(last, (length + TB - 1) / TB);
  for (int block = live - 1; block >= first; --block) {
    typename L::raw raw_u[PER], raw_delta[PER], raw_z[PER], raw_dy[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const long long t = min(block * TB + wave * PER + k, length - 1);
      raw_u[k] = L::load(u + t * a.us.t);
      raw_delta[k] = L::load(delta + t * a.ds.t);
      raw_dy[k] = L::load(dy + t * a.ys.t);
      raw_z[k] = L::load(z + t * z_t);
    }
    IO raw_row[STAGE];
#pragma unroll
    for (int k = 0; k < STAGE; ++k) {
      const int at = threadIdx.x + k * 64 * W, t = at / (2 * N), col = at % (2 * N);
      const bool is_c = col >= N;
      const IO* from = is_c ? static_cast<const IO*>(a.Cm) + b * a.C_b + group * a.C_g + (col - N)
                            : static_cast<const IO*>(a.Bm) + b * a.B_b + group * a.B_g + col;
      raw_row[k] = from[min(block * TB + t, length - 1) * (is_c ? a.C_t : a.B_t)];
    }
    float h[CH][NS];
    if (!MAP) {
      // where the forward pass has put them: eight states of a pair of 128 channels' on a lane, four at a time
      constexpr int PAIRS = kScanTile / 2;
      const int in_group = c_first + (here ? CH * lane : 0);        // channel of the group
      const unsigned all = a.G * ((of_group + kScanTile - 1) / kScanTile);
      const unsigned at_tile = group * ((of_group + kScanTile - 1) / kScanTile) + in_group / kScanTile;
      const f4* from = reinterpret_cast<const f4*>(a.kept) +
                       (((static_cast<size_t>(b) * a.blocks + block) * all + at_tile) * (N / 8) + wave * NS / 8) * 4 * PAIRS + in_group % kScanTile / 2;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
#pragma unroll
        for (int i = 0; i < NS; i += 4) {
          const int channel = CH == 1 ? in_group % 2 : j;
          const f4 x = from[(2 * channel + (wave * NS + i) % 8 / 4) * PAIRS];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[j][i + k] = x[k];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int t = block * TB + wave * PER + k;
      const bool in = t < length && here;
      float x[CH], raw[CH], e[CH], v[CH];
      L::widen(raw_u[k], x);
      L::widen(raw_delta[k], raw);
      L::widen(raw_dy[k], e);
      L::widen(raw_z[k], v);
      Vec<2 * CH> s;
      Vec<CH> w;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const float r = raw[j] + bias[j], d = a.softplus ? softplus(r) : r, gate = v[j] * sigmoid(v[j]);
        s.v[2 * j] = in ? d : 0.0f;
        s.v[2 * j + 1] = in ? d * x[j] : 0.0f;
        w.v[j] = in ? (gated ? e[j] * gate : e[j]) : 0.0f;
      }
      steps[wave * PER + k][lane] = s;
      grads[wave * PER + k][lane] = w;
    }
#pragma unroll
    for (int k = 0; k < STAGE; ++k) {
      const int at = threadIdx.x + k * 64 * W, t = at / (2 * N);
      float x[1];
      Lanes<1, IO>::widen(raw_row[k], x);
      rows[t][at % (2 * N)] = block * TB + t < length ? x[0] : 0.0f;
    }
    __syncthreads();
    if constexpr (MAP) {
#pragma unroll
      for (int t = TB - 1; t >= 0; --t) {
        const Vec<2 * CH> s = steps[t][lane];
        const Vec<CH> e = grads[t][lane];
        const f4* Ct = reinterpret_cast<const f4*>(&rows[t][N + wave * NS]);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
#pragma unroll
          for (int j = 0; j < CH; ++j) g[j][i] = fmaf(e.v[j], Ct[i / 4][i % 4], g[j][i]) * __builtin_amdgcn_exp2f(s.v[2 * j] * A2[j][i]);
        }
        if (wave == 0) {
#pragma unroll
          for (int j = 0; j < CH; ++j) sum_dt[j] += s.v[2 * j];
        }
      }
      __syncthreads();
    } else {
      float decayed[TB][CH][NS];   // a h_{t-1}
      float sums_C = 0.0f, sums_B = 0.0f;
      float p[kAtOnce];
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const Vec<2 * CH> s = steps[t][lane];
        const Vec<CH> e = grads[t][lane];
        const f4* Bt = reinterpret_cast<const f4*>(&rows[t][wave * NS]);
        const f4* Ct = reinterpret_cast<const f4*>(&rows[t][N + wave * NS]);
        Vec<CH> y{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          float along = 0.0f;
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            decayed[t][j][i] = __builtin_amdgcn_exp2f(s.v[2 * j] * A2[j][i]) * h[j][i];
            h[j][i] = fmaf(s.v[2 * j + 1], Bt[i / 4][i % 4], decayed[t][j][i]);
            y.v[j] = fmaf(Ct[i / 4][i % 4], h[j][i], y.v[j]);
            along = j == 0 ? e.v[0] * h[0][i] : fmaf(e.v[j], h[j][i], along);
          }
          p[t * NS % kAtOnce + i] = along;
        }
        part_y[wave][t][lane] = y;
        if ((t + 1) * NS % kAtOnce == 0) {
          const float total = lane_sums(p, turned[wave], lane);
          sums_C = lane / kAtOnce == t * NS / kAtOnce ? total : sums_C;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = TB - 1; t >= 0; --t) {
        const Vec<2 * CH> s = steps[t][lane];
        const Vec<CH> e = grads[t][lane];
        const f4* Bt = reinterpret_cast<const f4*>(&rows[t][wave * NS]);
        const f4* Ct = reinterpret_cast<const f4*>(&rows[t][N + wave * NS]);
        Vec<2 * CH> sum{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          float along = 0.0f;
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            g[j][i] = fmaf(e.v[j], Ct[i / 4][i % 4], g[j][i]);
            sum.v[j] = fmaf(g[j][i], Bt[i / 4][i % 4], sum.v[j]);
            const float m = g[j][i] * decayed[t][j][i];
            sum.v[CH + j] = fmaf(m, A2[j][i], sum.v[CH + j]);
            dA[j][i] = fmaf(m, s.v[2 * j], dA[j][i]);
            along = j == 0 ? g[0][i] * s.v[1] : fmaf(g[j][i], s.v[2 * j + 1], along);
            g[j][i] *= __builtin_amdgcn_exp2f(s.v[2 * j] * A2[j][i]);
          }
          p[t * NS % kAtOnce + i] = along;
        }
        part[wave][t][lane] = sum;
        if (t * NS % kAtOnce == 0) {
          const float total = lane_sums(p, turned[wave], lane);
          sums_B = lane / kAtOnce == t * NS / kAtOnce ? total : sums_B;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      {
        const int t = block * TB + lane / NS;      // eight numbers: kAtOnce / NS tokens
        if (t < length && lane < TB * NS) {
          float* to = a.dBC_part + ((static_cast<size_t>(tile) * a.nb + b) * a.T + t) * 2 * N + wave * NS + lane % NS;
          to[0] = sums_B;
          to[N] = sums_C;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int i = wave * PER + k, t = block * TB + i;
        const long long tl = min(t, length - 1);
        float x[CH], raw[CH], v[CH], d[CH];
        L::widen(L::load(u + tl * a.us.t), x);
        L::widen(L::load(delta + tl * a.ds.t), raw);
        L::widen(L::load(z + tl * z_t), v);
        L::widen(L::load(dy + tl * a.ys.t), d);
        const Vec<2 * CH> s = steps[i][lane];
        const Vec<CH> e = grads[i][lane];
        Vec<2 * CH> sum{};
        Vec<CH> y{};
#pragma unroll
        for (int o = 0; o < W; ++o) {
          const Vec<2 * CH> q = part[o][i][lane];
          const Vec<CH> r = part_y[o][i][lane];
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            sum.v[j] += q.v[j];
            sum.v[CH + j] += q.v[CH + j];
            y.v[j] += r.v[j];
          }
        }
        const bool in = t < length;
        float du[CH], ddelta[CH], dz[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const float inner = fmaf(D[j], x[j], y.v[j]), sig = sigmoid(v[j]);
          const float slope = a.softplus ? sigmoid(raw[j] + bias[j]) : 1.0f;
          du[j] = in ? fmaf(D[j], e.v[j], s.v[2 * j] * sum.v[j]) : 0.0f;
          ddelta[j] = in ? fmaf(x[j], sum.v[j], kLn2 * sum.v[CH + j]) * slope : 0.0f;
          dz[j] = in ? d[j] * inner * sig * fmaf(v[j], 1.0f - sig, 1.0f) : 0.0f;
          dD[j] += in ? e.v[j] * x[j] : 0.0f;
          dbias[j] += ddelta[j];
        }
        if (here && t < a.T) {
          L::store(static_cast<IO*>(a.du) + b * a.dus.b + t * a.dus.t + c, du);
          L::store(static_cast<IO*>(a.ddelta) + b * a.dds.b + t * a.dds.t + c, ddelta);
          if (gated) L::store(static_cast<IO*>(a.dz) + b * a.dzs.b + t * a.dzs.t + c, dz);
        }
      }
    }
  }
  if constexpr (MAP) {
    if (here) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        float* to = a.seg_h + (static_cast<size_t>(b) * a.n_seg + seg) * a.n * N + static_cast<size_t>(c + j) * N + wave * NS;
#pragma unroll
        for (int i = 0; i < NS; i += 4) *reinterpret_cast<f4*>(to + i) = f4{g[j][i], g[j][i + 1], g[j][i + 2], g[j][i + 3]};
        if (wave == 0) a.seg_dt[(static_cast<size_t>(b) * a.n_seg + seg) * a.n + c + j] = sum_dt[j];
      }
    }
  } else {
    for (int t = max(first, live) * TB + wave; t < min(last * TB, a.T); t += W) {
      const float zero[CH] = {};
      if (here) {
        L::store(static_cast<IO*>(a.du) + b * a.dus.b + t * a.dus.t + c, zero);
        L::store(static_cast<IO*>(a.ddelta) + b * a.dds.b + t * a.dds.t + c, zero);
        if (gated) L::store(static_cast<IO*>(a.dz) + b * a.dzs.b + t * a.dzs.t + c, zero);
      }
    }
    __syncthreads();      // the last block's parts have been read
    Vec<2 * CH> both;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      both.v[j] = dD[j];
      both.v[CH + j] = dbias[j];
    }
    part[wave][0][lane] = both;
    __syncthreads();
    if (!here) return;
    const size_t of_seg = static_cast<size_t>(b) * a.n_seg + seg;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const size_t at = static_cast<size_t>(c + j) * N + wave * NS;
#pragma unroll
      for (int i = 0; i < NS; i += 4) {
        *reinterpret_cast<f4*>(a.dA_part + of_seg * a.n * N + at + i) = f4{dA[j][i], dA[j][i + 1], dA[j][i + 2], dA[j][i + 3]};
        if (seg == 0 && a.dh0 != nullptr) {
          *reinterpret_cast<f4*>(a.dh0 + static_cast<size_t>(b) * a.n * N + at + i) = f4{g[j][i], g[j][i + 1], g[j][i + 2], g[j][i + 3]};
        }
      }
    }
    if (wave != 0) return;
    Vec<2 * CH> total{};
#pragma unroll
    for (int o = 0; o < W; ++o) {
      const Vec<2 * CH> q = part[o][0][lane];
#pragma unroll
      for (int j = 0; j < 2 * CH; ++j) total.v[j] += q.v[j];
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      a.dD_part[of_seg * a.n + c + j] = total.v[j];
      a.dbias_part[of_seg * a.n + c + j] = total.v[CH + j];
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
  if (t < length_of(a.lengths, b, a.T)) {
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

template <int N, int NS, int CH, typename IO>
hipError_t launch(const ScanArgs& a, bool map, hipStream_t stream) {
  const long long groups = static_cast<long long>(a.nb) * a.n_seg * a.G * a.tiles;
  ScanArgs args = a;
  void* params[] = {&args};
  const void* kernel = map ? reinterpret_cast<const void*>(&backward_kernel<N, NS, CH, IO, true>)
                           : reinterpret_cast<const void*>(&backward_kernel<N, NS, CH, IO, false>);
  return hipLaunchKernel(kernel, dim3(static_cast<unsigned>(groups)), dim3(64 * (N / NS)), params, 0, stream);
}
template <typename IO>
hipError_t launch_states(const ScanArgs& a, int N, bool map, hipStream_t stream) {
  switch (N) {
    case 8: return launch<8, 4, 2, IO>(a, map, stream);
    case 16: return launch<16, 4, 2, IO>(a, map, stream);
    case 32: return launch<32, 4, 2, IO>(a, map, stream);
    case 64: return launch<64, 8, 1, IO>(a, map, stream);
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

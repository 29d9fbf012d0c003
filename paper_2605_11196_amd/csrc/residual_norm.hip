// The norms around a block with its gate and its residual: what follows a block and what precedes the next one, in one pass over a row.
//
//   t = N(y) w1 act(gate) k,  N(y) = y r1, r1 = 1 / sqrt(mean y^2 + eps) over each group of columns;  s = x + t;
//   h = s r2 w2, r2 = 1 / sqrt(mean s^2 + eps) over the row;  any of x, w1 (with N), gate, k, w2 (with h) may be missing
//   backward: d = ds + r2 (dh w2 - s r2^2 mean(dh w2 s)) = dx;  c = d k act w1;  dy = r1 (c - N(y) mean(c N(y)));
//   dgate = d k N(y) w1 act'(gate);  dw1 = sum d k act N(y), dk = sum d act w1 N(y), dw2 = sum dh s r2 over the rows
//
// Bound by memory: every operand is read once and every result written once (the backward pass forms t, s and the two norms again from x,
// y and gate, which it has to read anyway; s is float32 in both).  A row lies on L lanes, from 8 to 1024, with eight neighbouring columns
// each; a workgroup goes through rows.  Sums go through DPP and lane swaps, and over the waves of a row through LDS and DPP again.  What decides is
// how much a compute unit has on its way, and how soon it asks for the next row (32768 rows of 4096 in bf16, all operands given): all operands of a row are
// asked for before the first is used (backward 604 -> 514 us, forward 327 -> 300), the backward pass keeps its weights in LDS rather than on
// registers beside their gradients (683 -> 604), no workgroup waits for a place (forward 295 -> 269), and the waves' sums are added by lanes
// and not by a loop (540 -> 465, 269 -> 264).  A row that fills its workgroup is numbered by the block alone, which takes the addresses
// off the vector registers.  Asking for the next row ahead was tried: 139 registers in the backward pass and one workgroup, 905 us.  5.1 TB/s
// forward and 4.6 backward, where a copy reaches 4.9.  That holds for the row's norm and for groups of a power of two of columns up to 512, whose sums stay in a
// wave.  Other groups are added up from LDS by every lane for itself: 80 to 320 columns 2.9 to 5 TB/s forward and 1.7 to 3.3 backward in bfloat16, two groups of
// 1024 columns 1.5 and 1.1, of 4096 0.4 and 0.3.
#include "mixer_util.h"

namespace vla {
namespace {

constexpr int kColumns = 8;   // of a lane, together

struct Eight {
  float v[kColumns];
  __device__ __forceinline__ float& operator[](int i) { return v[i]; }
  __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
// as they lie in memory: a row's operands are all asked for before the first one is widened, which waits for it
template <typename IO>
struct Raw8 {
  Piece<IO> p[kColumns / kPiece<IO>];
};
template <typename IO>
__device__ __forceinline__ Raw8<IO> raw8(const IO* p) {
  Raw8<IO> r;
#pragma unroll
  for (int i = 0; i < kColumns / kPiece<IO>; ++i) r.p[i] = load_piece(p + i * kPiece<IO>);
  return r;
}
template <typename IO>
__device__ __forceinline__ Eight wide8(const Raw8<IO>& r) {
  Eight e;
#pragma unroll
  for (int i = 0; i < kColumns; ++i) e[i] = r.p[i / kPiece<IO>][i % kPiece<IO>];
  return e;
}
template <typename IO> __device__ __forceinline__ Eight load8(const IO* p) { return wide8(raw8(p)); }
// Eight weights of either type; ones where there are none.  Asked for first and widened later, as above.
struct RawWeight {
  f4 lo, hi;
  __device__ __forceinline__ RawWeight(const void* w, int bf16, int c) : lo{1.0f, 1.0f, 1.0f, 1.0f}, hi{1.0f, 1.0f, 1.0f, 1.0f} {
    if (w == nullptr) return;
    if (!bf16) hi = *reinterpret_cast<const f4*>(static_cast<const float*>(w) + c + 4);
    lo = *reinterpret_cast<const f4*>(static_cast<const char*>(w) + static_cast<size_t>(c) * (bf16 ? 2 : 4));
  }
  __device__ __forceinline__ Eight wide(const void* w, int bf16) const {
    if (w == nullptr || !bf16) return Eight{{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
    Eight e;
#pragma unroll
    for (int i = 0; i < kColumns; i += 2) {
      const unsigned two = __float_as_uint(lo[i / 2]);
      e[i] = __uint_as_float(two << 16);
      e[i + 1] = __uint_as_float(two & 0xffff0000u);
    }
    return e;
  }
};
template <typename IO> __device__ __forceinline__ void store8(IO* p, const Eight& e) { store_piece(p, e.v); }

// Where a lane is in its workgroup, and the sums over its row and over its group of columns.  WHOLE: one row fills the workgroup, of three waves or more.
template <bool WHOLE>
struct RowLanes {
  int L, lane, row, rows, pieces, each;   // lanes of a row, this one's place, its row among the workgroup's; eights of a row and of a group
  float* whole;                           // LDS: [4][2][16]
  float* parts;                           // LDS: [2][threads]
  float* weights;                         // LDS: [3][n]
  bool here, split;                       // columns of the row; whether the sums over groups go through LDS

  __device__ __forceinline__ RowLanes(const ResidualArgs& a, int lanes, float* lds) {
    L = lanes;
    lane = threadIdx.x % L;
    row = threadIdx.x / L;
    rows = blockDim.x / L;
    pieces = a.n / kColumns;
    each = a.group / kColumns;
    whole = lds;
    parts = lds + 4 * 2 * 16;
    weights = parts + 2 * blockDim.x;
    here = lane < pieces;
    split = each != pieces && ((each & (each - 1)) != 0 || each > 64);
  }
  // w1, k, w2 as float32
  __device__ __forceinline__ void load_weights(const ResidualArgs& a) const {
    for (int i = threadIdx.x; i < 3 * pieces; i += blockDim.x) {
      const int which = i / pieces, c = i % pieces * kColumns;
      const void* w = which == 0 ? a.post_weight : which == 1 ? a.scale : a.weight;
      store_piece(weights + which * pieces * kColumns + c, RawWeight(w, a.w_bf16, c).wide(w, a.w_bf16).v);
    }
    __syncthreads();
  }
  __device__ __forceinline__ Eight weight(int which, int c) const { return load8(weights + which * pieces * kColumns + c); }
  // a (and b) summed over the row, in every lane of it.  `at`: a place in LDS; between two visits of one place lies the barrier of another.  The sums of
  // the waves are read by 16 lanes and added up like the lanes' own, which is sooner done than a loop over them.
  template <bool TWO>
  __device__ __forceinline__ void row_sums(float& a, float& b, int at) const {
    const int lanes = WHOLE || L > 64 ? 64 : L;
    a = group_sum(a, lanes);
    if (TWO) b = group_sum(b, lanes);
    if (!WHOLE && L <= 64) return;
    const int waves = L / 64, wave = threadIdx.x / 64, of = wave / waves * waves + (threadIdx.x & 15);
    float* slot = whole + at * 2 * 16;
    if ((threadIdx.x & 63) == 0) {
      slot[wave] = a;
      if (TWO) slot[16 + wave] = b;
    }
    __syncthreads();
    const bool in = (threadIdx.x & 15) < waves;
    a = group_sum(in ? slot[of] : 0.0f, 16);
    if (TWO) b = group_sum(in ? slot[16 + of] : 0.0f, 16);
  }
  // a summed over the lane's group
  __device__ __forceinline__ float group_total(float a, int at) const {
    if (each == pieces) {
      float none = 0.0f;
      row_sums<false>(a, none, at);
      return a;
    }
    if (!split) return group_sum(a, each);
    float* slot = parts + (at & 1) * blockDim.x + row * L;
    slot[lane] = a;
    __syncthreads();
    const int first = lane / each * each;
    float sum = 0.0f;
    for (int i = 0; i < each && first + i < L; ++i) sum += slot[first + i];
    return sum;
  }
};

// act(g), and with slope also its derivative
__device__ __forceinline__ float activation(int act, float g) {
  const float s = sigmoid(g);
  return act == 0 ? g * s : s;
}
__device__ __forceinline__ float slope(int act, float g) {
  const float s = sigmoid(g);
  return act == 0 ? s * fmaf(g, 1.0f - s, 1.0f) : s * (1.0f - s);
}

template <typename T>
__device__ __forceinline__ Raw8<T> row8(const void* p, Row2 step, long long b, long long t, int c) {
  return raw8(static_cast<const T*>(p) + b * step.b + t * step.t + c);
}
template <typename T>
__device__ __forceinline__ void row8_store(void* p, Row2 step, long long b, long long t, int c, const Eight& e) {
  store8(static_cast<T*>(p) + b * step.b + t * step.t + c, e);
}

template <typename IO, typename ST, bool WHOLE>
__global__ void __launch_bounds__(WHOLE ? 1024 : 256) residual_kernel(ResidualArgs a, int L) {
  extern __shared__ __align__(16) float lds[];
  const RowLanes<WHOLE> r(a, L, lds);
  const long long total = static_cast<long long>(a.B) * a.T, stride = static_cast<long long>(gridDim.x) * r.rows;
  const int c = r.here ? kColumns * r.lane : 0;
  const int row_here = WHOLE ? 0 : r.row;   // known to be the same for the whole workgroup
  const RawWeight raw1(a.post_weight, a.w_bf16, c), raw_k(a.scale, a.w_bf16, c), raw2(a.weight, a.w_bf16, c);
  const Eight w1 = raw1.wide(a.post_weight, a.w_bf16), k = raw_k.wide(a.scale, a.w_bf16), w2 = raw2.wide(a.weight, a.w_bf16);
  long long first = static_cast<long long>(blockIdx.x) * r.rows;
  int turn = 0;
  for (; first < total; first += stride) {
    const long long n = first + row_here;
    const bool live = n < total && r.here;
    const long long b = n < total ? n / a.T : 0, t = n < total ? n % a.T : 0;
    Raw8<IO> read_y{}, read_g{};
    Raw8<ST> read_x{};
    if (live) {
      if (a.y != nullptr) read_y = row8<IO>(a.y, a.ys, b, t, c);
      if (a.x != nullptr) read_x = row8<ST>(a.x, a.xs, b, t, c);
      if (a.gate != nullptr) read_g = row8<IO>(a.gate, a.gs, b, t, c);
    }
    Eight s = wide8(read_y);
    const Eight x = wide8(read_x), g = wide8(read_g);
    if (a.post_weight != nullptr) {
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < kColumns; ++i) sq = fmaf(s[i], s[i], sq);
      const float r1 = rsqrtf(fmaf(r.group_total(sq, turn), 1.0f / a.group, a.eps));
#pragma unroll
      for (int i = 0; i < kColumns; ++i) s[i] *= r1 * w1[i];
    }
    if (a.gate != nullptr) {
#pragma unroll
      for (int i = 0; i < kColumns; ++i) s[i] *= activation(a.act, g[i]);
    }
    if (a.scale != nullptr) {
#pragma unroll
      for (int i = 0; i < kColumns; ++i) s[i] *= k[i];
    }
    float sum = 0.0f, none = 0.0f;
#pragma unroll
    for (int i = 0; i < kColumns; ++i) {
      s[i] += x[i];
      sum = fmaf(s[i], s[i], sum);
    }
    if (live && a.s != nullptr) row8_store<ST>(a.s, a.ss, b, t, c, s);
    if (a.weight != nullptr) {
      r.template row_sums<false>(sum, none, 2 + turn);
      const float r2 = rsqrtf(fmaf(sum, 1.0f / a.n, a.eps));
#pragma unroll
      for (int i = 0; i < kColumns; ++i) s[i] *= r2 * w2[i];
      if (live) row8_store<IO>(a.h, a.hs, b, t, c, s);
    }
    turn ^= 1;
  }
}

template <typename IO, typename ST, bool WHOLE>
__global__ void __launch_bounds__(WHOLE ? 1024 : 512) residual_backward_kernel(ResidualArgs a, int L) {
  extern __shared__ __align__(16) float lds[];
  const RowLanes<WHOLE> r(a, L, lds);
  const long long total = static_cast<long long>(a.B) * a.T;
  const float inv_n = 1.0f / a.n, inv_group = 1.0f / a.group;
  const int c = r.here ? kColumns * r.lane : 0;
  const int row_here = WHOLE ? 0 : r.row;   // known to be the same for the whole workgroup
  r.load_weights(a);
  Eight dw1{}, dk{}, dw2{};
  long long first = static_cast<long long>(blockIdx.x) * r.rows;
  int turn = 0;
  for (; first < total; first += static_cast<long long>(gridDim.x) * r.rows) {
    const long long n = first + row_here;
    const bool live = n < total && r.here;
    const long long b = n < total ? n / a.T : 0, t = n < total ? n % a.T : 0;
    Raw8<IO> read_y{}, read_g{}, read_dh{};
    Raw8<ST> read_x{}, read_ds{};
    if (live) {
      if (a.y != nullptr) read_y = row8<IO>(a.y, a.ys, b, t, c);
      if (a.x != nullptr) read_x = row8<ST>(a.x, a.xs, b, t, c);
      if (a.gate != nullptr) read_g = row8<IO>(a.gate, a.gs, b, t, c);
      if (a.ds != nullptr) read_ds = row8<ST>(a.ds, a.ss, b, t, c);
      if (a.dh != nullptr) read_dh = row8<IO>(a.dh, a.hs, b, t, c);
    }
    Eight unit = wide8(read_y), s = wide8(read_x), g = wide8(read_g), d = wide8(read_ds);
    const Eight dh = wide8(read_dh);
    float r1 = 1.0f;
    if (a.post_weight != nullptr) {
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < kColumns; ++i) sq = fmaf(unit[i], unit[i], sq);
      r1 = rsqrtf(fmaf(r.group_total(sq, 0), inv_group, a.eps));      // the third sum's barrier lies before the next row's
#pragma unroll
      for (int i = 0; i < kColumns; ++i) unit[i] *= r1;
    }
    if (a.dh != nullptr) {
      asm volatile("" ::: "memory");   // the weights are read here: ahead of the sums they take 24 registers
      const Eight w1 = r.weight(0, c), k = r.weight(1, c), w2 = r.weight(2, c);
      float sq = 0.0f, along = 0.0f;
#pragma unroll
      for (int i = 0; i < kColumns; ++i) {
        float y = unit[i] * w1[i] * k[i];
        if (a.gate != nullptr) y *= activation(a.act, g[i]);
        s[i] += y;
        sq = fmaf(s[i], s[i], sq);
        along = fmaf(dh[i] * w2[i], s[i], along);
      }
      r.template row_sums<true>(sq, along, 2 + turn);
      const float r2 = rsqrtf(fmaf(sq, inv_n, a.eps)), f = along * r2 * r2 * inv_n;
#pragma unroll
      for (int i = 0; i < kColumns; ++i) {
        d[i] = fmaf(r2, fmaf(dh[i], w2[i], -s[i] * f), d[i]);
        dw2[i] = fmaf(dh[i], s[i] * r2, dw2[i]);
      }
    }
    turn ^= 1;
    if (live && a.dx != nullptr) row8_store<ST>(a.dx, a.dxs, b, t, c, d);
    if (a.y == nullptr) continue;
    // d becomes the gradient of N(y)
    asm volatile("" ::: "memory");
    const Eight w1 = r.weight(0, c), k = r.weight(1, c);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kColumns; ++i) {
      const float act = a.gate != nullptr ? activation(a.act, g[i]) : 1.0f;
      const float da = d[i] * act, du = d[i] * unit[i];
      dk[i] = fmaf(da * w1[i], unit[i], dk[i]);
      dw1[i] = fmaf(da * k[i], unit[i], dw1[i]);
      if (a.gate != nullptr) g[i] = du * w1[i] * k[i] * slope(a.act, g[i]);
      d[i] = da * k[i] * w1[i];
      m = fmaf(d[i], unit[i], m);
    }
    if (live && a.dgate != nullptr) row8_store<IO>(a.dgate, a.dgs, b, t, c, g);
    if (a.post_weight != nullptr) {
      const float f = r.group_total(m, 1) * inv_group;
#pragma unroll
      for (int i = 0; i < kColumns; ++i) d[i] = r1 * fmaf(-unit[i], f, d[i]);
    }
    if (live && a.dy != nullptr) row8_store<IO>(a.dy, a.dys, b, t, c, d);
  }
  if (a.sum_part == nullptr) return;
  // the rows of a workgroup, in their order
  float* part = a.sum_part + static_cast<size_t>(blockIdx.x) * 3 * a.n;
  const Eight* all[3] = {&dw2, &dw1, &dk};
  if (WHOLE) {
    if (!r.here) return;
#pragma unroll
    for (int j = 0; j < 3; ++j) store8(part + static_cast<size_t>(j) * a.n + c, *all[j]);
    return;
  }
  float* const rows = r.weights + 3 * a.n;      // LDS: [rows][8 L]
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    __syncthreads();
    store8(rows + kColumns * threadIdx.x, *all[j]);
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
      float sum = 0.0f;
      for (int row = 0; row < r.rows; ++row) sum += rows[row * kColumns * L + i];
      part[static_cast<size_t>(j) * a.n + i] = sum;
    }
  }
}

// Lanes of a row: a power of two up to a wave, whole waves beyond.
int row_width(int n) {
  const int pieces = n / kColumns;
  if (pieces > 64) return (pieces + 63) / 64 * 64;
  int L = 8;
  while (L < pieces) L *= 2;
  return L;
}
// Threads of a workgroup: as many whole rows as four waves hold, or one row (backward: eight waves, as the number of workgroups is held by what they leave of the
// weights' gradients; 87381 rows of 1536 in bfloat16, backward: 784 us with four waves, three of them at work).
int threads_of(int L, bool backward) {
  const int most = backward ? 512 : 256;
  return L < most ? most / L * L : L;
}

// As many as the card's 256 compute units hold at once, 24 waves each (their registers would let in 28, in workgroups of 3 to 16) and 16 in the backward pass: a
// workgroup more would go through its rows when all others have ended (backward pass of 52428 rows of 2560 in bfloat16 with 819 workgroups 993 us, with 768 706).
int workgroups_of(int threads, bool backward) {
  const int held = (backward ? 16 : 24) / (threads / 64);
  return 256 * (held > 0 ? held : 1);
}

template <typename IO, typename ST>
hipError_t launch(const ResidualArgs& a, bool backward, int* parts, hipStream_t stream) {
  int L = row_width(a.n);
  const int threads = threads_of(L, backward);
  const long long rows = static_cast<long long>(a.B) * a.T, groups = (rows + threads / L - 1) / (threads / L);
  const int most = workgroups_of(threads, backward);
  const int grid = static_cast<int>(groups < most ? groups : most);
  if (parts != nullptr) *parts = grid;
  if (grid == 0) return hipSuccess;
  const bool whole = L == threads;
  const void* forward_kernel = whole ? reinterpret_cast<const void*>(&residual_kernel<IO, ST, true>) : reinterpret_cast<const void*>(&residual_kernel<IO, ST, false>);
  const void* backward_kernel =
      whole ? reinterpret_cast<const void*>(&residual_backward_kernel<IO, ST, true>) : reinterpret_cast<const void*>(&residual_backward_kernel<IO, ST, false>);
  ResidualArgs args = a;
  const int lds = 4 * 2 * 16 + 2 * threads + (backward ? 3 * a.n + (whole ? 0 : kColumns * threads) : 0);
  void* params[] = {&args, &L};
  return hipLaunchKernel(backward ? backward_kernel : forward_kernel, dim3(grid), dim3(threads), params, lds * sizeof(float), stream);
}
hipError_t launch_types(const ResidualArgs& a, int io_dtype, int stream_dtype, bool backward, int* parts, hipStream_t stream) {
  if (io_dtype == 0) return launch<float, float>(a, backward, parts, stream);
  if (stream_dtype == 0) return launch<uint16_t, float>(a, backward, parts, stream);
  return launch<uint16_t, uint16_t>(a, backward, parts, stream);
}

}  // namespace

int residual_partials(int n) { return workgroups_of(threads_of(row_width(n), true), true); }
hipError_t launch_residual_norm(const ResidualArgs& a, int io_dtype, int stream_dtype, hipStream_t stream) {
  return launch_types(a, io_dtype, stream_dtype, false, nullptr, stream);
}
hipError_t launch_residual_norm_backward(const ResidualArgs& a, int io_dtype, int stream_dtype, int* parts, hipStream_t stream) {
  return launch_types(a, io_dtype, stream_dtype, true, parts, stream);
}

}  // namespace vla

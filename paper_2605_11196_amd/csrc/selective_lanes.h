// What the kernels of the selective state space scan share: how a wave's lanes hold the states, and how the operands of a block of tokens
// get to them.
//
// N / 4 neighbouring lanes hold a channel, four states (16 bytes of A, of a state, of B and C) each; a wave 256 / N channels. So sums over states stay
// in a row of lanes (DPP), states and A go to and from memory as they lie there, and the waves of a sequence need no barrier.  The tokens go by in
// blocks of eight.  What depends on the token and the channel alone (the step, the gate, the output) is formed once, for a token and a pair of channels a
// lane, so that a block's rows take one load of 4 (float32: 8) bytes a lane each, and passed on through LDS, as B and C are, which a wave stages
// for itself.
#pragma once

#include "mixer_util.h"

namespace vla {

constexpr int TB = kScanBlock;

// Waves of a workgroup: neighbouring channels' rows are pieces of one cache line, and dB and dC are summed over the waves.
constexpr int scan_waves(int N) { return 4; }
constexpr int scan_tile(int N) { return scan_waves(N) * 256 / N; }   // channels of a workgroup

// A thread's place: sequence, time segment, channel, states; and the tokens and pairs of channels that it loads and stores.
template <int N>
struct ScanPlace {
  static constexpr int LN = N / 4, CW = 64 / LN;          // lanes of a channel, channels of a wave
  static constexpr int PAIRS = CW / 2, OWN = TB * PAIRS >= 64 ? TB * PAIRS / 64 : 1;   // pairs of a wave's channels, tokens of a lane
  int b, seg, tile, group, lane, wave, q, in_wave;
  unsigned c;              // channel
  bool here;               // it is one of the group's (otherwise c is another one's, and nothing is stored)
  unsigned c2;             // first channel of the pair
  int pair;
  bool here2;              // the pair is the group's, and the lane has tokens
  int length, first, last, live;   // tokens of the sequence, of the segment, and where its sequence ends in it
  __device__ __forceinline__ explicit ScanPlace(const ScanArgs& a) {
    const unsigned tiles = a.G * a.tiles;
    tile = blockIdx.x % tiles;
    const unsigned rest = blockIdx.x / tiles;
    seg = rest % a.n_seg;
    b = rest / a.n_seg;
    group = tile / a.tiles;
    lane = threadIdx.x % 64;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    q = lane % LN;
    in_wave = lane / LN;
    pair = lane % PAIRS;
    const int of_group = a.n / a.G, from = tile % a.tiles * scan_tile(N) + wave * CW, at = from + in_wave, at2 = from + 2 * pair;
    here = at < of_group;
    c = group * of_group + (here ? at : of_group - 1);
    here2 = at2 < of_group && lane < TB * PAIRS;
    c2 = group * of_group + (at2 < of_group ? at2 : of_group - 2);
    length = a.lengths == nullptr ? a.T : min(max(a.lengths[b], 0), a.T);
    first = seg * a.seg_tokens;
    last = min(first + a.seg_tokens, a.T);
    live = min(last, length);
  }
  // token of the block that is this lane's k-th own one
  __device__ __forceinline__ int own(int k) const { return min(lane / PAIRS, TB - 1) + 64 / PAIRS * k; }
};

// Two neighbouring values as they lie in memory
template <typename IO> struct PairOf;
template <> struct PairOf<float> { typedef f2 type; };
template <> struct PairOf<uint16_t> { typedef uint32_t type; };
template <typename IO> using Pair = typename PairOf<IO>::type;
__device__ __forceinline__ f2 wide2(f2 x) { return x; }
__device__ __forceinline__ f2 wide2(uint32_t x) { return widen(x); }
__device__ __forceinline__ f2 or_zero(bool in, f2 x) { return f2{in ? x[0] : 0.0f, in ? x[1] : 0.0f}; }
__device__ __forceinline__ uint32_t or_zero(bool in, uint32_t x) { return in ? x : 0u; }
template <typename IO> __device__ __forceinline__ Pair<IO> narrow2(f2 x) {
  if constexpr (sizeof(IO) == 2) return pack_rne(x[0], x[1]);
  else return x;
}

// A [B, T, n] tensor seen from a lane: its own tokens' pairs of a block, from the block's first token on (`row`).
template <int N, typename IO>
struct ScanRows {
  static constexpr int OWN = ScanPlace<N>::OWN;
  char* base;              // of the sequence
  long long step;          // bytes from token to token
  unsigned at;             // bytes from a block's first token to the lane's own first one
  __device__ __forceinline__ ScanRows(const ScanPlace<N>& w, const void* p, Row2 r) {
    base = const_cast<char*>(static_cast<const char*>(p)) + w.b * r.b * static_cast<long long>(sizeof(IO));
    step = r.t * static_cast<long long>(sizeof(IO));
    at = w.own(0) * static_cast<unsigned>(step) + w.c2 * static_cast<unsigned>(sizeof(IO));
  }
  __device__ __forceinline__ char* row(int t0) const { return base + t0 * step; }
  // where the k-th own tokens' rows begin: the same for all lanes
  template <typename P> __device__ __forceinline__ P* own(P* row, int k) const { return row + k * (64 / ScanPlace<N>::PAIRS) * step; }
  __device__ __forceinline__ void load(const char* row, Pair<IO> (&v)[OWN]) const {
#pragma unroll
    for (int k = 0; k < OWN; ++k) v[k] = *reinterpret_cast<const Pair<IO>*>(own(row, k) + at);
  }
  // of a block with `tokens` of them, the rest of its rows being the last one
  __device__ __forceinline__ void load(const char* row, Pair<IO> (&v)[OWN], const ScanPlace<N>& w, int tokens) const {
#pragma unroll
    for (int k = 0; k < OWN; ++k) v[k] = *reinterpret_cast<const Pair<IO>*>(row + (at + k * (64 / ScanPlace<N>::PAIRS) * static_cast<unsigned>(step) - max(w.own(k) - (tokens - 1), 0) * static_cast<unsigned>(step)));
  }
  // of the block at t0 - skip, the `skip` tokens before t0 being the one at t0
  __device__ __forceinline__ void load(Pair<IO> (&v)[OWN], const ScanPlace<N>& w, int t0, int skip) const {
    const char* from = row(t0 - skip);
    if (skip == 0) {
      load(from, v);
    } else {
#pragma unroll
      for (int k = 0; k < OWN; ++k) v[k] = *reinterpret_cast<const Pair<IO>*>(own(from, k) + (at + max(skip - w.own(k), 0) * static_cast<unsigned>(step)));
    }
  }
  __device__ __forceinline__ void store(char* row, int k, Pair<IO> x) const { *reinterpret_cast<Pair<IO>*>(own(row, k) + at) = x; }
};

// B and C of a block: a wave's lanes load N / 4 neighbouring values each and put them into LDS as float32, [token][B | C].
template <int N, typename IO>
struct ScanStage {
  static constexpr int V = N / 4, WORDS = V * sizeof(IO) / 4;
  const char* row;         // this lane's piece of its token's row
  long long step;          // bytes from token to token
  int t, at;               // token of the block, float of the row
  uint32_t raw[WORDS];
  // row: of the block at t0
  __device__ __forceinline__ ScanStage(const ScanPlace<N>& w, const ScanArgs& a, int t0) {
    t = w.lane / 8;
    at = w.lane % 8 * V;
    const bool is_c = at >= N;
    step = (is_c ? a.C_t : a.B_t) * static_cast<long long>(sizeof(IO));
    row = (is_c ? static_cast<const char*>(a.Cm) + (w.b * a.C_b + w.group * a.C_g + (at - N)) * static_cast<long long>(sizeof(IO))
                : static_cast<const char*>(a.Bm) + (w.b * a.B_b + w.group * a.B_g + at) * static_cast<long long>(sizeof(IO))) + (t0 + t) * step;
  }
  template <bool BACK> __device__ __forceinline__ void go() { row = BACK ? row - TB * step : row + TB * step; }
  // of a block with `tokens` of them (TB: all), the rest of its rows being the last one
  __device__ __forceinline__ void load(int tokens) { load(tokens < TB ? row - max(t - (tokens - 1), 0) * step : row); }
  // of the block `skip` tokens earlier, those that lie before the row's own block being its first one
  __device__ __forceinline__ void load_behind(int skip) { load(skip != 0 ? row - min(skip, t) * step : row); }
  __device__ __forceinline__ void load(const char* from) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(from);
    if constexpr (WORDS == 1) {
      raw[0] = *p;
    } else if constexpr (WORDS == 2) {
      const u2 x = *reinterpret_cast<const u2*>(p);
      raw[0] = x[0];
      raw[1] = x[1];
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const u4 x = *reinterpret_cast<const u4*>(p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[i + k] = x[k];
      }
    }
  }
  // rows: the wave's own [TB][2 N]; in: whether the token counts, otherwise zeros
  __device__ __forceinline__ void put(float* rows, bool in) const {
    uint32_t kept[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) kept[i] = in ? raw[i] : 0u;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      f2 x;
      if constexpr (sizeof(IO) == 2) x = widen(kept[i / 2]);
      else x = f2{__uint_as_float(kept[i]), __uint_as_float(kept[i + 1])};
      *reinterpret_cast<f2*>(rows + t * 2 * N + at + i) = x;
    }
  }
};

// What a wave has written to its own part of LDS is there for its lanes: LDS serves a wave's instructions in order, so only the compiler is held.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ f2 pair_of(const float* p, unsigned c) { return p != nullptr ? f2{p[c], p[c + 1]} : f2{0.0f, 0.0f}; }
// Sum over a channel's lanes, in every one of them.
template <int LN> __device__ __forceinline__ float channel_sum(float x) {
  if constexpr (LN >= 2) x = dpp_sum<0xB1>(x);
  if constexpr (LN >= 4) x = dpp_sum<0x4E>(x);
  if constexpr (LN >= 8) x = dpp_sum<0x141>(x);
  if constexpr (LN >= 16) x = dpp_sum<0x140>(x);
  return x;
}

// The lanes' sums of a number for each token of a block.  Of every LN tokens lane q gets that of token q (LN > 8: of 8), own[k] that of token LN k + q.
template <int LN> constexpr int kTurns = LN >= TB ? 1 : TB / LN;
template <int LN>
__device__ __forceinline__ void keep_sum(float x, float (&some)[4], float (&own)[kTurns<LN>], int t, bool last, int q) {
  if constexpr (LN <= 4) {
    some[t % LN] = x;
    if (!last) return;
    const bool odd = q & 1, high = q & 2;
    float r[2];
#pragma unroll
    for (int h = 0; h < LN / 2; ++h) {
      const float keep = odd ? some[2 * h + 1] : some[2 * h], send = odd ? some[2 * h] : some[2 * h + 1];
      r[h] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), 0xB1, 0xf, 0xf, true));
    }
    if constexpr (LN == 4) {
      const float keep = high ? r[1] : r[0], send = high ? r[0] : r[1];
      r[0] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), 0x4E, 0xf, 0xf, true));
    }
    own[t / LN] = r[0];
  } else {
    const float sum = channel_sum<LN>(x);
    own[0] = q == t ? sum : own[0];
  }
}

}  // namespace vla

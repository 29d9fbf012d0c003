// What the kernels of the selective state space scan share: how a wave's lanes hold the states, and how the operands of a block of tokens
// get to them.
//
// N / 4 neighbouring lanes hold a channel, four states (16 bytes of A, of a state, of B and C) each; a wave 256 / N channels. So sums over states stay
// in a row of lanes (DPP), states and A go to and from memory as they lie there, and the waves of a sequence need no barrier.  The tokens go by in
// blocks of eight.  What depends on the token and the channel alone (the step, the gate) is formed once, by the lane whose place
// among the channel's is the token's, and passed to the others through LDS, as B and C are, which a wave stages for itself.
#pragma once

#include "mixer_util.h"

namespace vla {

constexpr int TB = kScanBlock;

// Waves of a workgroup: neighbouring channels' rows are pieces of one cache line, and dB and dC are summed over the waves.
constexpr int scan_waves(int N) { return 4; }
constexpr int scan_tile(int N) { return scan_waves(N) * 256 / N; }   // channels of a workgroup

// A thread's place: sequence, time segment, channel, states.
template <int N>
struct ScanPlace {
  static constexpr int LN = N / 4, CW = 64 / LN, OWN = LN >= TB ? 1 : TB / LN;   // lanes of a channel, channels of a wave, tokens of a lane
  int b, seg, tile, group, lane, wave, q;
  unsigned c;              // channel
  bool here;               // it is one of the group's (otherwise c is another one's, and nothing is stored)
  bool owner;              // the lane has tokens
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
    const int of_group = a.n / a.G, at = tile % a.tiles * scan_tile(N) + wave * CW + lane / LN;
    here = at < of_group;
    c = group * of_group + (here ? at : of_group - 1);
    owner = LN <= TB || q < TB;
    length = a.lengths == nullptr ? a.T : min(max(a.lengths[b], 0), a.T);
    first = seg * a.seg_tokens;
    last = min(first + a.seg_tokens, a.T);
    live = min(last, length);
  }
  // token of the block that is this lane's k-th own one
  __device__ __forceinline__ int own(int k) const { return LN > TB ? min(q, TB - 1) : q + LN * k; }
};

// A [B, T, n] tensor seen from a lane: its own tokens of a block, from a base that goes along with the block.
template <int N, typename IO>
struct ScanRows {
  static constexpr int OWN = ScanPlace<N>::OWN;
  char* base;              // of the sequence
  long long step;          // bytes from token to token
  unsigned at[OWN];        // bytes from the block's first token
  __device__ __forceinline__ ScanRows(const ScanPlace<N>& w, const void* p, Row2 r) {
    base = const_cast<char*>(static_cast<const char*>(p)) + w.b * r.b * static_cast<long long>(sizeof(IO));
    step = r.t * static_cast<long long>(sizeof(IO));
#pragma unroll
    for (int k = 0; k < OWN; ++k) at[k] = w.own(k) * static_cast<unsigned>(step) + w.c * static_cast<unsigned>(sizeof(IO));
  }
  // the rows of block t0 (past the end of memory the last one)
  __device__ __forceinline__ void load(const ScanPlace<N>& w, int T, int t0, IO (&v)[OWN]) const {
    const char* from = base + t0 * step;
    if (t0 + TB <= T) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) v[k] = *reinterpret_cast<const IO*>(from + at[k]);
    } else {
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        v[k] = *reinterpret_cast<const IO*>(from + (min(w.own(k), T - 1 - t0) * static_cast<unsigned>(step) + w.c * static_cast<unsigned>(sizeof(IO))));
      }
    }
  }
  __device__ __forceinline__ void store(int t0, int k, float x) const { put(reinterpret_cast<IO*>(base + t0 * step + at[k]), x); }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
  static __device__ __forceinline__ void put(uint16_t* p, float x) { *p = static_cast<uint16_t>(pack_rne(x, x)); }
};
__device__ __forceinline__ float wide1(float x) { return x; }
__device__ __forceinline__ float wide1(uint16_t x) { return bf16_to_f32(x); }

// B and C of a block: a wave's lanes load N / 4 neighbouring values each and put them into LDS as float32, [token][B | C].
template <int N, typename IO>
struct ScanStage {
  static constexpr int V = N / 4, WORDS = V * sizeof(IO) / 4;
  const char* from;        // of the sequence, this lane's piece of a row
  long long step;
  int t, at;               // token of the block, float of the row
  uint32_t raw[WORDS];
  __device__ __forceinline__ ScanStage(const ScanPlace<N>& w, const ScanArgs& a) {
    t = w.lane / 8;
    at = w.lane % 8 * V;
    const bool is_c = at >= N;
    step = (is_c ? a.C_t : a.B_t) * static_cast<long long>(sizeof(IO));
    from = is_c ? static_cast<const char*>(a.Cm) + (w.b * a.C_b + w.group * a.C_g + (at - N)) * static_cast<long long>(sizeof(IO))
                : static_cast<const char*>(a.Bm) + (w.b * a.B_b + w.group * a.B_g + at) * static_cast<long long>(sizeof(IO));
  }
  __device__ __forceinline__ void load(int T, int t0) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(from + min(t0 + t, T - 1) * step);
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
  // rows: the wave's own [TB][2 N]; tokens past the end of the sequence give zeros
  __device__ __forceinline__ void put(float* rows, int t0, int length) const {
    const bool in = t0 + t < length;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      f2 x;
      if constexpr (sizeof(IO) == 2) x = widen(raw[i / 2]);
      else x = f2{__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])};
      *reinterpret_cast<f2*>(rows + t * 2 * N + at + i) = f2{in ? x[0] : 0.0f, in ? x[1] : 0.0f};
    }
  }
};

// What a wave has written to its own part of LDS is there for its lanes: LDS serves a wave's instructions in order, so only the compiler is held.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// Sum over a channel's lanes, in every one of them.
template <int LN> __device__ __forceinline__ float channel_sum(float x) {
  if constexpr (LN >= 2) x = dpp_sum<0xB1>(x);
  if constexpr (LN >= 4) x = dpp_sum<0x4E>(x);
  if constexpr (LN >= 8) x = dpp_sum<0x141>(x);
  if constexpr (LN >= 16) x = dpp_sum<0x140>(x);
  return x;
}

}  // namespace vla

// The gated delta rule in blocks of 32 tokens (delta_block.h has the mathematics): one workgroup per head (and time segment) goes
// through the blocks with the state on registers.
//
// A wave has 16 rows of S; the waves of a head share the matrices between tokens, which different waves form at once, beside the products
// of K and Q with the state.  Three barriers a block: rows staged; matrices ready; rows no longer needed.
//
// 512 heads of 128, 8192 tokens, bf16 1.72 ms = 2.5 TB/s of q, k, v and o, two workgroups of eight waves a compute unit (128 registers).  Neither unit is full: the
// matrix unit is busy for 56 % of the SIMD cycles and other vector instructions take 51 %, which can overlap; a quarter of the matrix instructions
// form residuals of the three terms.  A workgroup alone takes 3.6 us a block, two 6.7, and few heads see the first: the substitution (700 cycles) and
// the solution, a chain of some ten dependent products and splits (3000 cycles).
//
// MAP: the affine map of a segment instead of its outputs, S_end = S_start X + Y: Y from d_v columns that start from zero, X from d_k
// columns without values that start from the identity.  The first segment needs no map: where that shortens the way (first_done), a
// workgroup beside the maps' forms its outputs and its end.
#pragma once

#include "delta_block.h"

namespace vla {
namespace delta {

template <int DK, int DV, bool MAP>
struct Shape {
  static constexpr int COLS = DV + (MAP ? DK : 0);
  static constexpr int WAVES = COLS / 16;
  static constexpr int THREADS = 64 * WAVES;
  // waves of a SIMD where as many workgroups share a compute unit as four waves a SIMD allow
  static constexpr int HELD = MAP ? (16 / WAVES * WAVES + 3) / 4 : 4;
  static constexpr int DKP = DK < 32 ? 32 : DK;               // key columns in pairs of tiles
  static constexpr int KT = DKP / 16;
};

template <typename IO, int DK, int DV, bool MAP>
__device__ __forceinline__ void chunk_segment(const DeltaArgs& a, int head, int seg) {
  using Sh = Shape<DK, DV, MAP>;
  using O = Ops<IO>;
  constexpr int KT = Sh::KT, WAVES = Sh::WAVES, THREADS = Sh::THREADS;
  constexpr int PK = DK / O::PER16, PV = DV / O::PER16;
  using RK = PieceRows<Sh::DKP / O::PER16>;
  using RV = PieceRows<PV>;
  __shared__ u4 sK[kTok * RK::STRIDE];
  __shared__ u4 sQ[MAP ? 1 : kTok * RK::STRIDE];
  __shared__ u4 sV[kTok * RV::STRIDE];
  __shared__ typename O::Image inverse[kTiles], below[kTiles * (kTiles - 1) / 2];
  __shared__ typename O::ImageOut att[MAP ? 1 : kTiles * (kTiles + 1) / 2];
  __shared__ __align__(16) float scratch[kTiles][16 * 20];
  __shared__ Gates gates[2];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  int c = lane % 16, g = lane / 16;
  const int b = head / a.H_v, h = head % a.H_v, hk = h / (a.H_v / a.H_k);
  const int len = __builtin_amdgcn_readfirstlane(a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T);
  const int first = seg * a.seg_tokens, last = seg == a.n_seg - 1 ? a.T : first + a.seg_tokens, end = min(len, last);
  const char* q = reinterpret_cast<const char*>(static_cast<const IO*>(a.q) + b * a.qs.b + hk * a.qs.h);
  const char* k = reinterpret_cast<const char*>(static_cast<const IO*>(a.k) + b * a.ks.b + hk * a.ks.h);
  const char* v = reinterpret_cast<const char*>(static_cast<const IO*>(a.v) + b * a.vs.b + h * a.vs.h);
  char* o = MAP ? nullptr : reinterpret_cast<char*>(static_cast<IO*>(a.o) + b * a.os.b + h * a.os.h);
  const long long q_step = a.qs.t * sizeof(IO), k_step = a.ks.t * sizeof(IO), v_step = a.vs.t * sizeof(IO), o_step = a.os.t * sizeof(IO);
  const float* gp = a.g + b * a.gs.b + h * a.gs.h;
  const float* bp = a.beta + b * a.bs.b + h * a.bs.h;
  const float scale = a.scale;
  const typename O::One one = O::one(c, g);
  const auto col = [&] { return wave * 16 + c; };      // column of this lane
  const f4 zero = f4{0.0f, 0.0f, 0.0f, 0.0f};

  // ---- the state: tile kt holds key columns 32 (kt / 2) + 8 g + 4 (kt % 2) + r
  f4 S[KT];
  const size_t slot = static_cast<size_t>(head) * a.n_slots + seg - (a.n_seg - a.n_slots);
  const float* S0 = !MAP && a.S0 ? a.S0 + (a.seg_states ? slot : static_cast<size_t>(head)) * DV * DK : nullptr;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
    S[kt] = zero;
    if ((DK == Sh::DKP || dk < DK) && S0 != nullptr) S[kt] = *reinterpret_cast<const f4*>(S0 + static_cast<uint32_t>(col() * DK + dk));
    if (MAP && col() >= DV) {
#pragma unroll
      for (int r = 0; r < 4; ++r) S[kt][r] = col() - DV == dk + r ? 1.0f : 0.0f;
    }
  }
  if constexpr (Sh::DKP > DK) {             // columns that no row fills
    for (int i = threadIdx.x; i < kTok * RK::STRIDE; i += THREADS) {
      sK[i] = u4{0, 0, 0, 0};
      if constexpr (!MAP) sQ[i] = u4{0, 0, 0, 0};
    }
    __syncthreads();
  }

  Stage<PK, THREADS> stK, stQ;
  Stage<PV, THREADS> stV;
  stK.init(k_step);
  if constexpr (!MAP) stQ.init(q_step);
  stV.init(v_step);
  float gate = 0.0f, beta = 0.0f;           // of one token a lane, a block ahead of the rows
  auto request = [&](int t0) {
    stK.load(k, k_step, t0, end);
    if constexpr (!MAP) stQ.load(q, q_step, t0, end);
    stV.load(v, v_step, t0, end);
  };
  auto request_gates = [&](int t0) {
    const int t = max(min(t0 + (lane & (kTok - 1)), end - 1), first);
    gate = gp[t * a.gs.t];
    beta = bp[t * a.bs.t];
  };
  auto next_gates = [&](int t0, Gates& to) {
    if (wave == WAVES - 1) put_gates(to, lane, lane, t0 + lane < end ? gate : 0.0f, t0 + lane < end ? beta : 0.0f);
  };
  if (first < end) {
    request_gates(first);
    request(first);
    next_gates(first, gates[0]);
    request_gates(first + kTok);
  }
  int turn = 0;

  for (int t0 = first; t0 < end;) {
    // the state at the start of every 256 tokens; the blocks between two such places in a loop of their own
    if (!MAP && a.kept != nullptr && t0 % kKeep == 0) {
      float* out = a.kept + (static_cast<size_t>(head) * a.n_kept + t0 / kKeep) * DV * DK;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
        if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<uint32_t>(col() * DK + dk)) = S[kt];
      }
    }
    const int stop = min(end, (t0 / kKeep + 1) * kKeep);
    for (; t0 < stop; t0 += kTok) {
      // the LDS addresses are formed anew in each block: kept over the loop they would take the registers of the state
      asm volatile("" : "+v"(c), "+v"(g));
      stK.template store<RK>(sK);
      if constexpr (!MAP) stQ.template store<RK>(sQ);
      stV.template store<RV>(sV);
      const Gates& gt = gates[turn];
      turn ^= 1;
      __syncthreads();
      // The chains of dependent steps go before the products with the state, which keep the matrix unit busy by themselves: the waves of
      // the other workgroup of the compute unit take turns better (512 heads: 1.762 -> 1.718 ms).
      __builtin_amdgcn_s_setprio(2);
      token_matrices<IO, RK, KT / 2, WAVES, false, !MAP>(sK, sQ, gt, inverse, below, att, scratch, scale, wave, c, g);
      __builtin_amdgcn_s_setprio(0);

      // ---- P = K S^T, Q S^T
      f4 P[kTiles] = {zero, zero}, QS[kTiles] = {zero, zero};
#pragma unroll
      for (int s = 0; s < KT / 2; ++s) {
        typename O::A ka[kTiles], qa[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          ka[i] = O::template rows<RK>(sK, i, s, c, g);
          if constexpr (!MAP) qa[i] = O::template rows<RK>(sQ, i, s, c, g);
        }
        const typename O::B x = O::pair(S[2 * s], S[2 * s + 1], one);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          P[i] = O::mul(ka[i], x, P[i]);
          if constexpr (!MAP) QS[i] = O::mul_out(qa[i], x, QS[i]);
        }
      }
      __syncthreads();
      if (t0 + kTok < end) request(t0 + kTok);

      // ---- what is written, the read-out, the state
      const auto gate4 = [&](const float* from, int tile) { return *reinterpret_cast<const f4*>(from + 16 * tile + 4 * g); };
      static_assert(kTiles == 2, "one pair of token tiles");
      __builtin_amdgcn_s_setprio(1);
      // what comes from LDS is asked for well before it is used: the compiler keeps that order
      f4 R[kTiles], gamma[kTiles];
      typename O::TB rb[kTiles];
      typename O::TA inv[kTiles];
      typename O::Raw vr[kTiles] = {};
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        gamma[i] = gate4(gt.gamma, i);
        inv[i] = O::image(inverse[i], c, g);
        if (!MAP || wave * 16 < DV) vr[i] = O::template tile_raw<RV>(sV, wave, i, c, g);
      }
      const typename O::TA under = O::image(below[0], c, g);
      R[0] = O::mul_tok(inv[0], O::tokens(O::value(vr[0]) - gamma[0] * P[0], one), zero);
      const f4 w0 = gate4(gt.rest, 0) * gate4(gt.beta, 0), w1 = gate4(gt.rest, 1) * gate4(gt.beta, 1);
      rb[0] = O::tokens(R[0], one);
      R[1] = O::mul_tok(inv[1], O::tokens(O::mul_tok(under, rb[0], O::value(vr[1]) - gamma[1] * P[1]), one), zero);
      if (!MAP) rb[1] = O::tokens(R[1], one);
      if (!MAP && a.rows != nullptr) {
        const __amdgpu_buffer_rsrc_t out = rows_buffer(a.rows + (static_cast<size_t>(head) * a.T + t0) * DV, DV * 4, end - t0, DV * 4);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) store_column(out, ((16 * i + 4 * g) * DV + col()) * 4, DV * 4, R[i], static_cast<float*>(nullptr));
      }
      const typename O::B w = O::pair(R[0] * w0, R[1] * w1, one);
      if constexpr (!MAP) {
        const decltype(O::image(att[0], c, g)) at[3] = {O::image(att[0], c, g), O::image(att[1], c, g), O::image(att[2], c, g)};
        const __amdgpu_buffer_rsrc_t out = rows_buffer(o + t0 * o_step, o_step, end - t0, DV * static_cast<int>(sizeof(IO)));
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          f4 x = gamma[i] * scale * QS[i];
#pragma unroll
          for (int j = 0; j <= i; ++j) x = O::mul_tok_out(at[i + j], rb[j], x);
          store_column(out, (16 * i + 4 * g) * static_cast<int>(o_step) + col() * static_cast<int>(sizeof(IO)), static_cast<int>(o_step), x,
                       static_cast<IO*>(nullptr));
        }
      }
      const float decay = gt.end;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) S[kt] = O::mul(O::template columns<RK>(sK, kt, 0, c, g), w, S[kt] * decay);
      __builtin_amdgcn_s_setprio(0);
      next_gates(t0 + kTok, gates[turn]);
      request_gates(t0 + 2 * kTok);
      __syncthreads();
    }
  }

  // ---- outputs of tokens past the end of the sequence (the block that it ends in stores none for them: they would be NaN beside an infinite
  // state), the state
  if constexpr (!MAP) {
    for (int t = max(first, end) + wave; t < last; t += WAVES) {
      for (int i = lane; i < DV; i += 64) io_store(reinterpret_cast<IO*>(o + t * o_step) + i, 0.0f);
    }
  }
  float* out = nullptr;
  if (MAP) out = a.seg_map + slot * Sh::COLS * DK;
  else if (a.seg_S != nullptr) out = a.seg_S + (slot + 1) * DV * DK;
  else if (a.S_T != nullptr && seg == a.n_seg - 1) out = a.S_T + static_cast<size_t>(head) * DV * DK;
  if (out == nullptr) return;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
    if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<uint32_t>(col() * DK + dk)) = S[kt];
  }
}

template <typename IO, int DK, int DV, bool MAP>
__global__ void __launch_bounds__((Shape<DK, DV, MAP>::THREADS), (Shape<DK, DV, MAP>::HELD)) delta_chunk_kernel(DeltaArgs a) {
  if constexpr (MAP) {      // of all segments but the last one on the way
    const int n = a.n_seg - 1, head = blockIdx.x / n, at = blockIdx.x % n, seg = at;
    if constexpr (delta_first_with_maps(DV)) {
      if (at == 0 && a.first_done) {
        if (__builtin_amdgcn_readfirstlane(threadIdx.x) < Shape<DK, DV, false>::THREADS) chunk_segment<IO, DK, DV, false>(a, head, seg);
        return;
      }
    }
    chunk_segment<IO, DK, DV, true>(a, head, seg);
  } else {
    const int n = a.n_seg - (a.first_done ? 1 : 0), head = blockIdx.x / n, at = blockIdx.x % n;
    chunk_segment<IO, DK, DV, false>(a, head, at + a.n_seg - n);
  }
}

template <int DK, int DV, bool MAP>
hipError_t launch_chunk(const DeltaArgs& a, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args};
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_chunk_kernel<uint16_t, DK, DV, MAP>)
                                 : reinterpret_cast<const void*>(&delta_chunk_kernel<float, DK, DV, MAP>);
  return hipLaunchKernel(fn, dim3(a.B * a.H_v * (a.n_seg - (MAP || a.first_done ? 1 : 0))), dim3(Shape<DK, DV, MAP>::THREADS), params, 0, stream);
}

template <int DK>
hipError_t launch_chunk_dk(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream) {
  switch (d_v) {
#define VLA_DV(N) case N: return map ? launch_chunk<DK, N, true>(a, io_dtype, stream) : launch_chunk<DK, N, false>(a, io_dtype, stream);
    VLA_DV(16) VLA_DV(32) VLA_DV(64) VLA_DV(96) VLA_DV(128)
#undef VLA_DV
    default: return hipErrorInvalidValue;
  }
}

}  // namespace delta
}  // namespace vla

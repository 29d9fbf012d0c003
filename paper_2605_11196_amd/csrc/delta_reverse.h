// The gradient of the gated delta rule's state, from the last block of 32 tokens to the first (delta_block.h has the forward mathematics).
// With dS the gradient of the state at the end of a block, D, gamma, beta as there and L_ij = beta_i D_ij (k_i . k_j), j < i:
//   dU = scale (D * Q K^T)^T dO + exp(G_end - G) (K dS^T);   (I + L)^T W = dU;   dV = beta W
//   dS <- gamma_end dS + scale (gamma dO)^T Q - (gamma beta W)^T K
// Nothing of it needs the state itself.  The rows of a block are staged with the last token first, which makes the system lower triangular,
// and then everything is as in the forward kernel (delta_chunk.h): a wave has 16 columns of what has d_v columns.  W is kept in float32,
// and dS at the end of every 256 tokens, for the kernel that forms the other gradients (delta_grad.h).
//
// Bound like the forward kernel: 64 heads of 128, 4096 tokens in five segments 150 us, and 168 us for the maps.
//
// MAP: the affine map of a segment, dS_start = dS_end X + Y.
#pragma once

#include "delta_chunk.h"

namespace vla {
namespace delta {

template <typename IO, int DK, int DV, bool MAP>
__device__ __forceinline__ void reverse_segment(const DeltaArgs& a, int head, int seg) {
  using Sh = Shape<DK, DV, MAP>;
  using O = Ops<IO>;
  constexpr int KT = Sh::KT, WAVES = Sh::WAVES, THREADS = Sh::THREADS;
  constexpr int PK = DK / O::PER16, PV = DV / O::PER16;
  using RK = PieceRows<Sh::DKP / O::PER16>;
  using RV = PieceRows<PV>;
  __shared__ u4 sK[kTok * RK::STRIDE];
  __shared__ u4 sQ[kTok * RK::STRIDE];
  __shared__ u4 sD[kTok * RV::STRIDE];
  __shared__ typename O::Image inverse[kTiles], below[kTiles * (kTiles - 1) / 2], att[kTiles * (kTiles + 1) / 2];
  __shared__ __align__(16) float scratch[kTiles][16 * 20];
  __shared__ Gates gates[2];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  int c = lane % 16, g = lane / 16;
  const int b = head / a.H_v, h = head % a.H_v, hk = h / (a.H_v / a.H_k);
  const int len = __builtin_amdgcn_readfirstlane(a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T);
  const int first = seg * a.seg_tokens, last = seg == a.n_seg - 1 ? a.T : first + a.seg_tokens, end = min(len, last);
  const char* q = reinterpret_cast<const char*>(static_cast<const IO*>(a.q) + b * a.qs.b + hk * a.qs.h);
  const char* k = reinterpret_cast<const char*>(static_cast<const IO*>(a.k) + b * a.ks.b + hk * a.ks.h);
  const char* dO = reinterpret_cast<const char*>(static_cast<const IO*>(a.dO) + b * a.os.b + h * a.os.h);
  char* dv = MAP ? nullptr : reinterpret_cast<char*>(static_cast<IO*>(a.dv) + b * a.dvs.b + h * a.dvs.h);
  const long long q_step = a.qs.t * sizeof(IO), k_step = a.ks.t * sizeof(IO), o_step = a.os.t * sizeof(IO), dv_step = a.dvs.t * sizeof(IO);
  const float* gp = a.g + b * a.gs.b + h * a.gs.h;
  const float* bp = a.beta + b * a.bs.b + h * a.bs.h;
  const float scale = a.scale;
  const typename O::One one = O::one(c, g);
  const auto col = [&] { return wave * 16 + c; };      // column of this lane
  const f4 zero = f4{0.0f, 0.0f, 0.0f, 0.0f};

  // ---- the state: tile kt holds key columns 32 (kt / 2) + 8 g + 4 (kt % 2) + r
  f4 S[KT];
  const size_t slot = static_cast<size_t>(head) * a.n_slots + seg;
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
      sQ[i] = u4{0, 0, 0, 0};
    }
    __syncthreads();
  }

  Stage<PK, THREADS> stK, stQ;
  Stage<PV, THREADS> stD;
  stK.init_reversed(k_step);
  stQ.init_reversed(q_step);
  stD.init_reversed(o_step);
  float gate = 0.0f, beta = 0.0f;           // of one token a lane, a block ahead of the rows
  auto request = [&](int t0) {
    stK.load(k, k_step, t0, end);
    stQ.load(q, q_step, t0, end);
    stD.load(dO, o_step, t0, end);
  };
  auto request_gates = [&](int t0) {
    const int t = max(min(t0 + (lane & (kTok - 1)), end - 1), first);
    gate = gp[t * a.gs.t];
    beta = bp[t * a.bs.t];
  };
  auto next_gates = [&](int t0, Gates& to) {
    if (wave == WAVES - 1) put_gates(to, lane, kTok - 1 - lane, t0 + lane < end ? gate : 0.0f, t0 + lane < end ? beta : 0.0f);
  };
  const int blocks = first < end ? (end - first + kTok - 1) / kTok : 0, start = first + max(0, blocks - 1) * kTok;
  if (blocks > 0) {
    request_gates(start);
    request(start);
    next_gates(start, gates[0]);
    request_gates(start - kTok);
  }
  int turn = 0;

  for (int t0 = start, left = blocks; left > 0;) {
    // dS at the end of every 256 tokens; the blocks between two such places in a loop of their own
    if (!MAP && ((t0 + kTok) % kKeep == 0 || t0 + kTok >= len)) {
      float* out = a.kept + (static_cast<size_t>(head) * a.n_kept + t0 / kKeep) * DV * DK;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
        if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<uint32_t>(col() * DK + dk)) = S[kt];
      }
    }
    for (int inner = min(left, t0 % kKeep / kTok + 1); inner > 0; --inner, --left, t0 -= kTok) {
      // the LDS addresses are formed anew in each block: kept over the loop they would take the registers of the state
      asm volatile("" : "+v"(c), "+v"(g));
      stK.template store<RK>(sK);
      stQ.template store<RK>(sQ);
      stD.template store<RV>(sD);
      const Gates& gt = gates[turn];
      turn ^= 1;
      __syncthreads();
      __builtin_amdgcn_s_setprio(2);   // as in the forward kernel
      token_matrices<IO, RK, KT / 2, WAVES, true, true>(sK, sQ, gt, inverse, below, att, scratch, scale, wave, c, g);
      __builtin_amdgcn_s_setprio(0);

      // ---- P = K dS^T
      f4 P[kTiles] = {zero, zero};
#pragma unroll
      for (int s = 0; s < KT / 2; ++s) {
        typename O::A ka[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) ka[i] = O::template rows<RK>(sK, i, s, c, g);
        const typename O::B x = O::pair(S[2 * s], S[2 * s + 1], one);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) P[i] = O::mul(ka[i], x, P[i]);
      }
      __syncthreads();
      if (left > 1) request(t0 - kTok);

      // ---- W, the gradient of v, the state's gradient
      const auto gate4 = [&](const float* from, int tile) { return *reinterpret_cast<const f4*>(from + 16 * tile + 4 * g); };
      static_assert(kTiles == 2, "one pair of token tiles");
      __builtin_amdgcn_s_setprio(1);
      const bool values = !MAP || wave * 16 < DV;      // the columns of the map have no dO
      const float decay = gt.end;
      typename O::Raw d[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) d[i] = values ? O::template tile_raw<RV>(sD, wave, i, c, g) : typename O::Raw{};
      f4 W[kTiles];
      typename O::TB wb[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const f4 rest = gate4(gt.rest, i);
        const typename O::TA inv = O::image(inverse[i], c, g);
        f4 x = rest * P[i];
#pragma unroll
        for (int j = 0; j <= i; ++j) {
          const typename O::TA m = O::image(att[i * (i + 1) / 2 + j], c, g);
          x = O::mul_tok_raw(m, d[j], x);
        }
#pragma unroll
        for (int j = 0; j < i; ++j) {
          const typename O::TA m = O::image(below[i * (i - 1) / 2 + j], c, g);
          x = O::mul_tok(m, wb[j], x);
        }
        W[i] = O::mul_tok(inv, O::tokens(x, one), zero);
        if (i + 1 < kTiles) wb[i] = O::tokens(W[i], one);
      }
      if constexpr (!MAP) {
        const __amdgpu_buffer_rsrc_t rows = rows_buffer(a.rows + (static_cast<size_t>(head) * a.T + t0) * DV, DV * 4, end - t0, DV * 4);
        const __amdgpu_buffer_rsrc_t out = rows_buffer(dv + t0 * dv_step, dv_step, end - t0, DV * static_cast<int>(sizeof(IO)));
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          const int t = kTok - 1 - (16 * i + 4 * g);
          store_column(rows, (t * DV + col()) * 4, -DV * 4, W[i], static_cast<float*>(nullptr));
          store_column(out, t * static_cast<int>(dv_step) + col() * static_cast<int>(sizeof(IO)), -static_cast<int>(dv_step), W[i] * gate4(gt.beta, i),
                       static_cast<IO*>(nullptr));
        }
      }
      f4 e[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const f4 gamma = gate4(gt.gamma, i);
        W[i] *= -gamma * gate4(gt.beta, i);
        e[i] = O::value(d[i]) * (gamma * scale);
      }
      const typename O::B wp = O::pair(W[0], W[1], one), ep = O::pair(e[0], e[1], one);
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const typename O::A kc = O::template columns<RK>(sK, kt, 0, c, g);
        f4 x = O::mul(kc, wp, S[kt] * decay);
        if (values) {
          const typename O::A qc = O::template columns<RK>(sQ, kt, 0, c, g);
          x = O::mul(qc, ep, x);
        }
        S[kt] = x;
      }
      __builtin_amdgcn_s_setprio(0);
      next_gates(t0 - kTok, gates[turn]);
      request_gates(t0 - 2 * kTok);
      __syncthreads();
    }
  }

  // ---- gradients of tokens past the end of the sequence, of the state
  if constexpr (!MAP) {
    for (int t = max(first, end) + wave; t < last; t += WAVES) {
      for (int i = lane; i < DV; i += 64) io_store(reinterpret_cast<IO*>(dv + t * dv_step) + i, 0.0f);
    }
  }
  float* out = nullptr;
  if (MAP) out = a.seg_map + slot * Sh::COLS * DK;
  else if (a.seg_S != nullptr) out = a.seg_S + (slot - 1) * DV * DK;
  else if (a.S_T != nullptr && seg == 0) out = a.S_T + static_cast<size_t>(head) * DV * DK;
  if (out == nullptr) return;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
    if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<uint32_t>(col() * DK + dk)) = S[kt];
  }
}

template <typename IO, int DK, int DV, bool MAP>
__global__ void __launch_bounds__((Shape<DK, DV, MAP>::THREADS), (Shape<DK, DV, MAP>::HELD)) delta_reverse_kernel(DeltaArgs a) {
  if constexpr (MAP) {      // of all segments but the last one on the way
    const int n = a.n_seg - 1, head = blockIdx.x / n, at = blockIdx.x % n, seg = a.n_seg - 1 - at;
    if constexpr (delta_first_with_maps(DV)) {
      if (at == 0 && a.first_done) {
        if (__builtin_amdgcn_readfirstlane(threadIdx.x) < Shape<DK, DV, false>::THREADS) reverse_segment<IO, DK, DV, false>(a, head, seg);
        return;
      }
    }
    reverse_segment<IO, DK, DV, true>(a, head, seg);
  } else {
    const int n = a.n_seg - (a.first_done ? 1 : 0), head = blockIdx.x / n, at = blockIdx.x % n;
    reverse_segment<IO, DK, DV, false>(a, head, at);
  }
}

template <int DK, int DV, bool MAP>
hipError_t launch_reverse(const DeltaArgs& a, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args};
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_reverse_kernel<uint16_t, DK, DV, MAP>)
                                 : reinterpret_cast<const void*>(&delta_reverse_kernel<float, DK, DV, MAP>);
  return hipLaunchKernel(fn, dim3(a.B * a.H_v * (a.n_seg - (MAP || a.first_done ? 1 : 0))), dim3(Shape<DK, DV, MAP>::THREADS), params, 0, stream);
}

template <int DK>
hipError_t launch_reverse_dk(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream) {
  switch (d_v) {
#define VLA_DV(N) case N: return map ? launch_reverse<DK, N, true>(a, io_dtype, stream) : launch_reverse<DK, N, false>(a, io_dtype, stream);
    VLA_DV(16) VLA_DV(32) VLA_DV(64) VLA_DV(96) VLA_DV(128)
#undef VLA_DV
    default: return hipErrorInvalidValue;
  }
}

}  // namespace delta
}  // namespace vla

// The gated delta rule in blocks of 32 tokens (delta_block.h has the mathematics): one workgroup per head (and time segment) goes
// through the blocks with the state on registers.
//
// A wave has 32 rows of S (16 where they do not divide); the four waves of d_v = 128 share the matrices between tokens: they are
// formed once, with the inverses of the diagonal tiles, by different waves at once, beside the products of K and Q with the state.
// Three barriers a block: rows staged, matrices ready, rows no longer needed.
//
// MAP: the affine map of a segment instead of its outputs, S_end = S_start X + Y: Y from d_v columns that start from zero, X from d_k
// columns without values that start from the identity.
#pragma once

#include "delta_block.h"

namespace vla {
namespace delta {

template <int DK, int DV, bool MAP>
struct Shape {
  static constexpr int COLS = DV + (MAP ? DK : 0);
  static constexpr int NT = 1;           // column tiles of a wave
  static constexpr int WAVES = COLS / (16 * NT);
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int DKP = DK < 32 ? 32 : DK;               // key columns in pairs of tiles
  static constexpr int KT = DKP / 16;
};

template <typename IO, int DK, int DV, bool MAP>
__global__ void __launch_bounds__((Shape<DK, DV, MAP>::THREADS), 4) delta_chunk_kernel(DeltaArgs a) {
  using Sh = Shape<DK, DV, MAP>;
  using O = Ops<IO>;
  constexpr int NT = Sh::NT, KT = Sh::KT, WAVES = Sh::WAVES, THREADS = Sh::THREADS;
  constexpr int PK = DK / O::PER16, PV = DV / O::PER16;
  using RK = PieceRows<Sh::DKP / O::PER16>;
  using RV = PieceRows<PV>;
  __shared__ u4 sK[kTok * RK::STRIDE];
  __shared__ u4 sQ[MAP ? 1 : kTok * RK::STRIDE];
  __shared__ u4 sV[kTok * RV::STRIDE];
  __shared__ typename O::Image inverse[kTiles], below[kTiles * (kTiles - 1) / 2], att[MAP ? 1 : kTiles * (kTiles + 1) / 2];
  __shared__ __align__(16) float diagonal[kTiles][16 * 20];
  __shared__ Gates gate_pair[2];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  int c = lane % 16, g = lane / 16;
  const int head = blockIdx.x / a.n_seg, seg = blockIdx.x % a.n_seg;
  const int b = head / a.H_v, h = head % a.H_v, hk = h / (a.H_v / a.H_k);
  const int len = __builtin_amdgcn_readfirstlane(a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T);
  const int first = seg * a.seg_tokens, last = min(a.T, first + a.seg_tokens), end = min(len, last);
  const char* q = reinterpret_cast<const char*>(static_cast<const IO*>(a.q) + b * a.qs.b + hk * a.qs.h);
  const char* k = reinterpret_cast<const char*>(static_cast<const IO*>(a.k) + b * a.ks.b + hk * a.ks.h);
  const char* v = reinterpret_cast<const char*>(static_cast<const IO*>(a.v) + b * a.vs.b + h * a.vs.h);
  char* o = MAP ? nullptr : reinterpret_cast<char*>(static_cast<IO*>(a.o) + b * a.os.b + h * a.os.h);
  const long long q_step = a.qs.t * sizeof(IO), k_step = a.ks.t * sizeof(IO), v_step = a.vs.t * sizeof(IO), o_step = a.os.t * sizeof(IO);
  const float* gp = a.g + b * a.gs.b + h * a.gs.h;
  const float* bp = a.beta + b * a.bs.b + h * a.bs.h;
  const typename O::One one = O::one(c, g);
  const int col0 = wave * 16 * NT + c;      // first column of this lane

  // ---- the state: tile kt holds key columns 32 (kt / 2) + 8 g + 4 (kt % 2) + r
  f4 S[NT][KT];
  const float* S0 = a.S0 ? a.S0 + (static_cast<size_t>(head) * (a.seg_states ? a.n_seg : 1) + (a.seg_states ? seg : 0)) * DV * DK : nullptr;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int col = col0 + 16 * n;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
      S[n][kt] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if ((DK == Sh::DKP || dk < DK) && (!MAP || col < DV) && S0 != nullptr) S[n][kt] = *reinterpret_cast<const f4*>(S0 + static_cast<size_t>(col) * DK + dk);
      if (MAP && col >= DV) {
#pragma unroll
        for (int r = 0; r < 4; ++r) S[n][kt][r] = col - DV == dk + r ? 1.0f : 0.0f;
      }
    }
  }
  if constexpr (Sh::DKP > DK) {            // columns that no row fills
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
  float gate = 0.0f, beta = 0.0f;   // of one token a lane, a block ahead of the rows
  auto request = [&](int t0) {
    stK.load(k, k_step, t0, end);
    if constexpr (!MAP) stQ.load(q, q_step, t0, end);
    stV.load(v, v_step, t0, end);
  };
  auto request_gates = [&](int t0) {
    const int t = min(t0 + (lane & (kTok - 1)), end - 1);
    gate = gp[t * a.gs.t];
    beta = bp[t * a.bs.t];
  };
  auto next_gates = [&](int t0, Gates& to) {
    if (wave == WAVES - 1) put_gates(to, lane, lane, t0 + lane < end ? gate : 0.0f, t0 + lane < end ? beta : 0.0f);
  };
  if (first < end) {
    request_gates(first);
    request(first);
    next_gates(first, gate_pair[0]);
    request_gates(first + kTok);
  }
  int turn = 0;

  for (int t0 = first; t0 < end;) {
    // the state at the start of every 256 tokens; the blocks between two such places in a loop of their own
    if (!MAP && a.kept != nullptr && t0 % kKeep == 0) {
      float* out = a.kept + (static_cast<size_t>(head) * a.n_kept + t0 / kKeep) * DV * DK;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
          if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<size_t>(col0 + 16 * n) * DK + dk) = S[n][kt];
        }
      }
    }
    const int stop = min(end, (t0 / kKeep + 1) * kKeep);
    for (; t0 < stop; t0 += kTok) {
    // the LDS addresses are formed anew in each block: kept over the loop they would take the registers of the state
    asm volatile("" : "+v"(c), "+v"(g));
    stK.template store<RK>(sK);
    if constexpr (!MAP) stQ.template store<RK>(sQ);
    stV.template store<RV>(sV);
    const Gates& gates = gate_pair[turn];
    turn ^= 1;
    __syncthreads();

    // ---- matrices between tokens, tile (i, j), j <= i: transposed products, so that a lane has four tokens j of row i = c
    constexpr int PAIRS = kTiles * (kTiles + 1) / 2;
    for (int job = wave; job < (MAP ? 1 : 2) * PAIRS; job += WAVES) {
      // the diagonal tiles of k k^T first: their inverses take longest
      const bool keys = job < PAIRS;
      int p = keys ? job : job - PAIRS, i, j;
      if (p < kTiles) {
        i = j = p;
      } else {
        p -= kTiles;
        i = 1;
        while (p >= i) p -= i++;
        j = p;
      }
      f4 x = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < KT / 2; ++s) {
        x = O::mul_rows(O::template rows<RK>(sK, j, s, c, g), O::template rows<RK>(keys || MAP ? sK : sQ, i, s, c, g), x);
      }
      const float hi = gates.hi[16 * i + c], lo = gates.lo[16 * i + c];
      const f4 hj = *reinterpret_cast<const f4*>(&gates.hi[16 * j + 4 * g]), lj = *reinterpret_cast<const f4*>(&gates.lo[16 * j + 4 * g]);
      const f4 bj = *reinterpret_cast<const f4*>(&gates.beta[16 * j + 4 * g]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int before = i - j > 0 ? 1 : (keys ? c - (4 * g + r) : c - (4 * g + r) + 1);   // > 0: token j counts for token i
        const float w = bj[r] * __builtin_amdgcn_exp2f((hi - hj[r]) + (lo - lj[r])) * (keys ? -1.0f : a.scale);
        x[r] = before > 0 ? x[r] * w : 0.0f;
      }
      if (keys && i == j) {
        invert_tile<IO>(x, diagonal[i], inverse[i], c, g);
      } else if (keys) {
        O::put(below[i * (i - 1) / 2 + j], c, g, x);
      } else {
        O::put(att[i * (i + 1) / 2 + j], c, g, x);
      }
    }

    // ---- P = K S^T, Q S^T
    f4 P[NT][kTiles], QS[NT][kTiles];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) P[n][i] = QS[n][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int s = 0; s < KT / 2; ++s) {
      typename O::A ka[kTiles], qa[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        ka[i] = O::template rows<RK>(sK, i, s, c, g);
        if constexpr (!MAP) qa[i] = O::template rows<RK>(sQ, i, s, c, g);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const typename O::B x = O::pair(S[n][2 * s], S[n][2 * s + 1], one);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          P[n][i] = O::mul(ka[i], x, P[n][i]);
          if constexpr (!MAP) QS[n][i] = O::mul_out(qa[i], x, QS[n][i]);
        }
      }
    }
    __syncthreads();
    if (t0 + kTok < end) request(t0 + kTok);

    // ---- what is written, the read-out, the state
    const float decay = gates.end;
    f4 R[NT][kTiles];
    typename O::TB rb[NT][kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const f4 gamma = *reinterpret_cast<const f4*>(&gates.gamma[16 * i + 4 * g]);
      const typename O::TA inv = O::image(inverse[i], c, g);
      f4 x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        x[n] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        if (!MAP || wave * 16 * NT + 16 * n < DV) x[n] = O::template tile<RV>(sV, wave * NT + n, i, c, g);
        x[n] -= gamma * P[n][i];
      }
#pragma unroll
      for (int j = 0; j < i; ++j) {
        const typename O::TA m = O::image(below[i * (i - 1) / 2 + j], c, g);
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n] = O::mul_tok(m, rb[n][j], x[n]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        R[n][i] = O::mul_tok(inv, O::tokens(x[n], one), f4{0.0f, 0.0f, 0.0f, 0.0f});
        if (!MAP || i + 1 < kTiles) rb[n][i] = O::tokens(R[n][i], one);
      }
    }
    if (!MAP && a.rows != nullptr) {
      const __amdgpu_buffer_rsrc_t out = rows_buffer(a.rows + (static_cast<size_t>(head) * a.T + t0) * DV, DV * 4, last - t0, DV * 4);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
#pragma unroll
        for (int n = 0; n < NT; ++n) store_column(out, ((16 * i + 4 * g) * DV + col0 + 16 * n) * 4, DV * 4, R[n][i], static_cast<float*>(nullptr));
      }
    }
    typename O::B w[NT];
    static_assert(kTiles == 2, "one pair of token tiles");
    {
      const f4 w0 = *reinterpret_cast<const f4*>(&gates.rest[4 * g]) * *reinterpret_cast<const f4*>(&gates.beta[4 * g]);
      const f4 w1 = *reinterpret_cast<const f4*>(&gates.rest[16 + 4 * g]) * *reinterpret_cast<const f4*>(&gates.beta[16 + 4 * g]);
#pragma unroll
      for (int n = 0; n < NT; ++n) w[n] = O::pair(R[n][0] * w0, R[n][1] * w1, one);
    }
    if constexpr (!MAP) {
      const __amdgpu_buffer_rsrc_t out = rows_buffer(o + t0 * o_step, o_step, last - t0, DV * static_cast<int>(sizeof(IO)));
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const f4 gamma = *reinterpret_cast<const f4*>(&gates.gamma[16 * i + 4 * g]) * a.scale;
        f4 x[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n] = gamma * QS[n][i];
#pragma unroll
        for (int j = 0; j <= i; ++j) {
          const typename O::TA m = O::image(att[i * (i + 1) / 2 + j], c, g);
#pragma unroll
          for (int n = 0; n < NT; ++n) x[n] = O::mul_tok_out(m, rb[n][j], x[n]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          store_column(out, (16 * i + 4 * g) * static_cast<int>(o_step) + (col0 + 16 * n) * static_cast<int>(sizeof(IO)), static_cast<int>(o_step), x[n],
                       static_cast<IO*>(nullptr));
        }
      }
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const typename O::A kc = O::template columns<RK>(sK, kt, 0, c, g);
#pragma unroll
      for (int n = 0; n < NT; ++n) S[n][kt] = O::mul(kc, w[n], S[n][kt] * decay);
    }
    next_gates(t0 + kTok, gate_pair[turn]);
    request_gates(t0 + 2 * kTok);
    __syncthreads();
    }
  }

  // ---- outputs of tokens past the end of the sequence, the state
  if constexpr (!MAP) {
    const int done = first < end ? first + (end - first + kTok - 1) / kTok * kTok : first;
    for (int t = done + wave; t < last; t += WAVES) {
      for (int i = lane; i < DV; i += 64) io_store(reinterpret_cast<IO*>(o + t * o_step) + i, 0.0f);
    }
  }
  float* out = nullptr;
  if (MAP) out = a.seg_map + (static_cast<size_t>(head) * a.n_seg + seg) * Sh::COLS * DK;
  else if (a.S_T != nullptr && seg == a.n_seg - 1) out = a.S_T + static_cast<size_t>(head) * DV * DK;
  if (out == nullptr) return;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const int dk = 32 * (kt / 2) + 8 * g + 4 * (kt % 2);
      if (DK == Sh::DKP || dk < DK) *reinterpret_cast<f4*>(out + static_cast<size_t>(col0 + 16 * n) * DK + dk) = S[n][kt];
    }
  }
}

template <int DK, int DV, bool MAP>
hipError_t launch_chunk(const DeltaArgs& a, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args};
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_chunk_kernel<uint16_t, DK, DV, MAP>)
                                 : reinterpret_cast<const void*>(&delta_chunk_kernel<float, DK, DV, MAP>);
  return hipLaunchKernel(fn, dim3(a.B * a.H_v * a.n_seg), dim3(Shape<DK, DV, MAP>::THREADS), params, 0, stream);
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

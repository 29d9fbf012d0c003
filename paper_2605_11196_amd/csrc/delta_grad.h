// The gradients of q, k, g and beta of the gated delta rule: one workgroup for every 256 tokens of a head, from the state at their start
// (kept by the forward pass), its gradient at their end, and R and W of every token (beta R is what a token writes, beta W the gradient
// of v; delta_reverse.h forms W).  Of a block of 32 tokens, S the state at its start, dS its gradient at the end:
//   X = scale D * (dO R^T) beta_j, j <= i;   Y = -D * (W R^T) beta_i beta_j, j < i
//   dQ = scale gamma (dO S) + X K
//   dK = X^T Q + (Y + Y^T) K - gamma beta (W S) + exp(G_end - G) beta (R dS)
//   dbeta_i = W_i . R_i
//   dg_t = sum over the tokens i >= t of (dO_i . O_i - v_i . dV_i), up to any later place, + <dS, S> there
// The last line: the loss does not change when the state and all that is written later grow by a factor and all that is read shrinks by it;
// so the gradient of a decay is <dS, S> right behind it, and between two places that differs by what the tokens read and write.  dO . O = q . dQ.
// A decay of 0 ends the sums, with 0.
//
// A sweep along the tokens carries S (everything but the last term of dK), a sweep back carries dS.  Here a wave has 16 columns of what has
// d_k columns, so that the products over d_v stay in it; states are tiles with d_v along the rows, left operands the rows of dO, R and W in
// LDS.  Twice the forward kernel's products; bound by memory and the waits for it, since both sweeps read K, Q, dO, R and W
// (64 heads of 128, 4096 tokens, bf16: 396 us, 1.5 GB, the waves wait 54 % of their cycles).  Nothing is added atomically.
#pragma once

#include "delta_block.h"

namespace vla {
namespace delta {

template <typename IO, int DK, int DV>
__global__ void __launch_bounds__(4 * DK, 4) delta_grad_kernel(DeltaArgs a) {
  using O = Ops<IO>;
  constexpr int WAVES = DK / 16, THREADS = 64 * WAVES;
  constexpr int DKP = DK < 32 ? 32 : DK, DVP = DV < 32 ? 32 : DV, VT = DVP / 16;
  constexpr int PK = DK / O::PER16, PV = DV / O::PER16;
  using RK = PieceRows<DKP / O::PER16>;
  using RV = PieceRows<DVP / O::PER16>;
  // Terms of R and of W.  W enters dK alone (dbeta and v . dV read it from memory), so 16 bits of it: the third term's 8 KB at d_v = 128 would leave one
  // workgroup on a compute unit instead of two.
  constexpr int TR = O::TERMS, TW = O::TERMS > 1 ? 2 : 1;
  __shared__ u4 sK[kTok * RK::STRIDE], sQ[kTok * RK::STRIDE], sD[kTok * RV::STRIDE], sR[TR * kTok * RV::STRIDE], sW[TW * kTok * RV::STRIDE];
  __shared__ typename O::Image X[3];                 // tiles (0,0), (1,0), (1,1)
  __shared__ typename O::ImageOut Xt[3], Z[4];       // X^T: (0,0), (0,1), (1,1);  Y + Y^T: (0,0), (0,1), (1,0), (1,1)
  __shared__ Gates gates;
  __shared__ float reads[WAVES][kTok], change[kKeep], whole[WAVES];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  int c = lane % 16, g = lane / 16;
  const int segs = (a.T + kKeep - 1) / kKeep, head = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int b = head / a.H_v, h = head % a.H_v, hk = h / (a.H_v / a.H_k);
  const int len = __builtin_amdgcn_readfirstlane(a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T);
  const int first = seg * kKeep, last = min(a.T, first + kKeep), end = min(len, last);
  const char* q = reinterpret_cast<const char*>(static_cast<const IO*>(a.q) + b * a.qs.b + hk * a.qs.h);
  const char* k = reinterpret_cast<const char*>(static_cast<const IO*>(a.k) + b * a.ks.b + hk * a.ks.h);
  const char* v = reinterpret_cast<const char*>(static_cast<const IO*>(a.v) + b * a.vs.b + h * a.vs.h);
  const char* dO = reinterpret_cast<const char*>(static_cast<const IO*>(a.dO) + b * a.os.b + h * a.os.h);
  const long long q_step = a.qs.t * sizeof(IO), k_step = a.ks.t * sizeof(IO), o_step = a.os.t * sizeof(IO), v_step = a.vs.t * sizeof(IO);
  const float* gp = a.g + b * a.gs.b + h * a.gs.h;
  const float* bp = a.beta + b * a.bs.b + h * a.bs.h;
  const size_t row0 = static_cast<size_t>(head) * a.T;
  const bool shared = a.dq_part != nullptr;
  char* dq = reinterpret_cast<char*>(static_cast<IO*>(a.dq) + b * a.dqs.b + hk * a.dqs.h);
  char* dk = reinterpret_cast<char*>(static_cast<IO*>(a.dk) + b * a.dks.b + hk * a.dks.h);
  const typename O::One one = O::one(c, g);
  const int col = wave * 16 + c;

  if constexpr (DKP > DK) {
    for (int i = threadIdx.x; i < kTok * RK::STRIDE; i += THREADS) sK[i] = sQ[i] = u4{0, 0, 0, 0};
  }
  if constexpr (DVP > DV) {
    for (int i = threadIdx.x; i < kTok * RV::STRIDE; i += THREADS) sD[i] = u4{0, 0, 0, 0};
    for (int i = threadIdx.x; i < TR * kTok * RV::STRIDE; i += THREADS) sR[i] = u4{0, 0, 0, 0};
    for (int i = threadIdx.x; i < TW * kTok * RV::STRIDE; i += THREADS) sW[i] = u4{0, 0, 0, 0};
  }
  if constexpr (DKP > DK || DVP > DV) __syncthreads();

  // tile vt of a state: rows 32 (vt / 2) + 8 g + 4 (vt % 2) + r
  auto load_state = [&](const float* from, f4 (&S)[VT]) {
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) {
      const int row = 32 * (vt / 2) + 8 * g + 4 * (vt % 2);
#pragma unroll
      for (int r = 0; r < 4; ++r) S[vt][r] = DV == DVP || row + r < DV ? from[static_cast<size_t>(row + r) * DK + col] : 0.0f;
    }
  };
  // the rows of a block on their way from memory to LDS, a block ahead where the state leaves the registers for it (d_v = 64: 118 -> 97 us for
  // 128 heads of 1024 tokens; d_v = 128 would keep 140 bytes a lane in scratch memory: 420 -> 540 us for 64 heads of 4096)
  constexpr bool AHEAD = DV <= 64;
  Stage<PK, THREADS> stK, stQ;
  Stage<PV, THREADS> stD;
  constexpr int ROWS4 = kTok * DV / 4, NR = (ROWS4 + THREADS - 1) / THREADS;
  f4 stR[NR], stW[NR];                      // four columns of R and W, rows one after the other
  stK.init(k_step);
  stQ.init(q_step);
  stD.init(o_step);
  float gate = 0.0f, beta = 0.0f;
  auto request = [&](int t0) {
    stK.load(k, k_step, t0, end);
    stQ.load(q, q_step, t0, end);
    stD.load(dO, o_step, t0, end);
    const __amdgpu_buffer_rsrc_t R = rows_buffer(a.R + (row0 + t0) * DV, DV * 4, end - t0, DV * 4);
    const __amdgpu_buffer_rsrc_t W = rows_buffer(a.rows + (row0 + t0) * DV, DV * 4, end - t0, DV * 4);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int p = threadIdx.x + i * THREADS;
      stR[i] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(R, p * 16, 0, 0));
      stW[i] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(W, p * 16, 0, 0));
    }
    const int t = min(t0 + (lane & (kTok - 1)), end - 1);
    gate = gp[t * a.gs.t];
    beta = bp[t * a.bs.t];
  };
  auto stage = [&](int t0) {
    stK.template store<RK>(sK);
    stQ.template store<RK>(sQ);
    stD.template store<RV>(sD);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int p = threadIdx.x + i * THREADS, row = p / (DV / 4), piece = p % (DV / 4);
      const f4 r = stR[i], w = stW[i];
      if (ROWS4 % THREADS == 0 || p < ROWS4) {
        O::template put_split<TR, RV>(sR, row, piece, r);
        O::template put_split<TW, RV>(sW, row, piece, w);
      }
    }
    if (wave == WAVES - 1) put_gates(gates, lane, lane, t0 + lane < end ? gate : 0.0f, t0 + lane < end ? beta : 0.0f);
  };
  const f4 zero = f4{0.0f, 0.0f, 0.0f, 0.0f};
  auto gate4 = [&](const float* from, int tile) { return *reinterpret_cast<const f4*>(from + 16 * tile + 4 * g); };

  f4 S[VT];
  load_state(a.kept_state + (static_cast<size_t>(head) * segs + seg) * DV * DK, S);
  if (first >= end) {
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) S[vt] = zero;
  }
  if (AHEAD && first < end) request(first);
  for (int t0 = first; t0 < end; t0 += kTok) {
    asm volatile("" : "+v"(c), "+v"(g));
    if (!AHEAD) request(t0);
    // the values of W, R and v that the sums of a token take, with the rows: asked for after them they took a third of the kernel
    struct {
      float w[DV / 16], r[DV / 16];
      IO y[DV / 16];
    } dots;
    auto request_dots = [&](int i) {
      const int t = min(t0 + i, end - 1), x = threadIdx.x % 16;
      const float* W = a.rows + (row0 + t) * DV + x;
      const float* R = a.R + (row0 + t) * DV + x;
      const IO* values = reinterpret_cast<const IO*>(v + t * v_step) + x;
#pragma unroll
      for (int n = 0; n < DV / 16; ++n) {
        dots.w[n] = W[16 * n];
        dots.r[n] = R[16 * n];
        dots.y[n] = values[16 * n];
      }
    };
    request_dots(threadIdx.x / 16);
    stage(t0);
    __syncthreads();

    // ---- dbeta and v . dV of a token for each 16 lanes
    for (int i = threadIdx.x / 16; i < kTok; i += THREADS / 16) {
      if (i >= THREADS / 16) request_dots(i);
      float wr = 0.0f, wv = 0.0f;
#pragma unroll
      for (int n = 0; n < DV / 16; ++n) {
        wr = fmaf(dots.w[n], dots.r[n], wr);
        wv = fmaf(dots.w[n], widen(dots.y[n]), wv);
      }
      wr = row_sum16(wr);
      wv = row_sum16(wv);
      if (threadIdx.x % 16 == 0) {
        if (t0 + i < last) a.dbeta[row0 + t0 + i] = t0 + i < end ? wr : 0.0f;
        change[t0 + i - first] = t0 + i < end ? -gates.beta[i] * wv : 0.0f;
      }
    }
    // ---- matrices between tokens
    // 0, 1: Z (0,0) and (1,1), twice the work of the others; 2-4: X (0,0), (1,0), (1,1); 5-7: X^T of the same; 8: Z (1,0), 9: Z (0,1)
    for (int round = 0; round * WAVES < 10; ++round) {
      const int order = job_of(round, wave, WAVES);
      if (order >= 10) continue;
      const int kind = order < 2 ? 4 : (order < 5 ? 0 : (order < 8 ? 1 : order - 6));
      const int tile = order < 2 ? 2 * order : (order < 8 ? (order - 2) % 3 : 1);
      const int i = tile > 0 ? 1 : 0, j = tile > 1 ? 1 : 0;       // row tile i, column tile j of X and Y
      // x: rows j = 4 g + r of tile j, column i = c of tile i; y: rows i, column j
      const bool writes = kind >= 2;          // Y and not X
      f4 x = zero, y = zero;
#pragma unroll
      for (int s = 0; s < DVP / 32; ++s) {
        const typename O::Split rj = O::template rows_split<TR, RV>(sR, j, s, c, g);
        if (!writes) {
          const typename O::A di = O::template rows<RV>(sD, i, s, c, g);
          if (kind == 0) x = O::mul_split_exact(rj, di, x);
          else y = O::mul(di, rj, y);
        } else {
          const typename O::Split wi = O::template rows_split<TW, RV>(sW, i, s, c, g);
          if (kind != 3) x = O::mul_split_out(rj, wi, x);
          if (kind != 2) y = O::mul_split_out(wi, rj, y);
        }
      }
      if (kind % 2 == 0) {
        const float hi = gates.hi[16 * i + c], lo = gates.lo[16 * i + c], factor = writes ? -gates.beta[16 * i + c] : a.scale;
        const f4 hj = gate4(gates.hi, j), lj = gate4(gates.lo, j), bj = gate4(gates.beta, j);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int before = i > j ? 1 : c - (4 * g + r) + (writes ? 0 : 1);
          x[r] = before > 0 ? x[r] * (__builtin_amdgcn_exp2f((hi - hj[r]) + (lo - lj[r])) * bj[r] * factor) : 0.0f;
        }
      }
      if (kind == 1 || kind >= 3) {
        const float hj = gates.hi[16 * j + c], lj = gates.lo[16 * j + c], bj = gates.beta[16 * j + c];
        const f4 hi = gate4(gates.hi, i), lo = gate4(gates.lo, i), bi = gate4(gates.beta, i);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int before = i > j ? 1 : (4 * g + r) - c + (writes ? 0 : 1);
          y[r] = before > 0 ? y[r] * (__builtin_amdgcn_exp2f((hi[r] - hj) + (lo[r] - lj)) * bj * (writes ? -bi[r] : a.scale)) : 0.0f;
        }
      }
      if (kind == 0) O::put(X[tile], c, g, x);
      else if (kind == 1) O::put(Xt[tile], c, g, y);
      else if (kind == 2) O::put(Z[2], c, g, x);
      else if (kind == 3) O::put(Z[1], c, g, y);
      else O::put(Z[3 * i], c, g, x + y);
    }

    // ---- products with the state
    f4 dQ[kTiles] = {zero, zero}, dK[kTiles] = {zero, zero};
#pragma unroll
    for (int s = 0; s < VT / 2; ++s) {
      const typename O::B x = O::pair(S[2 * s], S[2 * s + 1], one);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        dQ[i] = O::mul(O::template rows<RV>(sD, i, s, c, g), x, dQ[i]);
        dK[i] = O::mul_split_out(O::template rows_split<TW, RV>(sW, i, s, c, g), x, dK[i]);
      }
    }
    typename O::Raw kr[kTiles], qr[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      kr[i] = O::template tile_raw<RK>(sK, wave, i, c, g);
      qr[i] = O::template tile_raw<RK>(sQ, wave, i, c, g);
      dQ[i] *= gate4(gates.gamma, i) * a.scale;
      dK[i] *= -gate4(gates.gamma, i) * gate4(gates.beta, i);
    }
    __syncthreads();
    dQ[0] = O::mul_tok_raw(O::image(X[0], c, g), kr[0], dQ[0]);
    dQ[1] = O::mul_tok_raw(O::image(X[2], c, g), kr[1], O::mul_tok_raw(O::image(X[1], c, g), kr[0], dQ[1]));
    dK[0] = O::mul_tok_raw(O::image(Xt[1], c, g), qr[1], O::mul_tok_raw(O::image(Xt[0], c, g), qr[0], dK[0]));
    dK[1] = O::mul_tok_raw(O::image(Xt[2], c, g), qr[1], dK[1]);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j) dK[i] = O::mul_tok_raw(O::image(Z[2 * i + j], c, g), kr[j], dK[i]);
    }
    {
      const __amdgpu_buffer_rsrc_t part = rows_buffer(a.dk_part + (row0 + t0) * DK, DK * 4, end - t0, DK * 4);
      const __amdgpu_buffer_rsrc_t qpart = rows_buffer(a.dq_part + (row0 + t0) * DK, DK * 4, shared ? end - t0 : 0, DK * 4);
      const __amdgpu_buffer_rsrc_t out = rows_buffer(dq + t0 * a.dqs.t * sizeof(IO), a.dqs.t * sizeof(IO), shared ? 0 : end - t0, DK * static_cast<int>(sizeof(IO)));
      const int step = static_cast<int>(a.dqs.t * sizeof(IO));
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const int t = 16 * i + 4 * g;
        if (shared) store_column(qpart, (t * DK + col) * 4, DK * 4, dQ[i], static_cast<float*>(nullptr));
        else store_column(out, t * step + col * static_cast<int>(sizeof(IO)), step, dQ[i], static_cast<IO*>(nullptr));
        store_column(part, (t * DK + col) * 4, DK * 4, dK[i], static_cast<float*>(nullptr));
        const f4 qv = O::value(qr[i]) * dQ[i];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float sum = row_sum16(qv[r]);
          if (c == 0) reads[wave][t + r] = sum;
        }
      }
    }
    const float decay = gates.end;
    const typename O::B x = O::pair(O::value(kr[0]) * (gate4(gates.rest, 0) * gate4(gates.beta, 0)),
                                    O::value(kr[1]) * (gate4(gates.rest, 1) * gate4(gates.beta, 1)), one);
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) S[vt] = O::mul_split(O::template columns_split<TR, RV>(sR, vt, 0, c, g), x, S[vt] * decay);
    if (AHEAD && t0 + kTok < end) request(t0 + kTok);
    __syncthreads();
    if (threadIdx.x < kTok) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += reads[w][threadIdx.x];
      change[t0 - first + threadIdx.x] += sum;
    }
  }

  // ---- back along the tokens with the state's gradient, from the kept one at their end.  What is carried over up to eight blocks is for dK alone, so its
  // updates are formed from 16 bits of their factors as well (of each 2^-17, against the 2^-9 that dK is rounded to).
  {
    f4 dS[VT];
    load_state(a.kept + (static_cast<size_t>(head) * segs + seg) * DV * DK, dS);
    float dot = 0.0f;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) {
#pragma unroll
      for (int r = 0; r < 4; ++r) dot = fmaf(dS[vt][r], S[vt][r], dot);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) dot += __shfl_xor(dot, d, 64);
    if (lane == 0) whole[wave] = dot;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) S[vt] = dS[vt];
  }
  const int start = first + max(0, (end - first - 1)) / kTok * kTok;
  for (int t0 = start; t0 >= first && first < end; t0 -= kTok) {
    asm volatile("" : "+v"(c), "+v"(g));
    if (t0 != start) {      // the last block is still staged
      if (!AHEAD) request(t0);
      stage(t0);
      __syncthreads();
    }
    if (AHEAD && t0 > first) request(t0 - kTok);
    f4 dK[kTiles] = {zero, zero};
#pragma unroll
    for (int s = 0; s < VT / 2; ++s) {
      const typename O::B x = O::pair(S[2 * s], S[2 * s + 1], one);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) dK[i] = O::mul_split_out(O::template rows_split<TW, RV>(sR, i, s, c, g), x, dK[i]);
    }
    const __amdgpu_buffer_rsrc_t part = rows_buffer(a.dk_part + (row0 + t0) * DK, DK * 4, end - t0, DK * 4);
    const __amdgpu_buffer_rsrc_t out = rows_buffer(dk + t0 * a.dks.t * sizeof(IO), a.dks.t * sizeof(IO), end - t0, DK * static_cast<int>(sizeof(IO)));
    const int step = static_cast<int>(a.dks.t * sizeof(IO));
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int t = 16 * i + 4 * g;
      f4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(part, ((t + r) * DK + col) * 4, 0, 0));
      x += dK[i] * (gate4(gates.rest, i) * gate4(gates.beta, i));
      if (shared) store_column(part, (t * DK + col) * 4, DK * 4, x, static_cast<float*>(nullptr));
      else store_column(out, t * step + col * static_cast<int>(sizeof(IO)), step, x, static_cast<IO*>(nullptr));
    }
    const float decay = gates.end;
    const f4 g0 = gate4(gates.gamma, 0), g1 = gate4(gates.gamma, 1);
    const typename O::B qx = O::pair(O::template tile<RK>(sQ, wave, 0, c, g) * (g0 * a.scale), O::template tile<RK>(sQ, wave, 1, c, g) * (g1 * a.scale), one);
    const typename O::B kx = O::pair(O::template tile<RK>(sK, wave, 0, c, g) * (-g0 * gate4(gates.beta, 0)),
                                     O::template tile<RK>(sK, wave, 1, c, g) * (-g1 * gate4(gates.beta, 1)), one);
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) {
      f4 x = O::mul_split_out(O::template columns_split<TW, RV>(sW, vt, 0, c, g), kx, S[vt] * decay);
      S[vt] = O::mul_out(O::template columns<RV>(sD, vt, 0, c, g), qx, x);
    }
    __syncthreads();
  }

  // ---- the decays' gradients: sums from the end of the 256 tokens in float64.  Past a decay that is 0 in float32 nothing counts: its own gradient
  // and what lies behind it add up to 0, but their rounding would not.
  __syncthreads();
  if (wave == 0) {
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += static_cast<double>(whole[w]);
    constexpr int EACH = kKeep / 64;
    constexpr float kForgets = -104.0f;      // exp of less is below half of the smallest float32 number
    double sum[EACH], tail = 0.0;
    int cut = 0, cuts[EACH];                 // whether a token from here to the lane's last one forgets the state
#pragma unroll
    for (int i = EACH - 1; i >= 0; --i) {
      const int t = first + EACH * lane + i;
      if (t < end) {
        tail += static_cast<double>(change[t - first]);
        if (gp[t * a.gs.t] < kForgets) {
          tail = 0.0;
          cut = 1;
        }
      }
      sum[i] = tail;
      cuts[i] = cut;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {        // of the lanes from here on, up to the first that cuts
      const double other = __shfl_down(tail, d, 64);
      const int other_cut = __shfl_down(cut, d, 64);
      if (lane + d < 64 && !cut) {
        tail += other;
        cut = other_cut;
      }
    }
    double later = __shfl_down(tail, 1, 64);
    if (lane == 63) later = 0.0;
    if (__shfl_down(cut, 1, 64) == 0 || lane == 63) later += all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int t = first + EACH * lane + i;
      if (t < last) a.dg[row0 + t] = t < end ? static_cast<float>(cuts[i] ? sum[i] : sum[i] + later) : 0.0f;
    }
  }
  // ---- tokens past the end of the sequence
  for (int t = max(first, end) + static_cast<int>(threadIdx.x) / 16; t < last; t += THREADS / 16) {
    for (int x = threadIdx.x % 16; x < DK; x += 16) {
      if (shared) {
        a.dq_part[(row0 + t) * DK + x] = 0.0f;
        a.dk_part[(row0 + t) * DK + x] = 0.0f;
      } else {
        io_store(reinterpret_cast<IO*>(dq) + t * a.dqs.t + x, 0.0f);
        io_store(reinterpret_cast<IO*>(dk) + t * a.dks.t + x, 0.0f);
      }
    }
    if (threadIdx.x % 16 == 0) a.dbeta[row0 + t] = 0.0f;
  }
}

template <int DK, int DV>
hipError_t launch_grad(const DeltaArgs& a, int io_dtype, hipStream_t stream) {
  DeltaArgs args = a;
  void* params[] = {&args};
  const void* fn = io_dtype == 1 ? reinterpret_cast<const void*>(&delta_grad_kernel<uint16_t, DK, DV>)
                                 : reinterpret_cast<const void*>(&delta_grad_kernel<float, DK, DV>);
  return hipLaunchKernel(fn, dim3(a.B * a.H_v * ((a.T + kKeep - 1) / kKeep)), dim3(4 * DK), params, 0, stream);
}

template <int DK>
hipError_t launch_grad_dk(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream) {
  switch (d_v) {
    case 16: return launch_grad<DK, 16>(a, io_dtype, stream);
    case 32: return launch_grad<DK, 32>(a, io_dtype, stream);
    case 64: return launch_grad<DK, 64>(a, io_dtype, stream);
    case 96: return launch_grad<DK, 96>(a, io_dtype, stream);
    case 128: return launch_grad<DK, 128>(a, io_dtype, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace delta
}  // namespace vla

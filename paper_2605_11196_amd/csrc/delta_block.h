// Building blocks of the gated delta rule's block form: a block of 32 tokens on the matrix unit (forward and backward kernels).
//
// Mathematics of a block (tokens i, j of it; G the running sum of g, gamma = exp(G), D_ij = exp(G_i - G_j), S the state at its start):
//   P = K S^T;   (I + M) R = V - gamma P,  M_ij = D_ij (k_i . k_j) beta_j for j < i;   the writes are beta R
//   O = scale gamma (Q S^T) + A R,  A_ij = scale D_ij (q_i . k_j) beta_j for j <= i
//   S <- gamma_end S + (exp(G_end - G) beta R)^T K
// I + M is solved by tiles of 16 tokens, with the inverses of the diagonal tiles by substitution (stable for keys that repeat, which
// powers of M are not).
//
// Layout.  A wave holds its columns (rows of S, 16 for each tile) of everything that has d_v columns, transposed: accumulator tiles with
// tokens or key columns along the rows (4 g + r) and d_v along the 16 lanes.  Such a tile is the right operand of the next product as it
// stands, because the order of the contraction is free: row 4 g + r of the two tiles of a pair is slot r (4 + r) of lane group g.  For a
// contraction over key columns slot i of group g is column 32 j + 8 g + i, so that rows of K and Q lie in LDS as they lie in memory, in
// 16-byte pieces whose place in a row is turned by the row (banks).  No value of a wave's columns ever leaves the wave.
//
// Precision.  bf16: K, Q, V and dO are exact operands, the state and the writes three bf16 terms (all 24 bits); matrices between tokens
// six of nine products of three terms each.  float32: the FP32 matrix instruction.
#pragma once

#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace delta {

constexpr int kTok = 32;          // tokens of a block
constexpr int kTiles = kTok / 16;

__host__ __device__ constexpr int pow2_at_least(int n) { return n <= 1 ? 1 : 2 * pow2_at_least((n + 1) / 2); }

// Rows of 16-byte pieces in LDS, PIECES used of a row.
template <int PIECES>
struct PieceRows {
  static constexpr int STRIDE = pow2_at_least(PIECES < 4 ? 4 : PIECES);
  static __device__ __forceinline__ int at(int row, int piece) {
    const int turn = STRIDE >= 16 ? (row & 15) : ((row / (16 / STRIDE)) & (STRIDE - 1));
    return row * STRIDE + (piece ^ turn);
  }
};

typedef short s4v __attribute__((ext_vector_type(4)));

// four rows' values of one column for each lane of 16 (bf16): lane i gives the address of four columns of row i / 4
__device__ __forceinline__ u2 read_transposed(const u4* base, int piece_at, int half) {
  typedef __attribute__((address_space(3))) s4v lds_s4;
  const char* p = reinterpret_cast<const char*>(base + piece_at) + 8 * half;
  return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p)));
}
__device__ __forceinline__ f4 widen4(u2 b) {
  return f4{__uint_as_float(b[0] << 16), __uint_as_float(b[0] & 0xffff0000u), __uint_as_float(b[1] << 16),
            __uint_as_float(b[1] & 0xffff0000u)};
}

template <typename IO> struct Ops;

// bf16 numbers, products on the bf16 matrix instruction
template <> struct Ops<uint16_t> {
  static constexpr int PER16 = 8;            // values of a piece
  using A = u4;                              // 32 columns of a row, exact
  using B = Terms<3>;                        // 32 rows of a tile pair
  struct Image { u4 hm[64]; u2 l[64]; };     // a 16 x 16 matrix between tokens as a left operand
  using TA = TokA;
  using TB = TokB;
  template <class R> static __device__ __forceinline__ A rows(const u4* m, int row, int j, int g) { return m[R::at(row, 4 * j + g)]; }
  static __device__ __forceinline__ f4 mul_rows(A a, A b, f4 acc) { return mfma_bf16(a, b, acc); }
  static __device__ __forceinline__ B pair(f4 x0, f4 x1) { return split_tiles(x0, x1); }
  static __device__ __forceinline__ f4 mul(A a, const B& b, f4 acc) { return mfma_terms(Terms<1>{{a}}, b, acc); }
  // without the lowest term: for results that are rounded to bf16
  static __device__ __forceinline__ f4 mul_out(A a, const B& b, f4 acc) { return mfma_bf16(a, b.t[0], mfma_bf16(a, b.t[1], acc)); }
  // rows of the state's tile kt (m = key column 32 (kt / 2) + 8 (m / 4) + 4 (kt % 2) + m % 4) against the tokens of tiles t and t + 1
  template <class R> static __device__ __forceinline__ A columns(const u4* m, int kt, int t, int c, int g) {
    const int piece = 4 * (kt / 2) + c % 4, row = 16 * t + 4 * g + c / 4;
    return cat(read_transposed(m, R::at(row, piece), kt % 2), read_transposed(m, R::at(row + 16, piece), kt % 2));
  }
  // accumulator tile of columns 16 n + lane, tokens of tile t; exact
  template <class R> static __device__ __forceinline__ u2 tile_raw(const u4* m, int n, int t, int c, int g) {
    return read_transposed(m, R::at(16 * t + 4 * g + c / 4, 2 * n + (c % 4) / 2), c % 2);
  }
  template <class R> static __device__ __forceinline__ f4 tile(const u4* m, int n, int t, int c, int g) { return widen4(tile_raw<R>(m, n, t, c, g)); }
  static __device__ __forceinline__ void put(Image& im, int row, int g, f4 x) { tok_store(im.hm, im.l, row, row, g, x); }
  static __device__ __forceinline__ TA image(const Image& im, int c, int g) { return tok_load(im.hm, im.l, c, c, g); }
  static __device__ __forceinline__ TB tokens(f4 x) { return tok_b(x); }
  static __device__ __forceinline__ f4 mul_tok(const TA& a, const TB& b, f4 acc) { return mfma_tok(a, b, acc); }
  static __device__ __forceinline__ f4 mul_tok_out(const TA& a, const TB& b, f4 acc) {
    return mfma_bf16(a.hm, b.hm, mfma_bf16(a.hm, b.mh, acc));
  }
};

// float32 numbers, products on the FP32 matrix instruction
template <> struct Ops<float> {
  static constexpr int PER16 = 4;
  struct A { f4 x0, x1; };
  struct B { f4 x0, x1; };
  struct Image { f4 x[64]; };
  using TA = f4;
  using TB = f4;
  static __device__ __forceinline__ f4 mul4(f4 a, f4 b, f4 acc) {
#pragma unroll
    for (int r = 0; r < 4; ++r) acc = mfma16(a[r], b[r], acc);
    return acc;
  }
  template <class R> static __device__ __forceinline__ A rows(const u4* m, int row, int j, int g) {
    return A{__builtin_bit_cast(f4, m[R::at(row, 8 * j + 2 * g)]), __builtin_bit_cast(f4, m[R::at(row, 8 * j + 2 * g + 1)])};
  }
  static __device__ __forceinline__ f4 mul_rows(const A& a, const A& b, f4 acc) { return mul4(a.x1, b.x1, mul4(a.x0, b.x0, acc)); }
  static __device__ __forceinline__ B pair(f4 x0, f4 x1) { return B{x0, x1}; }
  static __device__ __forceinline__ f4 mul(const A& a, const B& b, f4 acc) { return mul4(a.x1, b.x1, mul4(a.x0, b.x0, acc)); }
  static __device__ __forceinline__ f4 mul_out(const A& a, const B& b, f4 acc) { return mul(a, b, acc); }
  static __device__ __forceinline__ float value(const u4* m, int piece_at, int i) { return reinterpret_cast<const float*>(m + piece_at)[i]; }
  template <class R> static __device__ __forceinline__ A columns(const u4* m, int kt, int t, int c, int g) {
    A a;
    const int piece = 8 * (kt / 2) + 2 * (c / 4) + kt % 2, row = 16 * t + 4 * g;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      a.x0[r] = value(m, R::at(row + r, piece), c % 4);
      a.x1[r] = value(m, R::at(row + 16 + r, piece), c % 4);
    }
    return a;
  }
  template <class R> static __device__ __forceinline__ f4 tile(const u4* m, int n, int t, int c, int g) {
    f4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = value(m, R::at(16 * t + 4 * g + r, 4 * n + c / 4), c % 4);
    return x;
  }
  template <class R> static __device__ __forceinline__ f4 tile_raw(const u4* m, int n, int t, int c, int g) { return tile<R>(m, n, t, c, g); }
  static __device__ __forceinline__ void put(Image& im, int row, int g, f4 x) { im.x[4 * row + tok_chunk(row, g)] = x; }
  static __device__ __forceinline__ TA image(const Image& im, int c, int g) { return im.x[4 * c + tok_chunk(c, g)]; }
  static __device__ __forceinline__ TB tokens(f4 x) { return x; }
  static __device__ __forceinline__ f4 mul_tok(const TA& a, const TB& b, f4 acc) { return mul4(a, b, acc); }
  static __device__ __forceinline__ f4 mul_tok_out(const TA& a, const TB& b, f4 acc) { return mul4(a, b, acc); }
};

// A block's rows on their way from memory to LDS: N pieces a thread.
template <int PIECES, int THREADS>
struct Stage {
  static constexpr int ALL = kTok * PIECES;
  static constexpr int N = (ALL + THREADS - 1) / THREADS;
  u4 x[N];
  // rows t0 .. t0 + 31 from base, `pieces` 16-byte pieces of each at element stride `step`; zeros from row `end` on
  template <typename IO>
  __device__ __forceinline__ void load(const IO* base, long long step, int t0, int end) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + i * THREADS, row = at / PIECES, piece = at % PIECES;
      x[i] = u4{0, 0, 0, 0};
      if ((ALL % THREADS == 0 || at < ALL) && t0 + row < end) {
        x[i] = *reinterpret_cast<const u4*>(base + (t0 + row) * step + piece * Ops<IO>::PER16);
      }
    }
  }
  template <class R>
  __device__ __forceinline__ void store(u4* m) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + i * THREADS;
      if (ALL % THREADS == 0 || at < ALL) m[R::at(at / PIECES, at % PIECES)] = x[i];
    }
  }
};

// The decays of a block.  G is summed in float64 and kept as a float32 pair, in units of log 2: differences stay exact to some 2^-24
// however far G runs, as it does after a token that forgets the state (g is held at -10000, whose exponential is 0 all the same).
struct Gates {
  float hi[kTok], lo[kTok];
  float gamma[kTok];    // exp(G_i)
  float rest[kTok];     // exp(G_end - G_i)
  float beta[kTok];
  float end;            // exp(G_end)
};
__device__ __forceinline__ float exp2_of(double x) {
  const float hi = static_cast<float>(x);
  return exp2f(hi) * fmaf(0.69314718f, static_cast<float>(x - static_cast<double>(hi)), 1.0f);
}
// by the first wave; g and beta of token `lane` (0 past the end of the sequence)
__device__ __forceinline__ void put_gates(Gates& s, int lane, float g, float beta) {
  double G = static_cast<double>(g < -10000.0f ? -10000.0f : g) * 1.4426950408889634;
#pragma unroll
  for (int d = 1; d < kTok; d *= 2) {
    const double other = __shfl_up(G, d, 64);
    if (lane >= d) G += other;
  }
  const double all = __shfl(G, kTok - 1, 64);
  if (lane < kTok) {
    const float hi = static_cast<float>(G);
    s.hi[lane] = hi;
    s.lo[lane] = static_cast<float>(G - static_cast<double>(hi));
    s.gamma[lane] = exp2_of(G);
    s.rest[lane] = exp2_of(all - G);
    s.beta[lane] = beta;
    if (lane == 0) s.end = exp2_of(all);
  }
}

// (I + M)^-1 of one 16 x 16 tile: `m` holds -M transposed ([column][row], stride 20); lanes 0 to 15 hold a row of the inverse each and go
// from its last column to the first: t_j = e_j - sum_{k > j} t_k M_kj.
template <typename IO>
__device__ __forceinline__ void invert_tile(const float* m, typename Ops<IO>::Image& out, int lane) {
  if (lane >= 16) return;
  float t[16];
#pragma unroll
  for (int j = 15; j >= 0; --j) {
    float s = j == lane ? 1.0f : 0.0f;
#pragma unroll
    for (int q = j / 4; q < 4; ++q) {
      const f4 row = *reinterpret_cast<const f4*>(m + 20 * j + 4 * q);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (4 * q + i > j) s = fmaf(t[4 * q + i], row[i], s);
      }
    }
    t[j] = s;
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) Ops<IO>::put(out, lane, g, f4{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]});
}

}  // namespace delta
}  // namespace vla

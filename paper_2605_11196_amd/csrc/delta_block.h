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
// 16-byte pieces.  No value of a wave's columns ever leaves the wave.
//
// Precision.  bf16: K, Q, V and dO are exact operands, the state and the writes three bf16 terms (all 24 bits); matrices between tokens
// six of nine products of three terms each.  What is only rounded to bf16 next (the read-out, the gradient of K) is formed from two terms of a factor, 16
// bits.  float32: the FP32 matrix instruction.
#pragma once

#include "layer_common.h"
#include "vla_mfma_util.h"

namespace vla {
namespace delta {

constexpr int kTok = 32;          // tokens of a block
constexpr int kTiles = kTok / 16;

__host__ __device__ constexpr int pow2_at_least(int n) { return n <= 1 ? 1 : 2 * pow2_at_least((n + 1) / 2); }

// Rows of 16-byte pieces in LDS, a power of two of them, in an order that the row turns, so that the pieces of one place in 16 rows lie in
// different banks.  Places differ by exclusive or with the place, so that one register holds the address of a lane's row and the
// places of a tile are constants applied to it.
template <int PIECES>
struct PieceRows {
  static constexpr int STRIDE = pow2_at_least(PIECES < 2 ? 2 : PIECES);
  static __device__ __forceinline__ int turn(int row) {   // of the row modulo 16
    return STRIDE >= 16 ? row & 15 : (row / (16 / STRIDE)) & (STRIDE - 1);
  }
  static __device__ __forceinline__ int at(int row, int piece) { return row * STRIDE + (piece ^ turn(row)); }
  // `place` (a constant) has no bits in common with `piece`
  static __device__ __forceinline__ int at(int tile, int row, int piece, int place) { return (at(row, piece) ^ place) + 16 * tile * STRIDE; }
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
  // row c of tile t, columns of pair j
  template <class R> static __device__ __forceinline__ A rows(const u4* m, int t, int j, int c, int g) { return m[R::at(t, c, g, 4 * j)]; }
  static __device__ __forceinline__ f4 mul_rows(A a, A b, f4 acc) { return mfma_bf16(a, b, acc); }
  // terms of float32 tiles; the residuals come from the matrix unit, 6 vector and 2 matrix instructions a tile for 22 vector ones
  using One = u2;
  static __device__ __forceinline__ One one(int c, int g) { return minus_identity(c, g); }
  static __device__ __forceinline__ B pair(f4 x0, f4 x1, One one) { return split_tiles(x0, x1, one); }
  static __device__ __forceinline__ f4 mul(A a, const B& b, f4 acc) { return mfma_terms(Terms<1>{{a}}, b, acc); }
  // without the lowest term: for results that are rounded to bf16 next.  The read-out with all three terms (and A in three): 512 heads of 128 1.71 -> 1.93 ms
  // and 20 bytes a lane in scratch memory; 0.02 % of its values are then not the nearest bf16 number, instead of 0.6 %.
  static __device__ __forceinline__ f4 mul_out(A a, const B& b, f4 acc) { return mfma_bf16(a, b.t[0], mfma_bf16(a, b.t[1], acc)); }
  // rows of the state's tile kt (m = key column 32 (kt / 2) + 8 (m / 4) + 4 (kt % 2) + m % 4) against the tokens of tiles t and t + 1
  template <class R> static __device__ __forceinline__ A columns(const u4* m, int kt, int t, int c, int g) {
    const int row = 4 * g + c / 4, piece = c % 4, place = 4 * (kt / 2);
    return cat(read_transposed(m, R::at(t, row, piece, place), kt % 2), read_transposed(m, R::at(t + 1, row, piece, place), kt % 2));
  }
  // accumulator tile of columns 16 n + lane, tokens of tile t; exact
  template <class R> static __device__ __forceinline__ u2 tile_raw(const u4* m, int n, int t, int c, int g) {
    return read_transposed(m, R::at(t, 4 * g + c / 4, (c % 4) / 2, 2 * n), c % 2);
  }
  template <class R> static __device__ __forceinline__ f4 tile(const u4* m, int n, int t, int c, int g) { return widen4(tile_raw<R>(m, n, t, c, g)); }
  static __device__ __forceinline__ void put(Image& im, int row, int g, f4 x) { tok_store(im.hm, im.l, row, row, g, x); }
  static __device__ __forceinline__ TA image(const Image& im, int c, int g) { return tok_load(im.hm, im.l, c, c, g); }
  static __device__ __forceinline__ TB tokens(f4 x, One one) {
    u2 h, m, l;
    split3_cut_matrix(x, one, h, m, l);
    return TokB{cat(h, m), cat(m, h), cat(h, l)};
  }
  static __device__ __forceinline__ f4 mul_tok(const TA& a, const TB& b, f4 acc) { return mfma_tok(a, b, acc); }
  // Matrices that are kept in float32 (R, W) are staged in terms, one set of rows for each (a right operand is laid out alike).
  static constexpr int TERMS = 3;
  using Split = Terms<3>;
  template <int N, class R> static __device__ __forceinline__ Split rows_split(const u4* m, int t, int j, int c, int g) {
    Split s{};
#pragma unroll
    for (int i = 0; i < N; ++i) s.t[i] = m[i * kTok * R::STRIDE + R::at(t, c, g, 4 * j)];
    return s;
  }
  template <int N, class R> static __device__ __forceinline__ Split columns_split(const u4* m, int kt, int t, int c, int g) {
    Split s{};
#pragma unroll
    for (int i = 0; i < N; ++i) s.t[i] = columns<R>(m + i * kTok * R::STRIDE, kt, t, c, g);
    return s;
  }
  // four values of a row, the p-th four
  template <int N, class R> static __device__ __forceinline__ void put_split(u4* m, int row, int p, f4 x) {
    u2 t[3];
    split3_rne(x, t[0], t[1], t[2]);
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<u2*>(m + i * kTok * R::STRIDE + R::at(row, p / 2))[p % 2] = t[i];
  }
  static __device__ __forceinline__ f4 mul_split(const Split& a, const B& b, f4 acc) { return mfma_terms(a, b, acc); }
  static __device__ __forceinline__ f4 mul_split_exact(const Split& a, A b, f4 acc) { return mfma_terms_left(a, Terms<1>{{b}}, acc); }
  // 16 bits of each factor: for gradients that are rounded to bf16
  static __device__ __forceinline__ f4 mul_split_out(const Split& a, const B& b, f4 acc) {
    acc = mfma_bf16(a.t[1], b.t[0], acc);
    acc = mfma_bf16(a.t[0], b.t[1], acc);
    return mfma_bf16(a.t[0], b.t[0], acc);
  }
  struct ImageOut { u4 hm[64]; };
  static __device__ __forceinline__ void put(ImageOut& im, int row, int g, f4 x) {
    u2 h, m, l;
    split3_rne(x, h, m, l);
    im.hm[4 * row + tok_chunk(row, g)] = cat(h, m);
  }
  static __device__ __forceinline__ u4 image(const ImageOut& im, int c, int g) { return im.hm[4 * c + tok_chunk(c, g)]; }
  // an exact right operand
  using Raw = u2;
  static __device__ __forceinline__ f4 mul_tok_raw(u4 a, Raw b, f4 acc) { return mfma_bf16(a, cat(b, b), acc); }
  static __device__ __forceinline__ f4 value(Raw x) { return widen4(x); }
  static __device__ __forceinline__ f4 mul_tok_raw(const TA& a, Raw b, f4 acc) {
    return mfma_bf16(a.hm, cat(b, b), mfma_bf16(a.lh, cat(b, u2{0, 0}), acc));
  }
  static __device__ __forceinline__ f4 mul_tok_out(u4 a, const TB& b, f4 acc) { return mfma_bf16(a, b.hm, mfma_bf16(a, b.mh, acc)); }
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
  template <class R> static __device__ __forceinline__ A rows(const u4* m, int t, int j, int c, int g) {
    return A{__builtin_bit_cast(f4, m[R::at(t, c, 2 * g, 8 * j)]), __builtin_bit_cast(f4, m[R::at(t, c, 2 * g, 8 * j + 1)])};
  }
  static __device__ __forceinline__ f4 mul_rows(const A& a, const A& b, f4 acc) { return mul4(a.x1, b.x1, mul4(a.x0, b.x0, acc)); }
  struct One {};
  static __device__ __forceinline__ One one(int, int) { return One{}; }
  static __device__ __forceinline__ B pair(f4 x0, f4 x1, One) { return B{x0, x1}; }
  static __device__ __forceinline__ f4 mul(const A& a, const B& b, f4 acc) { return mul4(a.x1, b.x1, mul4(a.x0, b.x0, acc)); }
  static __device__ __forceinline__ f4 mul_out(const A& a, const B& b, f4 acc) { return mul(a, b, acc); }
  static __device__ __forceinline__ float value(const u4* m, int piece_at, int i) { return reinterpret_cast<const float*>(m + piece_at)[i]; }
  template <class R> static __device__ __forceinline__ A columns(const u4* m, int kt, int t, int c, int g) {
    A a;
    const int piece = 2 * (c / 4), place = 8 * (kt / 2) + kt % 2;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      a.x0[r] = value(m, R::at(t, 4 * g + r, piece, place), c % 4);
      a.x1[r] = value(m, R::at(t + 1, 4 * g + r, piece, place), c % 4);
    }
    return a;
  }
  template <class R> static __device__ __forceinline__ f4 tile(const u4* m, int n, int t, int c, int g) {
    f4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = value(m, R::at(t, 4 * g + r, c / 4, 4 * n), c % 4);
    return x;
  }
  template <class R> static __device__ __forceinline__ f4 tile_raw(const u4* m, int n, int t, int c, int g) { return tile<R>(m, n, t, c, g); }
  static __device__ __forceinline__ void put(Image& im, int row, int g, f4 x) { im.x[4 * row + tok_chunk(row, g)] = x; }
  static __device__ __forceinline__ TA image(const Image& im, int c, int g) { return im.x[4 * c + tok_chunk(c, g)]; }
  static __device__ __forceinline__ TB tokens(f4 x, One) { return x; }
  static __device__ __forceinline__ f4 mul_tok(const TA& a, const TB& b, f4 acc) { return mul4(a, b, acc); }
  static __device__ __forceinline__ f4 mul_tok_out(const TA& a, const TB& b, f4 acc) { return mul4(a, b, acc); }
  static constexpr int TERMS = 1;
  using Split = A;
  template <int N, class R> static __device__ __forceinline__ Split rows_split(const u4* m, int t, int j, int c, int g) { return rows<R>(m, t, j, c, g); }
  template <int N, class R> static __device__ __forceinline__ Split columns_split(const u4* m, int kt, int t, int c, int g) { return columns<R>(m, kt, t, c, g); }
  template <int N, class R> static __device__ __forceinline__ void put_split(u4* m, int row, int p, f4 x) { m[R::at(row, p)] = __builtin_bit_cast(u4, x); }
  static __device__ __forceinline__ f4 mul_split(const A& a, const B& b, f4 acc) { return mul(a, b, acc); }
  static __device__ __forceinline__ f4 mul_split_exact(const A& a, const A& b, f4 acc) { return mul_rows(a, b, acc); }
  static __device__ __forceinline__ f4 mul_split_out(const A& a, const B& b, f4 acc) { return mul(a, b, acc); }
  static __device__ __forceinline__ f4 mul(const A& a, const A& b, f4 acc) { return mul_rows(a, b, acc); }
  static __device__ __forceinline__ f4 mul_split_out(const A& a, const A& b, f4 acc) { return mul_rows(a, b, acc); }
  using ImageOut = Image;
  using Raw = f4;
  static __device__ __forceinline__ f4 value(Raw x) { return x; }
  static __device__ __forceinline__ f4 mul_tok_raw(const TA& a, Raw b, f4 acc) { return mul4(a, b, acc); }
};

// Rows of memory as a buffer whose bounds the hardware checks: loads past the last row give zeros, stores past it are dropped, so that
// the last block needs no branches.  Rows are at most 2^31 / 32 bytes apart (checked on the host) and do not overlap.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void* base, long long step_bytes, int rows, int row_bytes) {
  const int bytes = rows <= 0 ? 0 : static_cast<int>((min(rows, kTok) - 1) * step_bytes) + row_bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}

// A block's rows on their way from memory to LDS: N pieces a thread.
template <int PIECES, int THREADS>
struct Stage {
  static constexpr int ALL = kTok * PIECES;
  static constexpr int N = (ALL + THREADS - 1) / THREADS;
  u4 x[N];
  int at[N];   // byte offset of each piece from the block's first row
  __device__ __forceinline__ void init(long long step_bytes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + i * THREADS;
      at[i] = p < ALL ? p / PIECES * static_cast<int>(step_bytes) + p % PIECES * 16 : 0x7fffffff;
    }
  }
  // the last token in the first row
  __device__ __forceinline__ void init_reversed(long long step_bytes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + i * THREADS;
      at[i] = p < ALL ? (kTok - 1 - p / PIECES) * static_cast<int>(step_bytes) + p % PIECES * 16 : 0x7fffffff;
    }
  }
  // rows t0 .. t0 + 31 of base; zeros from row `end` on
  __device__ __forceinline__ void load(const char* base, long long step_bytes, int t0, int end) {
    const __amdgpu_buffer_rsrc_t r = rows_buffer(base + t0 * step_bytes, step_bytes, end - t0, PIECES * 16);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, at[i], 0, 0);
  }
  template <class R>
  __device__ __forceinline__ void store(u4* m) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + i * THREADS;
      if (ALL % THREADS == 0 || p < ALL) m[R::at(p / PIECES, p % PIECES)] = x[i];
    }
  }
};

// four tokens' values of one column, at the byte offset of the first; rows past the end are dropped
__device__ __forceinline__ void store_column(__amdgpu_buffer_rsrc_t r, int at, int step_bytes, f4 x, float*) {
#pragma unroll
  for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[i]), r, at + i * step_bytes, 0, 0);
}
__device__ __forceinline__ void store_column(__amdgpu_buffer_rsrc_t r, int at, int step_bytes, f4 x, uint16_t*) {
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint32_t two = pack_rne(x[i], x[i + 1]);
    __builtin_amdgcn_raw_buffer_store_b16(static_cast<uint16_t>(two), r, at + i * step_bytes, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b16(static_cast<uint16_t>(two >> 16), r, at + (i + 1) * step_bytes, 0, 0);
  }
}

// The decays of a block.  G is summed in float64 and kept as a float32 pair, in units of log 2: differences stay exact to some 2^-24
// however far G runs, as it does after a token that forgets the state (g is held at -10000, whose exponential is 0 all the same).
struct __align__(16) Gates {
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
// x of lane l - N of the same 16 lanes, 0 where there is none
template <int N>
__device__ __forceinline__ double shifted_up(double x) {
  const uint2 b = __builtin_bit_cast(uint2, x);
  const uint2 s = {static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b.x), 0x110 + N, 0xf, 0xf, true)),
                   static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b.y), 0x110 + N, 0xf, 0xf, true))};
  return __builtin_bit_cast(double, s);
}
__device__ __forceinline__ double of_lane(double x, int lane) {
  const uint2 b = __builtin_bit_cast(uint2, x);
  return __builtin_bit_cast(double, uint2{static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b.x), lane)),
                                          static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b.y), lane))});
}
// by one wave; g and beta of token `lane` (0 past the end of the sequence), whose place in the arrays is `at`
__device__ __forceinline__ void put_gates(Gates& s, int lane, int at, float g, float beta) {
  static_assert(kTok == 32, "two rows of lanes");
  double G = static_cast<double>(g < -10000.0f ? -10000.0f : g) * 1.4426950408889634;
  G += shifted_up<1>(G);
  G += shifted_up<2>(G);
  G += shifted_up<4>(G);
  G += shifted_up<8>(G);
  const double first = of_lane(G, 15);
  if (lane >= 16) G += first;
  const double all = of_lane(G, kTok - 1);
  if (lane < kTok) {
    const float hi = static_cast<float>(G);
    s.hi[at] = hi;
    s.lo[at] = static_cast<float>(G - static_cast<double>(hi));
    s.gamma[at] = exp2_of(G);
    s.rest[at] = exp2_of(all - G);
    s.beta[at] = beta;
    if (lane == 0) s.end = exp2_of(all);
  }
}

// (I + M)^-1 of one 16 x 16 tile.  x: -M, four columns 4 g + r of row c a lane; m: scratch of 16 rows at stride 20.  Each 16 lanes hold the
// rows of the inverse, one a lane, and go from its last column to the first, t_j = e_j - sum_{k > j} t_k M_kj: what multiplies t_k is a
// register of lane k, broadcast inside the multiplication (DPP), 120 of them, without LDS in the chain.
template <int K, int J>
struct SubstituteColumn {
  static __device__ __forceinline__ void run(float (&t)[16], const float (&m)[16]) {
    if constexpr (J >= 0) {
      fmac_row_bcast<K>(t[J], m[J], t[K]);
      SubstituteColumn<K, J - 1>::run(t, m);
    }
  }
};
template <int K>
__device__ __forceinline__ void substitute(float (&t)[16], const float (&m)[16]) {
  if constexpr (K > 0) {
    SubstituteColumn<K, K - 1>::run(t, m);
    substitute<K - 1>(t, m);
  }
}
template <typename IO>
__device__ __forceinline__ void invert_tile(f4 x, float* m, typename Ops<IO>::Image& out, int c, int g) {
  *reinterpret_cast<f4*>(m + 20 * c + 4 * g) = x;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float row[16], t[16];
#pragma unroll
  for (int j = 0; j < 16; j += 4) {
    const f4 y = *reinterpret_cast<const f4*>(m + 20 * c + j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      row[j + i] = y[i];
      t[j + i] = j + i == c ? 1.0f : 0.0f;
    }
  }
  substitute<15>(t, row);
  f4 mine;
#pragma unroll
  for (int r = 0; r < 4; ++r) mine[r] = g < 2 ? (g == 0 ? t[r] : t[4 + r]) : (g == 2 ? t[8 + r] : t[12 + r]);
  Ops<IO>::put(out, c, g, mine);
}

// Jobs in turn, the long ones first: from the second round on the waves take them in reverse, so that the first ones have the fewest.
__device__ __forceinline__ int job_of(int round, int wave, int waves) { return round * waves + (round == 0 ? wave : waves - 1 - wave); }

// The matrices between the tokens of a block, tile by tile on different waves, as left operands of the products that follow:
//   inverse  (I + M)^-1 of the diagonal tiles,  below  -M of the tiles below,  att  A (with ATT)
// Products are transposed, so that a lane has four tokens j of row i.  REVERSE: rows are the block's tokens with the last one first, M =
// exp(G_j - G_i) (k_i . k_j) beta_j of them, A = scale exp(G_j - G_i) (q_j . k_i).
template <typename IO, class RK, int PAIRS, int WAVES, bool REVERSE, bool ATT, typename AttImage>
__device__ __forceinline__ void token_matrices(const u4* sK, const u4* sQ, const Gates& gates, typename Ops<IO>::Image* inverse,
                                               typename Ops<IO>::Image* below, AttImage* att, float (*scratch)[16 * 20], float scale, int wave, int c, int g) {
  using O = Ops<IO>;
  constexpr int TILES = kTiles * (kTiles + 1) / 2;
  constexpr int JOBS = (ATT ? 2 : 1) * TILES;
  for (int round = 0; round * WAVES < JOBS; ++round) {
    // the diagonal tiles of k k^T first: their inverses take longest
    const int job = job_of(round, wave, WAVES);
    if (job >= JOBS) continue;
    const bool keys = job < TILES;
    int p = keys ? job : job - TILES, i, j;
    if (p < kTiles) {
      i = j = p;
    } else {
      p -= kTiles;
      i = 1;
      while (p >= i) p -= i++;
      j = p;
    }
    const u4* from_j = REVERSE && !keys ? sQ : sK;
    const u4* from_i = !REVERSE && !keys ? sQ : sK;
    typename O::A rj[PAIRS], ri[PAIRS];
#pragma unroll
    for (int s = 0; s < PAIRS; ++s) {
      rj[s] = O::template rows<RK>(from_j, j, s, c, g);
      ri[s] = O::template rows<RK>(from_i, i, s, c, g);
    }
    const float hi = gates.hi[16 * i + c], lo = gates.lo[16 * i + c];
    const f4 hj = *reinterpret_cast<const f4*>(&gates.hi[16 * j + 4 * g]), lj = *reinterpret_cast<const f4*>(&gates.lo[16 * j + 4 * g]);
    const f4 bj = *reinterpret_cast<const f4*>(&gates.beta[16 * j + 4 * g]);
    f4 x = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < PAIRS; ++s) x = O::mul_rows(rj[s], ri[s], x);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int before = i - j > 0 ? 1 : (keys ? c - (4 * g + r) : c - (4 * g + r) + 1);   // > 0: token j counts for token i
      const float apart = REVERSE ? (hj[r] - hi) + (lj[r] - lo) : (hi - hj[r]) + (lo - lj[r]);
      const float w = __builtin_amdgcn_exp2f(apart) * (keys ? -bj[r] : (REVERSE ? scale : scale * bj[r]));
      x[r] = before > 0 ? x[r] * w : 0.0f;
    }
    if (keys && i == j) {
      invert_tile<IO>(x, scratch[i], inverse[i], c, g);
    } else if (keys) {
      O::put(below[i * (i - 1) / 2 + j], c, g, x);
    } else if constexpr (ATT) {
      O::put(att[i * (i + 1) / 2 + j], c, g, x);
    }
  }
}

}  // namespace delta
}  // namespace vla

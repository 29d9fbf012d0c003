// Internal declarations of the operators on rows of channels [B, T, n]: the short causal convolution, the selective state space
// scan, and the norms around a block (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vla {

// Element strides of a [B, T, n] tensor whose last dimension is contiguous.
struct Row2 {
  long long b, t;
};

// Sums over the rows of parts[rows][stride] in a fixed order: out[i * step] = sum of parts[.][i], i < columns.
struct ColumnSum {
  const float* parts;
  size_t stride;
  int rows, columns;
  void* out;
  int bf16, step;
};
constexpr int kColumnSums = 5;
struct ColumnSums {
  ColumnSum job[kColumnSums];
  int n;
};
hipError_t launch_column_sums(const ColumnSums& s, hipStream_t stream);

constexpr int kConvWidth = 4;        // taps at most
constexpr int kConvThreads = 256;    // of a workgroup, 16 bytes of channels each
struct ConvArgs {
  const void* x;
  const void* weight;    // [n][width]
  const void* bias;      // [n] or nullptr
  const void* state;     // [B][width - 1][n] or nullptr (zero)
  void* y;
  void* state_T;         // or nullptr; may be state
  const int* lengths;    // [B] or nullptr: T
  const void* dy;        // backward: strides ys
  const void* dstate_T;  // or nullptr (zero)
  void* dx;              // strides dxs
  void* dstate;          // or nullptr
  float* sum_part;       // [parts][width + 1][n]: what runs of tokens give of the gradients of weight and bias, or nullptr
  int joined;            // a part for each workgroup (otherwise for each run)
  Row2 xs, ys, dxs;
  int B, T, n, w_bf16, silu;
  int run, runs;         // tokens of a run, runs of a sequence
};
hipError_t launch_causal_conv(const ConvArgs& a, int width, int io_dtype, hipStream_t stream);
hipError_t launch_causal_conv_step(const ConvArgs& a, int width, int io_dtype, hipStream_t stream);
hipError_t launch_causal_conv_backward(const ConvArgs& a, int width, int io_dtype, hipStream_t stream);

constexpr int kScanBlock = 8;    // tokens between two states that are kept
int selective_tile(int N);       // channels of a workgroup
struct ScanArgs {
  const void* u;
  const void* delta;
  const float* A;         // [n][N]
  const void* Bm;
  const void* Cm;
  const float* D;         // [n] or nullptr (zero)
  const void* z;          // or nullptr (no gate)
  const float* bias;      // [n] or nullptr (zero)
  const float* h0;        // [B][n][N] or nullptr (zero)
  void* y;
  float* h_T;             // or nullptr
  const int* lengths;     // [B] or nullptr: T
  Row2 us, ds, zs, ys;    // (backward: dy has ys)
  long long B_b, B_g, B_t, C_b, C_g, C_t;   // element strides of B and C [B, T, G, N]
  int nb, T, n, G, softplus;
  int tiles;              // workgroups of a group's channels
  // what is kept for the backward pass: the state before every 8th token, or nullptr
  float* kept;            // [B][blocks][n][N]
  int blocks;
  // time segments
  int n_seg, seg_tokens;
  float* seg_h;           // [B][n_seg][n][N]: the maps' own ends, then the states that the segments start from
  float* seg_dt;          // [B][n_seg][n]: sums of the steps
  // backward
  const void* dy;
  const float* dh_T;      // or nullptr (zero)
  void* du;
  void* ddelta;
  void* dz;
  Row2 dus, dds, dzs;
  float* dh0;             // or nullptr
  void* dB;               // [B][T][G][N]
  void* dC;
  float* dA_part;         // [B][n_seg][n][N]
  float* dD_part;         // [B][n_seg][n]
  float* dbias_part;
  float* dBC_part;        // [G * tiles][B][T][2][N]
};
hipError_t launch_selective_scan(const ScanArgs& a, int N, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_selective_combine(const ScanArgs& a, int N, bool backward, hipStream_t stream);
hipError_t launch_selective_step(const ScanArgs& a, int N, int io_dtype, hipStream_t stream);   // T = 1, h_T holds the state
hipError_t launch_selective_backward(const ScanArgs& a, int N, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_selective_shared(const ScanArgs& a, int N, int io_dtype, hipStream_t stream);
inline bool scan_state_size(int N) { return N == 8 || N == 16 || N == 32 || N == 64; }

constexpr int kResidualColumns = 8192;  // columns of a row at most
struct ResidualArgs {
  const void* x;            // the residual stream, or nullptr
  const void* y;            // the block's output
  const void* gate;         // or nullptr
  const void* post_weight;  // [n] each, or nullptr
  const void* scale;
  const void* weight;
  void* s;
  void* h;
  const void* ds;           // backward: strides ss, hs
  const void* dh;
  void* dx;
  void* dy;
  void* dgate;
  float* sum_part;          // [workgroups][3][n]: weight, post_weight, scale
  Row2 xs, ys, gs, ss, hs, dxs, dys, dgs;
  int B, T, n, group;       // columns of a group of the norm of y
  int w_bf16, act;          // act 0: silu, 1: sigmoid
  float eps;
};
int residual_partials(int n);   // workgroups of the backward pass at most: rows of sum_part
hipError_t launch_residual_norm(const ResidualArgs& a, int io_dtype, int stream_dtype, hipStream_t stream);
hipError_t launch_residual_norm_backward(const ResidualArgs& a, int io_dtype, int stream_dtype, int* parts, hipStream_t stream);

}  // namespace vla

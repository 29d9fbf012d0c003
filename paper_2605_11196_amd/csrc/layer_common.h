// Internal declarations of the operators around the recurrence: the gated delta rule and the norm of queries and keys with
// the position rotation (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vla {

// Element strides of a [B, H, T, d] tensor whose last dimension is contiguous.
struct Rows {
  long long b, h, t;
};

struct NormArgs {
  const void* x[2];        // queries, keys: [B, H, T, d] by strides
  const void* w[2];        // [d] or nullptr (ones)
  const float* cos;        // [places][rot / 2]
  const float* sin;
  const int* positions;    // [B][T] or nullptr: offset + t
  void* y[2];              // forward
  const void* dy[2];       // backward
  void* dx[2];
  float* dw_part;          // [workgroups][2][d]
  void* dw[2];             // [d], of the weights' type, or nullptr
  Rows xs[2], ys[2], dxs[2];
  int H[2];
  int B, T, rot, places, offset;
  float eps, inv_n;        // 1 / d (RMS) or 1 (L2)
  int w_bf16;
};
constexpr int kNormPartials = 1024;   // workgroups of the backward pass at most: rows of dw_part
hipError_t launch_qk_norm_rope(const NormArgs& a, int d, int io_dtype, bool interleaved, hipStream_t stream);
hipError_t launch_qk_norm_rope_backward(const NormArgs& a, int d, int io_dtype, bool interleaved, hipStream_t stream);

constexpr int kKeep = 256;   // tokens between two states that are kept for the backward pass

struct DeltaArgs {
  const void* q;
  const void* k;
  const void* v;
  const float* g;
  const float* beta;
  const float* S0;
  void* o;
  float* S_T;
  const int* lengths;      // [B] or nullptr: T
  Rows qs, ks, vs, os, gs, bs;
  int B, H_k, H_v, T;
  float scale;
  // for the backward pass, or nullptr
  float* kept;             // [B * H_v][n_kept][d_v][d_k]: the state at the start of every 256 tokens (backward: its gradient at their end)
  float* rows;             // [B * H_v][T][d_v]: R, beta R is what a token writes (backward: W, beta W is the gradient of v)
  int n_kept;
  // backward
  const void* dO;          // strides os
  void* dv;                // outputs by strides
  void* dq;
  void* dk;
  Rows dvs, dqs, dks;
  const float* kept_state; // of the forward pass: kept, rows
  const float* R;
  float* dk_part;          // [B * H_v][T][d_k]: what the sweep along the tokens gives of dk
                           // (with dq_part: the whole of it)
  float* dq_part;          // [B * H_v][T][d_k]: dq of a value head where heads share a key head, or nullptr
  float* dg;               // [B * H_v][T]
  float* dbeta;
  // time segments
  int n_seg, seg_tokens;
  bool first_done;         // the first segment on the way goes with the maps
  bool seg_states;         // S0 holds a state for each segment: [B * H_v][n_slots][d_v][d_k]
  int n_slots;             // places of the arrays for each head: one for each segment but a first one that goes with the maps
  float* seg_map;          // [B * H_v][n_slots][d_v + d_k][d_k]: the segments' affine maps, Y then X
  float* seg_S;            // with the maps: [B * H_v][n_slots][d_v][d_k], the states that the segments start from
};
// Token by token, the rows of the state on registers (delta_step.hip): single tokens and short sequences.
hipError_t launch_delta_step(const DeltaArgs& a, int d_k, int d_v, int io_dtype, hipStream_t stream);

// Whether the first of several time segments can go with the maps of the others.  With fewer waves for its outputs it would take longer than they
// (32 heads of 128 x 16, 4096 tokens, 16 segments 154 -> 196 us).
constexpr bool delta_first_with_maps(int d_v) { return d_v >= 64; }

// In blocks of 32 tokens (delta_chunk.h); map: the affine maps of the segments instead of outputs.
hipError_t launch_delta_chunk_16(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_chunk_32(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_chunk_64(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_chunk_96(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_chunk_128(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);

// The states from segment to segment, S <- S X + Y, from S0 on, or with first_done from that of the second segment on, which is there
// (delta_combine.hip; backward: from the last segment on).
hipError_t launch_delta_combine(const DeltaArgs& a, int d_k, int d_v, bool backward, hipStream_t stream);

// The chain of the state's gradient from the last block to the first (delta_reverse.h): S0 is the gradient of S_T and S_T that of S0.
hipError_t launch_delta_reverse_16(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_reverse_32(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_reverse_64(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_reverse_96(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);
hipError_t launch_delta_reverse_128(const DeltaArgs& a, int d_v, int io_dtype, bool map, hipStream_t stream);

// The gradients of q, k, g and beta, every 256 tokens at once (delta_grad.h), and the sum over the heads that share a key head.
hipError_t launch_delta_grad_16(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream);
hipError_t launch_delta_grad_32(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream);
hipError_t launch_delta_grad_64(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream);
hipError_t launch_delta_grad_96(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream);
hipError_t launch_delta_grad_128(const DeltaArgs& a, int d_v, int io_dtype, hipStream_t stream);
hipError_t launch_delta_shared(const DeltaArgs& a, int d_k, int io_dtype, hipStream_t stream);

inline bool layer_head_size(int d) { return d == 16 || d == 32 || d == 64 || d == 96 || d == 128; }

}  // namespace vla

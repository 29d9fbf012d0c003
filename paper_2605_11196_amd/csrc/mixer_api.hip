// Host side of the operators on rows of channels (include/vla.h): validation and dispatch of the short causal convolution, the selective
// state space scan and the norms around a block.
#include "../../include/vla.h"

#include "host_checks.h"
#include "mixer_common.h"

#include <math.h>

namespace {

size_t padded(size_t n) { return (n + 255) / 256 * 256; }
size_t size_of(int dtype) { return dtype == VLA_BF16 ? 2 : 4; }
bool is_type(int dtype) { return dtype == VLA_F32 || dtype == VLA_BF16; }

// Sizes that the operators on [B, T, n] share: whole eights of channels, 32-bit tokens with a block of look-ahead.
int check_rows(int B, int T, int n, int io_dtype) {
  if (B <= 0 || T < 0 || n <= 0 || !is_type(io_dtype)) return VLA_ERR_INVALID_ARG;
  if (n % 8 != 0 || T > 0x7fffff00) return VLA_ERR_UNSUPPORTED;
  return VLA_OK;
}
// Strides of a [B, T, n] tensor, read or (apart) written.
bool rows2(const vla_strides& s, int B, int T, int n, int dtype, bool written, vla::Row2* out) {
  vla::Rows r;
  if (s.h != 0 || !rows_of(s, 1, T, n, static_cast<int>(16 / size_of(dtype)), &r)) return false;
  if (written && !rows_apart(r, B, 1, T, n)) return false;
  *out = vla::Row2{r.b, r.t};
  return true;
}
// the scan's kernels address the rows of a block with 31-bit byte offsets
bool rows_near(const vla::Row2& r, int n, int dtype) {
  return r.t < 0x7fffffffLL / (2 * vla::kScanBlock * static_cast<long long>(size_of(dtype))) && n <= 0x7fffffffLL / (2 * static_cast<long long>(size_of(dtype)));
}
size_t reach2(const vla::Row2& r, int B, int T, int n, int dtype) { return reach(vla::Rows{r.b, 0, r.t}, B, 1, T, n, size_of(dtype)); }
bool all_aligned(const void* const* p, int n) {
  for (int i = 0; i < n; ++i) {
    if (!aligned16(p[i])) return false;
  }
  return true;
}
bool any_null(const void* const* p, int n) {
  for (int i = 0; i < n; ++i) {
    if (p[i] == nullptr) return true;
  }
  return false;
}

// ---- short causal convolution

// Tokens of a thread's run: 16, so that short and narrow calls fill the card (the backward pass of 3 x 1537 rows of 1664 in float32: runs of
// 64 take 38 us, of 32 25, of 16 18), and longer ones as long as there are enough threads, so that the rows before a run, read again, and
// its part of the weights' gradient weigh little.
int conv_run(int B, int T, int n, int io_dtype) {
  const long long threads = static_cast<long long>(B) * (n / (16 / size_of(io_dtype)));
  long long run = 16;
  while (run < 256 && threads * (T / (2 * run)) >= 256 * 1024) run *= 2;
  return static_cast<int>(run < T ? run : T > 0 ? T : 1);
}
int runs_of(int T, int run) { return T > 0 ? (T + run - 1) / run : 1; }
// Parts of the weights' gradient: a run each, or, with channels that a workgroup holds at least twice, a workgroup each.
bool conv_joined(int n, int io_dtype) { return n / (16 / static_cast<int>(size_of(io_dtype))) <= vla::kConvThreads / 2; }
long long conv_parts(int B, int runs, int n, int io_dtype) {
  const long long all = static_cast<long long>(B) * runs, pieces = n / (16 / static_cast<int>(size_of(io_dtype)));
  return conv_joined(n, io_dtype) ? (all * pieces + vla::kConvThreads - 1) / vla::kConvThreads : all;
}
size_t conv_parts_bytes(int B, int T, int n, int width, int io_dtype) {
  return static_cast<size_t>(conv_parts(B, runs_of(T, conv_run(B, T, n, io_dtype)), n, io_dtype)) * (width + 1) * n * 4;
}

int conv_args(const void* x, const void* weight, const void* bias, const void* state, int B, int T, int n, int width, int io_dtype,
              const vla_conv_opts* opts, vla_conv_opts* op, vla::ConvArgs* a) {
  vla_conv_default_opts(op);
  if (opts != nullptr) *op = *opts;
  const int st = check_rows(B, T, n, io_dtype);
  if (st != VLA_OK) return st;
  if (!is_type(op->weight_dtype) || width <= 0) return VLA_ERR_INVALID_ARG;
  if (width < 2 || width > vla::kConvWidth) return VLA_ERR_UNSUPPORTED;
  if (weight == nullptr || (T > 0 && x == nullptr)) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {x, weight, bias, state};
  if (!all_aligned(ptrs, 4)) return VLA_ERR_INVALID_ARG;
  *a = vla::ConvArgs{};
  if (!rows2(op->x, B, T, n, io_dtype, false, &a->xs)) return VLA_ERR_INVALID_ARG;
  a->x = x; a->weight = weight; a->bias = bias; a->state = state;
  a->lengths = op->lengths;
  a->B = B; a->T = T; a->n = n;
  a->w_bf16 = op->weight_dtype == VLA_BF16;
  a->silu = op->silu != 0;
  return VLA_OK;
}
bool conv_fits(const vla::ConvArgs& a, int io_dtype) {
  return static_cast<long long>(a.B) * a.runs <= 0x7fffffff && fits_launch(static_cast<long long>(a.B) * a.runs, a.n / (16 / static_cast<int>(size_of(io_dtype)))) &&
         static_cast<long long>(a.B) * a.runs * (a.n / (16 / static_cast<int>(size_of(io_dtype)))) < kMostItems - 256;
}

// ---- selective state space scan

vla_scan_opts scan_opts(const vla_scan_opts* o) {
  vla_scan_opts r;
  vla_scan_default_opts(&r);
  if (o != nullptr) r = *o;
  return r;
}
int tiles_of(int n, int groups, int tile) { return (n / groups + tile - 1) / tile; }
int blocks_of(int T) { return (T + vla::kScanBlock - 1) / vla::kScanBlock; }

int check_scan(int B, int T, int n, int N, int io_dtype, const vla_scan_opts& o) {
  const int st = check_rows(B, T, n, io_dtype);
  if (st == VLA_ERR_INVALID_ARG) return st;
  if (N <= 0 || o.groups <= 0 || n % o.groups != 0 || o.segments < 0) return VLA_ERR_INVALID_ARG;
  if (st != VLA_OK) return st;
  if (!vla::scan_state_size(N) || n / o.groups % 8 != 0 || static_cast<long long>(n) * N > 0x7fffff00) return VLA_ERR_UNSUPPORTED;
  if (!fits_launch(static_cast<long long>(B) * o.groups * tiles_of(n, o.groups, vla::selective_tile(N)), 512)) return VLA_ERR_UNSUPPORTED;
  if (!fits_launch(static_cast<long long>(B) * n, N) || static_cast<long long>(B) * n * N > kMostItems - 256) return VLA_ERR_UNSUPPORTED;
  return VLA_OK;
}

// Time segments.  In segments the tokens are gone through twice (the second time without the read-out), which pays while sequences and channels
// leave SIMDs idle: with fewer than 1400 waves on the card's 1024.  8 x 2048 tokens, 16 states, bfloat16, forward that saves and backward
// together, whole and in segments: 1024 channels (512 waves) 858 us and 428, 2048 (1024) 904 and 815, 2560 (1280) 1177 and 1039, 3584 (1792) 1195 and (two) 1505.
// As many segments as give 8192 waves, of four blocks at least; the maps hold 6 to 8 of them a SIMD, the outputs 4 to 6, the gradients 2, and the others
// come when these have ended (2048 channels of one sequence of 16384: 16 segments 864 us, 64 831; of 32768: 48 1601, 64 1582, 96 1587).
// From 1400 waves on what does not fit at once is a round of its own, two waves a SIMD of the gradients: 4096 channels (2048 waves) take 1205 us, 4160 1750,
// 5120 1844, 8192 2372.
struct ScanPlan {
  int n, tokens;             // segments, tokens of each: whole blocks
  size_t h_bytes, dt_bytes;  // of the states and the sums of steps
};
ScanPlan scan_plan(int B, int T, int n, int N, int groups, int requested) {
  ScanPlan p{1, T, 0, 0};
  const int blocks = blocks_of(T), threads = 256;
  const long long workgroups = static_cast<long long>(B) * groups * tiles_of(n, groups, vla::selective_tile(N)), waves = workgroups * (threads / 64);
  long long s = requested;
  if (requested == 0) {
    s = 1;
    if (waves < 1400) s = (8192 + waves - 1) / waves;
    if (s > blocks / 4) s = blocks / 4;
  }
  if (s > blocks) s = blocks;
  if (s > 1024) s = 1024;
  if (s > 1 && !fits_launch(workgroups * s, threads)) s = 1;
  if (s <= 1) return p;
  p.tokens = vla::kScanBlock * static_cast<int>((blocks + s - 1) / s);
  p.n = (T + p.tokens - 1) / p.tokens;
  p.h_bytes = padded(static_cast<size_t>(B) * p.n * n * N * 4);
  p.dt_bytes = padded(static_cast<size_t>(B) * p.n * n * 4);
  return p;
}

size_t scan_saved(int B, int T, int n, int N) { return static_cast<size_t>(B) * blocks_of(T) * n * N * 4; }
struct ScanBackwardParts {
  ScanPlan seg;
  size_t dA, dD, dbias, dBC, seg_h, seg_dt, bytes;   // offsets
};
ScanBackwardParts scan_backward_parts(int B, int T, int n, int N, int groups, int requested) {
  ScanBackwardParts p{};
  p.seg = scan_plan(B, T, n, N, groups, requested);
  const size_t rows = static_cast<size_t>(B) * p.seg.n;
  p.dD = p.dA + padded(rows * n * N * 4);
  p.dbias = p.dD + padded(rows * n * 4);
  p.dBC = p.dbias + padded(rows * n * 4);
  p.seg_h = p.dBC + padded(static_cast<size_t>(groups) * tiles_of(n, groups, vla::selective_tile(N)) * B * T * 2 * N * 4);
  p.seg_dt = p.seg_h + p.seg.h_bytes;
  p.bytes = p.seg_dt + p.seg.dt_bytes;
  return p;
}

// B's and C's strides: [B, T, groups, N] contiguous where none are given.
bool state_rows(const vla_strides& s, int B, int T, int groups, int N, int dtype, vla::Rows* out) {
  if (s.b == 0 && s.h == 0 && s.t == 0) {
    *out = vla::Rows{static_cast<long long>(T) * groups * N, N, static_cast<long long>(groups) * N};
    return true;
  }
  return rows_of(s, groups, T, N, static_cast<int>(16 / size_of(dtype)), out);
}
int scan_args(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z, const float* bias,
              int B, int T, int n, int N, int io_dtype, const vla_scan_opts& op, vla::ScanArgs* a) {
  const int st = check_scan(B, T, n, N, io_dtype, op);
  if (st != VLA_OK) return st;
  const void* needed[] = {u, delta, Bm, Cm};
  if (A == nullptr || (T > 0 && any_null(needed, 4))) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {u, delta, A, Bm, Cm, D, z, bias};
  if (!all_aligned(ptrs, 8)) return VLA_ERR_INVALID_ARG;
  *a = vla::ScanArgs{};
  vla::Rows rb, rc;
  if (!rows2(op.u, B, T, n, io_dtype, false, &a->us) || !rows2(op.delta, B, T, n, io_dtype, false, &a->ds) ||
      !rows2(op.z, B, T, n, io_dtype, false, &a->zs) || !state_rows(op.B, B, T, op.groups, N, io_dtype, &rb) ||
      !state_rows(op.C, B, T, op.groups, N, io_dtype, &rc)) {
    return VLA_ERR_INVALID_ARG;
  }
  for (const vla::Row2* r : {&a->us, &a->ds, &a->zs}) {
    if (!rows_near(*r, n, io_dtype)) return VLA_ERR_UNSUPPORTED;
  }
  a->B_b = rb.b; a->B_g = rb.h; a->B_t = rb.t;
  a->C_b = rc.b; a->C_g = rc.h; a->C_t = rc.t;
  a->u = u; a->delta = delta; a->A = A; a->Bm = Bm; a->Cm = Cm; a->D = D; a->z = z; a->bias = bias;
  a->lengths = op.lengths;
  a->nb = B; a->T = T; a->n = n; a->G = op.groups;
  a->softplus = op.softplus != 0;
  a->tiles = tiles_of(n, op.groups, vla::selective_tile(N));
  a->blocks = blocks_of(T);
  a->n_seg = 1;
  a->seg_tokens = vla::kScanBlock * blocks_of(T);
  return VLA_OK;
}
// what all calls of the scan read
constexpr int kScanReads = 9;
void scan_reads(const vla::ScanArgs& a, int N, int io_dtype, Range* r) {
  const size_t es = size_of(io_dtype);
  r[0] = {a.u, reach2(a.us, a.nb, a.T, a.n, io_dtype), false};
  r[1] = {a.delta, reach2(a.ds, a.nb, a.T, a.n, io_dtype), false};
  r[2] = {a.A, static_cast<size_t>(a.n) * N * 4, false};
  r[3] = {a.Bm, reach(vla::Rows{a.B_b, a.B_g, a.B_t}, a.nb, a.G, a.T, N, es), false};
  r[4] = {a.Cm, reach(vla::Rows{a.C_b, a.C_g, a.C_t}, a.nb, a.G, a.T, N, es), false};
  r[5] = {a.D, static_cast<size_t>(a.n) * 4, false};
  r[6] = {a.z, reach2(a.zs, a.nb, a.T, a.n, io_dtype), false};
  r[7] = {a.bias, static_cast<size_t>(a.n) * 4, false};
  r[8] = {a.lengths, static_cast<size_t>(a.nb) * 4, false};
}

// ---- norms around a block

int residual_args(const void* x, const void* y, const void* gate, const void* post_weight, const void* scale, const void* weight, int B, int T,
                  int n, int io_dtype, const vla_residual_opts* opts, vla_residual_opts* op, vla::ResidualArgs* a) {
  vla_residual_default_opts(op);
  if (opts != nullptr) *op = *opts;
  const int st = check_rows(B, T, n, io_dtype);
  if (st == VLA_ERR_INVALID_ARG) return st;
  if (!is_type(op->weight_dtype) || !is_type(op->stream_dtype) || !(op->eps > 0.0f) || !(op->eps <= 3.4e38f)) return VLA_ERR_INVALID_ARG;
  if (op->group < 0 || (op->group > 0 && n % op->group != 0) || op->activation < 0 || op->activation > 1) return VLA_ERR_INVALID_ARG;
  if (x == nullptr && y == nullptr && T > 0) return VLA_ERR_INVALID_ARG;
  if (y == nullptr && T > 0 && (gate != nullptr || post_weight != nullptr || scale != nullptr)) return VLA_ERR_INVALID_ARG;
  if (st != VLA_OK) return st;
  if (n > vla::kResidualColumns || op->group % 8 != 0 || (op->stream_dtype != io_dtype && op->stream_dtype != VLA_F32)) return VLA_ERR_UNSUPPORTED;
  const void* ptrs[] = {x, y, gate, post_weight, scale, weight};
  if (!all_aligned(ptrs, 6)) return VLA_ERR_INVALID_ARG;
  *a = vla::ResidualArgs{};
  if (!rows2(op->x, B, T, n, op->stream_dtype, false, &a->xs) || !rows2(op->y, B, T, n, io_dtype, false, &a->ys) ||
      !rows2(op->gate, B, T, n, io_dtype, false, &a->gs) || !rows2(op->s, B, T, n, op->stream_dtype, false, &a->ss) ||
      !rows2(op->h, B, T, n, io_dtype, false, &a->hs)) {
    return VLA_ERR_INVALID_ARG;
  }
  a->x = x; a->y = y; a->gate = gate; a->post_weight = post_weight; a->scale = scale; a->weight = weight;
  a->B = B; a->T = T; a->n = n;
  a->group = op->group > 0 ? op->group : n;
  a->w_bf16 = op->weight_dtype == VLA_BF16;
  a->act = op->activation;
  a->eps = op->eps;
  return VLA_OK;
}
constexpr int kResidualReads = 6;
void residual_reads(const vla::ResidualArgs& a, int io_dtype, const vla_residual_opts& op, Range* r) {
  const size_t w = static_cast<size_t>(a.n) * size_of(op.weight_dtype);
  r[0] = {a.x, reach2(a.xs, a.B, a.T, a.n, op.stream_dtype), false};
  r[1] = {a.y, reach2(a.ys, a.B, a.T, a.n, io_dtype), false};
  r[2] = {a.gate, reach2(a.gs, a.B, a.T, a.n, io_dtype), false};
  r[3] = {a.post_weight, w, false};
  r[4] = {a.scale, w, false};
  r[5] = {a.weight, w, false};
}

}  // namespace

extern "C" {

void vla_conv_default_opts(vla_conv_opts* opts) {
  if (opts == nullptr) return;
  *opts = vla_conv_opts{};
  opts->silu = 1;
}

size_t vla_causal_conv_workspace_bytes(int B, int T, int n, int width, int io_dtype) {
  if (check_rows(B, T, n, io_dtype) != VLA_OK || width < 2 || width > vla::kConvWidth) return 0;
  return conv_parts_bytes(B, T, n, width, io_dtype);
}

int vla_causal_conv(const void* x, const void* weight, const void* bias, const void* state, void* y, void* state_T, int B, int T, int n,
                    int width, int io_dtype, const vla_conv_opts* opts, void* stream) {
  vla_conv_opts op;
  vla::ConvArgs a;
  const int st = conv_args(x, weight, bias, state, B, T, n, width, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if ((T > 0 && y == nullptr) || !aligned16(y) || !aligned16(state_T)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, T, n, io_dtype, true, &a.ys)) return VLA_ERR_INVALID_ARG;
  const size_t columns = n, es = size_of(io_dtype), ws = size_of(op.weight_dtype), window = static_cast<size_t>(B) * (width - 1) * n * es;
  const Range r[] = {{x, reach2(a.xs, B, T, n, io_dtype), false}, {weight, columns * width * ws, false}, {bias, columns * ws, false}, {state, window, false},
                     {op.lengths, static_cast<size_t>(B) * 4, false}, {y, reach2(a.ys, B, T, n, io_dtype), true}, {state_T, window, true}};
  if (!disjoint(r, 7, state, state_T)) return VLA_ERR_INVALID_ARG;
  a.y = y;
  a.state_T = state_T;
  a.run = conv_run(B, T, n, io_dtype);
  a.runs = runs_of(T, a.run);
  if (!conv_fits(a, io_dtype)) return VLA_ERR_UNSUPPORTED;
  return launched(vla::launch_causal_conv(a, width, io_dtype, static_cast<hipStream_t>(stream)));
}

int vla_causal_conv_step(const void* x, const void* weight, const void* bias, void* state, void* y, int B, int n, int width, int io_dtype,
                         const vla_conv_opts* opts, void* stream) {
  vla_conv_opts op;
  vla::ConvArgs a;
  const int st = conv_args(x, weight, bias, nullptr, B, 1, n, width, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if (state == nullptr || y == nullptr || op.lengths != nullptr || !aligned16(state) || !aligned16(y)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, 1, n, io_dtype, true, &a.ys)) return VLA_ERR_INVALID_ARG;
  const size_t columns = n, es = size_of(io_dtype), ws = size_of(op.weight_dtype);
  const Range r[] = {{x, reach2(a.xs, B, 1, n, io_dtype), false}, {weight, columns * width * ws, false}, {bias, columns * ws, false},
                     {state, static_cast<size_t>(B) * (width - 1) * n * es, true}, {y, reach2(a.ys, B, 1, n, io_dtype), true}};
  if (!disjoint(r, 5, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.y = y;
  a.state_T = state;
  a.run = a.runs = 1;
  if (!conv_fits(a, io_dtype)) return VLA_ERR_UNSUPPORTED;
  return launched(vla::launch_causal_conv_step(a, width, io_dtype, static_cast<hipStream_t>(stream)));
}

int vla_causal_conv_backward(const void* x, const void* weight, const void* bias, const void* state, const void* dy, const void* dstate_T,
                             void* dx, void* dweight, void* dbias, void* dstate, int B, int T, int n, int width, int io_dtype,
                             const vla_conv_opts* opts, void* workspace, size_t workspace_bytes, void* stream) {
  vla_conv_opts op;
  vla::ConvArgs a;
  const int st = conv_args(x, weight, bias, state, B, T, n, width, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if (T > 0 && (dy == nullptr || dx == nullptr)) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {dy, dstate_T, dx, dweight, dbias, dstate, workspace};
  if (!all_aligned(ptrs, 7)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, T, n, io_dtype, false, &a.ys) || !rows2(op.dx, B, T, n, io_dtype, true, &a.dxs)) return VLA_ERR_INVALID_ARG;
  const bool sums = dweight != nullptr || dbias != nullptr;
  const size_t columns = n, need = conv_parts_bytes(B, T, n, width, io_dtype), es = size_of(io_dtype), ws = size_of(op.weight_dtype);
  if (sums && (workspace == nullptr || workspace_bytes < need)) return VLA_ERR_WORKSPACE;
  const size_t window = static_cast<size_t>(B) * (width - 1) * n * es;
  const Range r[] = {{x, reach2(a.xs, B, T, n, io_dtype), false}, {weight, columns * width * ws, false}, {bias, columns * ws, false}, {state, window, false},
                     {op.lengths, static_cast<size_t>(B) * 4, false}, {dy, reach2(a.ys, B, T, n, io_dtype), false}, {dstate_T, window, false},
                     {dx, reach2(a.dxs, B, T, n, io_dtype), true}, {dweight, columns * width * ws, true}, {dbias, columns * ws, true}, {dstate, window, true},
                     {sums ? workspace : nullptr, need, true}};
  if (!disjoint(r, 12, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.dy = dy; a.dstate_T = dstate_T; a.dx = dx; a.dstate = dstate;
  a.sum_part = sums ? static_cast<float*>(workspace) : nullptr;
  a.run = conv_run(B, T, n, io_dtype);
  a.runs = runs_of(T, a.run);
  if (!conv_fits(a, io_dtype)) return VLA_ERR_UNSUPPORTED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  a.joined = sums && conv_joined(n, io_dtype);
  const hipError_t err = vla::launch_causal_conv_backward(a, width, io_dtype, s);
  if (err != hipSuccess || !sums) return launched(err);
  const int parts = static_cast<int>(conv_parts(B, a.runs, n, io_dtype));
  vla::ColumnSums all{};
  const size_t row = static_cast<size_t>(width + 1) * n;
  for (int j = 0; j < width && dweight != nullptr; ++j) {
    all.job[all.n++] = {a.sum_part + static_cast<size_t>(j) * n, row, parts, n, static_cast<char*>(dweight) + j * ws, a.w_bf16, width};
  }
  if (dbias != nullptr) all.job[all.n++] = {a.sum_part + static_cast<size_t>(width) * n, row, parts, n, dbias, a.w_bf16, 1};
  return launched(vla::launch_column_sums(all, s));
}

void vla_scan_default_opts(vla_scan_opts* opts) {
  if (opts == nullptr) return;
  *opts = vla_scan_opts{};
  opts->softplus = 1;
  opts->groups = 1;
}

size_t vla_selective_scan_workspace_bytes(int B, int T, int n, int N, int io_dtype, const vla_scan_opts* opts, int backward) {
  const vla_scan_opts op = scan_opts(opts);
  if (check_scan(B, T, n, N, io_dtype, op) != VLA_OK) return 0;
  if (backward) return scan_backward_parts(B, T, n, N, op.groups, op.segments).bytes;
  const ScanPlan s = scan_plan(B, T, n, N, op.groups, op.segments);
  return s.h_bytes + s.dt_bytes;
}

size_t vla_selective_scan_saved_bytes(int B, int T, int n, int N, int io_dtype, const vla_scan_opts* opts) {
  const vla_scan_opts op = scan_opts(opts);
  return check_scan(B, T, n, N, io_dtype, op) == VLA_OK ? scan_saved(B, T, n, N) : 0;
}

int vla_selective_scan(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                       const float* delta_bias, const float* h0, void* y, float* h_T, int B, int T, int n, int N, int io_dtype,
                       const vla_scan_opts* opts, void* workspace, size_t workspace_bytes, void* stream) {
  const vla_scan_opts op = scan_opts(opts);
  vla::ScanArgs a;
  const int st = scan_args(u, delta, A, Bm, Cm, D, z, delta_bias, B, T, n, N, io_dtype, op, &a);
  if (st != VLA_OK) return st;
  const void* ptrs[] = {h0, y, h_T, workspace, op.saved};
  if ((T > 0 && y == nullptr) || !all_aligned(ptrs, 5)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, T, n, io_dtype, true, &a.ys)) return VLA_ERR_INVALID_ARG;
  if (!rows_near(a.ys, n, io_dtype)) return VLA_ERR_UNSUPPORTED;
  const size_t states = static_cast<size_t>(B) * n * N * 4, saved = scan_saved(B, T, n, N);
  const ScanPlan seg = scan_plan(B, T, n, N, op.groups, op.segments);
  const size_t need = seg.h_bytes + seg.dt_bytes;
  const bool cut = seg.n > 1 && workspace != nullptr && workspace_bytes >= need;
  Range r[kScanReads + 5];
  scan_reads(a, N, io_dtype, r);
  r[kScanReads] = {h0, states, false};
  r[kScanReads + 1] = {y, reach2(a.ys, B, T, n, io_dtype), true};
  r[kScanReads + 2] = {h_T, states, true};
  r[kScanReads + 3] = {cut ? workspace : nullptr, need, true};
  r[kScanReads + 4] = {op.saved, saved, true};
  if (!disjoint(r, kScanReads + 5, h0, h_T)) return VLA_ERR_INVALID_ARG;
  if (op.saved != nullptr && op.saved_bytes < saved) return VLA_ERR_WORKSPACE;
  if (T == 0 && h_T == nullptr) return VLA_OK;
  a.h0 = h0; a.y = y; a.h_T = h_T;
  a.kept = static_cast<float*>(op.saved);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = hipSuccess;
  if (cut) {
    a.n_seg = seg.n;
    a.seg_tokens = seg.tokens;
    a.seg_h = static_cast<float*>(workspace);
    a.seg_dt = reinterpret_cast<float*>(static_cast<char*>(workspace) + seg.h_bytes);
    err = vla::launch_selective_scan(a, N, io_dtype, true, s);
    if (err == hipSuccess) err = vla::launch_selective_combine(a, N, false, s);
  }
  if (err == hipSuccess) err = vla::launch_selective_scan(a, N, io_dtype, false, s);
  return launched(err);
}

int vla_selective_scan_step(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                            const float* delta_bias, float* h, void* y, int B, int n, int N, int io_dtype, const vla_scan_opts* opts,
                            void* stream) {
  const vla_scan_opts op = scan_opts(opts);
  vla::ScanArgs a;
  const int st = scan_args(u, delta, A, Bm, Cm, D, z, delta_bias, B, 1, n, N, io_dtype, op, &a);
  if (st != VLA_OK) return st;
  if (h == nullptr || y == nullptr || op.lengths != nullptr || !aligned16(h) || !aligned16(y)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, 1, n, io_dtype, true, &a.ys)) return VLA_ERR_INVALID_ARG;
  Range r[kScanReads + 2];
  scan_reads(a, N, io_dtype, r);
  r[kScanReads] = {h, static_cast<size_t>(B) * n * N * 4, true};
  r[kScanReads + 1] = {y, reach2(a.ys, B, 1, n, io_dtype), true};
  if (!disjoint(r, kScanReads + 2, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.y = y;
  a.h_T = h;
  return launched(vla::launch_selective_step(a, N, io_dtype, static_cast<hipStream_t>(stream)));
}

int vla_selective_scan_backward(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                                const float* delta_bias, const void* dy, const float* dh_T, void* du, void* ddelta, float* dA, void* dBm,
                                void* dCm, float* dD, void* dz, float* ddelta_bias, float* dh0, int B, int T, int n, int N, int io_dtype,
                                const vla_scan_opts* opts, void* workspace, size_t workspace_bytes, void* stream) {
  const vla_scan_opts op = scan_opts(opts);
  vla::ScanArgs a;
  const int st = scan_args(u, delta, A, Bm, Cm, D, z, delta_bias, B, T, n, N, io_dtype, op, &a);
  if (st != VLA_OK) return st;
  const void* needed[] = {dy, du, ddelta, dBm, dCm, op.saved};
  if (dA == nullptr || (T > 0 && any_null(needed, 6)) || (T > 0 && z != nullptr && dz == nullptr)) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {dy, dh_T, du, ddelta, dA, dBm, dCm, dD, dz, ddelta_bias, dh0, workspace, op.saved};
  if (!all_aligned(ptrs, 13)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.y, B, T, n, io_dtype, false, &a.ys) || !rows2(op.du, B, T, n, io_dtype, true, &a.dus) ||
      !rows2(op.ddelta, B, T, n, io_dtype, true, &a.dds) || !rows2(op.dz, B, T, n, io_dtype, true, &a.dzs)) {
    return VLA_ERR_INVALID_ARG;
  }
  for (const vla::Row2* r : {&a.ys, &a.dus, &a.dds, &a.dzs}) {
    if (!rows_near(*r, n, io_dtype)) return VLA_ERR_UNSUPPORTED;
  }
  const ScanBackwardParts parts = scan_backward_parts(B, T, n, N, op.groups, op.segments);
  const size_t states = static_cast<size_t>(B) * n * N * 4, saved = scan_saved(B, T, n, N);
  const size_t of_rows = static_cast<size_t>(B) * T * op.groups * N * size_of(io_dtype);
  Range r[kScanReads + 13];
  scan_reads(a, N, io_dtype, r);
  Range* w = r + kScanReads;
  w[0] = {dy, reach2(a.ys, B, T, n, io_dtype), false};
  w[1] = {dh_T, states, false};
  w[2] = {op.saved, saved, false};
  w[3] = {du, reach2(a.dus, B, T, n, io_dtype), true};
  w[4] = {ddelta, reach2(a.dds, B, T, n, io_dtype), true};
  w[5] = {dA, static_cast<size_t>(n) * N * 4, true};
  w[6] = {dBm, of_rows, true};
  w[7] = {dCm, of_rows, true};
  w[8] = {dD, static_cast<size_t>(n) * 4, true};
  w[9] = {z != nullptr ? dz : nullptr, reach2(a.dzs, B, T, n, io_dtype), true};
  w[10] = {ddelta_bias, static_cast<size_t>(n) * 4, true};
  w[11] = {dh0, states, true};
  w[12] = {workspace, parts.bytes, true};
  if (!disjoint(r, kScanReads + 13, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  if ((T > 0 && op.saved_bytes < saved) || workspace == nullptr || workspace_bytes < parts.bytes) return VLA_ERR_WORKSPACE;
  if (static_cast<long long>(B) * T * op.groups > (kMostItems - 256) / (N / 4)) return VLA_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(workspace);
  const auto at = [&](size_t offset) { return reinterpret_cast<float*>(ws + offset); };
  a.dy = dy; a.dh_T = dh_T; a.du = du; a.ddelta = ddelta; a.dz = dz; a.dh0 = dh0; a.dB = dBm; a.dC = dCm;
  a.kept = static_cast<float*>(op.saved);
  a.dA_part = at(parts.dA); a.dD_part = at(parts.dD); a.dbias_part = at(parts.dbias); a.dBC_part = at(parts.dBC);
  a.n_seg = parts.seg.n;
  if (a.n_seg > 1) a.seg_tokens = parts.seg.tokens;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = hipSuccess;
  if (a.n_seg > 1) {
    a.seg_h = at(parts.seg_h);
    a.seg_dt = at(parts.seg_dt);
    err = vla::launch_selective_backward(a, N, io_dtype, true, s);
    if (err == hipSuccess) err = vla::launch_selective_combine(a, N, true, s);
  }
  if (err == hipSuccess) err = vla::launch_selective_backward(a, N, io_dtype, false, s);
  if (err == hipSuccess) err = vla::launch_selective_shared(a, N, io_dtype, s);
  if (err != hipSuccess) return launched(err);
  vla::ColumnSums all{};
  const int rows = B * a.n_seg;
  all.job[all.n++] = {a.dA_part, static_cast<size_t>(n) * N, rows, n * N, dA, 0, 1};
  if (dD != nullptr) all.job[all.n++] = {a.dD_part, static_cast<size_t>(n), rows, n, dD, 0, 1};
  if (ddelta_bias != nullptr) all.job[all.n++] = {a.dbias_part, static_cast<size_t>(n), rows, n, ddelta_bias, 0, 1};
  return launched(vla::launch_column_sums(all, s));
}

void vla_residual_default_opts(vla_residual_opts* opts) {
  if (opts == nullptr) return;
  *opts = vla_residual_opts{};
  opts->eps = 1e-6f;
}

size_t vla_residual_norm_workspace_bytes(int n) {
  return n > 0 && n % 8 == 0 && n <= vla::kResidualColumns ? static_cast<size_t>(vla::residual_partials(n)) * 3 * n * 4 : 0;
}

int vla_residual_norm(const void* x, const void* y, const void* gate, const void* post_weight, const void* scale, const void* weight, void* s,
                      void* h, int B, int T, int n, int io_dtype, const vla_residual_opts* opts, void* stream) {
  vla_residual_opts op;
  vla::ResidualArgs a;
  const int st = residual_args(x, y, gate, post_weight, scale, weight, B, T, n, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if (T == 0) return VLA_OK;
  if ((y != nullptr) != (s != nullptr) || (weight != nullptr) != (h != nullptr) || !aligned16(s) || !aligned16(h)) return VLA_ERR_INVALID_ARG;
  vla::Row2 unused;
  if (!rows2(op.s, B, T, n, op.stream_dtype, true, &unused) || !rows2(op.h, B, T, n, io_dtype, true, &unused)) return VLA_ERR_INVALID_ARG;
  Range r[kResidualReads + 2];
  residual_reads(a, io_dtype, op, r);
  r[kResidualReads] = {s, reach2(a.ss, B, T, n, op.stream_dtype), true};
  r[kResidualReads + 1] = {h, reach2(a.hs, B, T, n, io_dtype), true};
  const bool in_place = a.xs.b == a.ss.b && a.xs.t == a.ss.t;
  if (!disjoint(r, kResidualReads + 2, in_place ? x : nullptr, s)) return VLA_ERR_INVALID_ARG;
  a.s = s;
  a.h = h;
  return launched(vla::launch_residual_norm(a, io_dtype, op.stream_dtype, static_cast<hipStream_t>(stream)));
}

int vla_residual_norm_backward(const void* x, const void* y, const void* gate, const void* post_weight, const void* scale, const void* weight,
                               const void* ds, const void* dh, void* dx, void* dy, void* dgate, void* dpost_weight, void* dscale, void* dweight,
                               int B, int T, int n, int io_dtype, const vla_residual_opts* opts, void* workspace, size_t workspace_bytes,
                               void* stream) {
  vla_residual_opts op;
  vla::ResidualArgs a;
  const int st = residual_args(x, y, gate, post_weight, scale, weight, B, T, n, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if ((dh != nullptr && weight == nullptr) || (dx != nullptr && x == nullptr) || (dy != nullptr && y == nullptr) ||
      (dgate != nullptr && gate == nullptr) || (dpost_weight != nullptr && post_weight == nullptr) || (dscale != nullptr && scale == nullptr) ||
      (dweight != nullptr && weight == nullptr)) {
    return VLA_ERR_INVALID_ARG;
  }
  const void* ptrs[] = {ds, dh, dx, dy, dgate, dpost_weight, dscale, dweight, workspace};
  if (!all_aligned(ptrs, 9)) return VLA_ERR_INVALID_ARG;
  if (!rows2(op.dx, B, T, n, op.stream_dtype, true, &a.dxs) || !rows2(op.dy, B, T, n, io_dtype, true, &a.dys) ||
      !rows2(op.dgate, B, T, n, io_dtype, true, &a.dgs)) {
    return VLA_ERR_INVALID_ARG;
  }
  const bool sums = dpost_weight != nullptr || dscale != nullptr || dweight != nullptr;
  const size_t need = vla_residual_norm_workspace_bytes(n), w = static_cast<size_t>(n) * size_of(op.weight_dtype);
  if (sums && (workspace == nullptr || workspace_bytes < need)) return VLA_ERR_WORKSPACE;
  Range r[kResidualReads + 9];
  residual_reads(a, io_dtype, op, r);
  Range* q = r + kResidualReads;
  q[0] = {ds, reach2(a.ss, B, T, n, op.stream_dtype), false};
  q[1] = {dh, reach2(a.hs, B, T, n, io_dtype), false};
  q[2] = {dx, reach2(a.dxs, B, T, n, op.stream_dtype), true};
  q[3] = {dy, reach2(a.dys, B, T, n, io_dtype), true};
  q[4] = {dgate, reach2(a.dgs, B, T, n, io_dtype), true};
  q[5] = {dpost_weight, w, true};
  q[6] = {dscale, w, true};
  q[7] = {dweight, w, true};
  q[8] = {sums ? workspace : nullptr, need, true};
  if (!disjoint(r, kResidualReads + 9, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.ds = ds; a.dh = dh; a.dx = dx; a.dy = dy; a.dgate = dgate;
  a.sum_part = sums ? static_cast<float*>(workspace) : nullptr;
  const hipStream_t stm = static_cast<hipStream_t>(stream);
  int rows = 0;
  const hipError_t err = vla::launch_residual_norm_backward(a, io_dtype, op.stream_dtype, &rows, stm);
  if (err != hipSuccess || !sums) return launched(err);
  vla::ColumnSums all{};
  void* out[3] = {dweight, dpost_weight, dscale};
  for (int j = 0; j < 3; ++j) {
    if (out[j] != nullptr) all.job[all.n++] = {a.sum_part + static_cast<size_t>(j) * n, 3 * static_cast<size_t>(n), rows, n, out[j], a.w_bf16, 1};
  }
  return launched(vla::launch_column_sums(all, stm));
}

}  // extern "C"

// Host side of the operators around the recurrence (include/vla.h): validation and dispatch of the gated delta rule and of the
// norm of queries and keys with the position rotation.
#include "../../include/vla.h"

#include "host_checks.h"
#include "layer_common.h"

#include <math.h>

namespace {

// the kernels address the rows of a block of 32 tokens with 31-bit byte offsets
bool rows_near(const vla::Rows& r, size_t es) { return r.t < 0x7fffffffLL / 32 / static_cast<long long>(es); }

// ---- gated delta rule

int check_delta(int B, int H_k, int H_v, int T, int d_k, int d_v, int io_dtype, const vla_delta_opts& o) {
  if (B <= 0 || H_k <= 0 || H_v <= 0 || T < 0 || d_k <= 0 || d_v <= 0 || H_v % H_k != 0) return VLA_ERR_INVALID_ARG;
  if (io_dtype != VLA_F32 && io_dtype != VLA_BF16) return VLA_ERR_INVALID_ARG;
  if (!(fabsf(o.scale) <= 3.4e38f) || o.segments < 0) return VLA_ERR_INVALID_ARG;
  if (!vla::layer_head_size(d_k) || !vla::layer_head_size(d_v)) return VLA_ERR_UNSUPPORTED;
  // workgroups (up to 32 a head and segment) and tokens with a block of look-ahead are 32-bit indices; a workgroup has a wave for 16 columns
  if (static_cast<long long>(B) * H_v > 0x7fffffff / 32 || T > 0x7fffff00) return VLA_ERR_UNSUPPORTED;
  if (!fits_launch(static_cast<long long>(B) * H_v, 4 * d_v)) return VLA_ERR_UNSUPPORTED;
  return VLA_OK;
}
vla_delta_opts delta_opts(const vla_delta_opts* o, int d_k) {
  vla_delta_opts r;
  vla_delta_default_opts(&r);
  if (o != nullptr) r = *o;
  if (r.scale == 0.0f && d_k > 0) r.scale = 1.0f / sqrtf(static_cast<float>(d_k));
  return r;
}

// Strides of the gates: any, in elements.
bool gate_rows(const vla_strides& s, long long H, long long T, vla::Rows* out) {
  *out = vla::Rows{s.b, s.h, s.t};
  if (s.b == 0 && s.h == 0 && s.t == 0) *out = vla::Rows{H * T, T, 1};
  return out->b >= 0 && out->h >= 0 && out->t >= 0;
}

// Time segments of a sequence.  Few heads leave most of the card idle; in segments the sequence goes through twice (maps, then outputs:
// 2.6 times the work of a block, one after the other).  `held`: the maps' workgroups of (d_v + d_k) / 16 waves that the card holds at
// once for each head.  The first of 3 to 17 segments goes with the maps of the others (first), which allows held + 1 of them: with more they get hardly
// shorter, and the first one takes longer than a map.  Where that is not done (d_v < 64) twice as many still gain with small heads.
// The number of segments, of 1, 2, 3, 4, 6, 8 ... blocks or as many as the card holds, is the one of least time by a model that is fitted to measurements
// of 1 to 33 segments for 4 to 256 heads of 16 to 128 columns and 192 to 4096 tokens (microseconds): a block by the rounds in which its waves
// form the six matrices between tokens and by its products; a map by its waves; a step from one segment to the next d_k / 60; d_k / 8 for the
// launches.  Against the best of up to 12 other numbers at 150 points (profiles/gated_delta_segments.txt) its choices take 1 % more in the geometric mean
// and 4.5 % or less at nine in ten; at worst 19 % (16 heads of 32, float32, 4096 tokens: 73, 62 with 32 segments) and 15 % (256 heads of 128 x 64, bf16,
// 4096 tokens: 709, 614 with 3).  With the backward pass, whose chain is cut alike: 0.2 %, 1.5 %, 11 %.
// Forward, microseconds, bf16 but where said, 1 segment and the rule's:
//   4 heads of 64: 256 tokens 27, 22 (8 segments); 1024 tokens 94, 34 (16).  The same in float32 41, 24 and 151, 41
//   4 heads of 128: 256 tokens 36, 36 (none; 4: 38); 384 tokens 51, 43 (6); 1024 tokens 124, 61 (11); 32 heads, 1024 tokens 124, 68 (8)
//   128 heads of 128: 768 tokens 95, 95 (none; 3: 100); 1536 tokens 184, 162 (3); 4096 tokens 479, 382 (3)
//   64 heads of 128, 4096 tokens: 475, 248 (5; all maps, 4: 293); 16 heads, 32768 tokens, 17: 540 (16: 561); one head 266 (64; 32: 325, 128: 328)
//   128 heads of 64, 4096 tokens: 370, 190 (5); 256 heads: 512 tokens 50, 50 (none; 3: 58); 4096 tokens 371, 303 (3)
//   39 heads of 128 x 64, float32, 1537 tokens: 338, 140 (7; all maps, 6: 171)
struct Segments {
  int n, tokens, slots;
  bool first;
  size_t map_bytes, bytes;   // of the maps, of both arrays
};
Segments delta_segments(long long heads, int T, int d_k, int d_v, int io_dtype, int requested) {
  Segments s{1, T, 1, false, 0, 0};
  const int blocks = (T + 31) / 32;
  const bool can = vla::delta_first_with_maps(d_v);
  long long n = requested;
  if (requested == 0) {
    const int waves = (d_v + d_k) / 16;
    const long long slots = 256 * (waves < 16 ? 16 / waves : 1), held = slots / heads;
    const long long most = can ? (held <= 16 ? held + 1 : held) : (waves <= 8 ? 2 : 1) * held;
    const bool f32 = io_dtype == VLA_F32;
    const int rounds = (6 + d_v / 16 - 1) / (d_v / 16);       // of the matrices between tokens on d_v / 16 waves
    const float block = f32 ? (0.6f + 0.002f * d_k) * rounds + (1.2f + 0.032f * d_k) * (d_v > 64 ? 1.6f : 1.0f)
                            : 1.4f + 0.45f * rounds + 1.1e-4f * d_k * d_k + (d_v > 64 ? 1.4f - 0.011f * d_k : 0.0f);
    const float both = block + 2.0f + (f32 ? 0.6f : 0.18f) * waves;
    float least = 0.97f * (block * blocks + 7.0f);
    n = 1;
    const auto consider = [&](long long each) {      // blocks of a segment
      const long long m = (blocks + each - 1) / each;
      if (m < 2 || m > most || m > 256) return;
      const long long maps = heads * (m - (can ? 1 : 0));
      const float crowd = 2 * maps < slots || waves > 8 ? 1.0f : (1.0f + 0.8f / waves) * (f32 ? 1.25f : 1.0f);
      const float time = both * each * crowd * (maps > slots ? 2.1f : 1.0f) + d_k / 60.0f * m + d_k / 8.0f +
                         (2 * maps >= slots ? 4.0f : -3.0f);
      if (time < least) {
        least = time;
        n = m;
      }
    };
    if (held >= 2 && blocks >= (f32 ? 6 : 8)) {
      for (long long each = 1; each < blocks; each *= 2) {
        consider(each);
        consider(each + (each + 1) / 2);
      }
      consider((blocks + most - 1) / most);
    }
  }
  if (n > blocks) n = blocks;
  if (n > 256) n = 256;
  if (n > kMostItems / (heads * 4 * (d_v + d_k))) n = kMostItems / (heads * 4 * (d_v + d_k));   // work-items of the maps
  if (!fits_launch(heads * (d_v / 16), 4 * d_k)) n = 1;                                         // of the states between segments
  if (n <= 1) return s;
  const int each = static_cast<int>((blocks + n - 1) / n);
  s.n = (blocks + each - 1) / each;
  s.tokens = 32 * each;
  s.first = can && s.n >= 3 && s.n <= 17;
  s.slots = s.n - (s.first ? 1 : 0);
  s.map_bytes = static_cast<size_t>(heads) * s.slots * (d_v + d_k) * d_k * 4;
  s.bytes = s.map_bytes + static_cast<size_t>(heads) * s.slots * d_v * d_k * 4;
  return s;
}

// What the forward pass keeps, and what the backward pass works on; each part starts at a multiple of 256 bytes.
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
int kept_states(int T) { return (T + vla::kKeep - 1) / vla::kKeep; }
size_t kept_bytes(long long heads, int T, int d_k, int d_v) { return padded(static_cast<size_t>(heads) * kept_states(T) * d_v * d_k * 4); }
size_t row_bytes(long long heads, int T, int d) { return padded(static_cast<size_t>(heads) * T * d * 4); }
struct BackwardParts {
  Segments seg;
  size_t kept, rows, dk, dq, seg_map, seg_S, bytes;   // offsets
};
BackwardParts backward_parts(long long heads, int T, int d_k, int d_v, int io_dtype, bool shared, int requested) {
  BackwardParts p{};
  p.seg = delta_segments(heads, T, d_k, d_v, io_dtype, requested);
  p.kept = 0;
  p.rows = p.kept + kept_bytes(heads, T, d_k, d_v);
  p.dk = p.rows + row_bytes(heads, T, d_v);
  p.dq = p.dk + row_bytes(heads, T, d_k);
  p.seg_map = p.dq + (shared ? row_bytes(heads, T, d_k) : 0);
  p.seg_S = p.seg_map + padded(p.seg.map_bytes);
  p.bytes = p.seg_S + padded(p.seg.bytes - p.seg.map_bytes);
  return p;
}

hipError_t launch_reverse(const vla::DeltaArgs& a, int d_k, int d_v, int io_dtype, bool map, hipStream_t stream) {
  switch (d_k) {
    case 16: return vla::launch_delta_reverse_16(a, d_v, io_dtype, map, stream);
    case 32: return vla::launch_delta_reverse_32(a, d_v, io_dtype, map, stream);
    case 64: return vla::launch_delta_reverse_64(a, d_v, io_dtype, map, stream);
    case 96: return vla::launch_delta_reverse_96(a, d_v, io_dtype, map, stream);
    case 128: return vla::launch_delta_reverse_128(a, d_v, io_dtype, map, stream);
    default: return hipErrorInvalidValue;
  }
}
hipError_t launch_grad(const vla::DeltaArgs& a, int d_k, int d_v, int io_dtype, hipStream_t stream) {
  switch (d_k) {
    case 16: return vla::launch_delta_grad_16(a, d_v, io_dtype, stream);
    case 32: return vla::launch_delta_grad_32(a, d_v, io_dtype, stream);
    case 64: return vla::launch_delta_grad_64(a, d_v, io_dtype, stream);
    case 96: return vla::launch_delta_grad_96(a, d_v, io_dtype, stream);
    case 128: return vla::launch_delta_grad_128(a, d_v, io_dtype, stream);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_blocks(const vla::DeltaArgs& a, int d_k, int d_v, int io_dtype, bool map, hipStream_t stream) {
  switch (d_k) {
    case 16: return vla::launch_delta_chunk_16(a, d_v, io_dtype, map, stream);
    case 32: return vla::launch_delta_chunk_32(a, d_v, io_dtype, map, stream);
    case 64: return vla::launch_delta_chunk_64(a, d_v, io_dtype, map, stream);
    case 96: return vla::launch_delta_chunk_96(a, d_v, io_dtype, map, stream);
    case 128: return vla::launch_delta_chunk_128(a, d_v, io_dtype, map, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

extern "C" {

void vla_delta_default_opts(vla_delta_opts* opts) {
  if (opts != nullptr) *opts = vla_delta_opts{};
}

size_t vla_delta_workspace_bytes(int B, int H_k, int H_v, int T, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts, int backward) {
  const vla_delta_opts op = delta_opts(opts, d_k);
  if (check_delta(B, H_k, H_v, T, d_k, d_v, io_dtype, op) != VLA_OK) return 0;
  const long long heads = static_cast<long long>(B) * H_v;
  if (!backward) return delta_segments(heads, T, d_k, d_v, io_dtype, op.segments).bytes;
  return backward_parts(heads, T, d_k, d_v, io_dtype, H_v != H_k, op.segments).bytes;
}

size_t vla_delta_saved_bytes(int B, int H_v, int T, int d_k, int d_v, int io_dtype) {
  vla_delta_opts op;
  vla_delta_default_opts(&op);
  if (check_delta(B, 1, H_v, T, d_k, d_v, io_dtype, op) != VLA_OK) return 0;
  return kept_bytes(static_cast<long long>(B) * H_v, T, d_k, d_v) + row_bytes(static_cast<long long>(B) * H_v, T, d_v);
}
int vla_delta_forward(const void* q, const void* k, const void* v, const float* g, const float* beta, const float* S0, void* o,
                      float* S_T, int B, int H_k, int H_v, int T, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts,
                      void* workspace, size_t workspace_bytes, void* stream) {
  const vla_delta_opts op = delta_opts(opts, d_k);
  const int st = check_delta(B, H_k, H_v, T, d_k, d_v, io_dtype, op);
  if (st != VLA_OK) return st;
  if (T > 0 && (q == nullptr || k == nullptr || v == nullptr || g == nullptr || beta == nullptr || o == nullptr)) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {q, k, v, S0, o, S_T};
  for (const void* p : ptrs) {
    if (!aligned16(p)) return VLA_ERR_INVALID_ARG;
  }
  const size_t es = io_dtype == VLA_BF16 ? 2 : 4;
  const int per16 = static_cast<int>(16 / es);
  vla::DeltaArgs a{};
  if (!rows_of(op.q, H_k, T, d_k, per16, &a.qs) || !rows_of(op.k, H_k, T, d_k, per16, &a.ks) || !rows_of(op.v, H_v, T, d_v, per16, &a.vs) ||
      !rows_of(op.o, H_v, T, d_v, per16, &a.os) || !gate_rows(op.g, H_v, T, &a.gs) || !gate_rows(op.beta, H_v, T, &a.bs) ||
      !rows_apart(a.os, B, H_v, T, d_v) || !tokens_apart(a.qs, T, d_k) || !tokens_apart(a.ks, T, d_k) || !tokens_apart(a.vs, T, d_v)) {
    return VLA_ERR_INVALID_ARG;
  }
  for (const vla::Rows* r : {&a.qs, &a.ks, &a.vs, &a.os}) {
    if (!rows_near(*r, es)) return VLA_ERR_UNSUPPORTED;
  }
  const size_t nS = static_cast<size_t>(B) * H_v * d_v * d_k * 4;
  const Range r[] = {{q, reach(a.qs, B, H_k, T, d_k, es), false}, {k, reach(a.ks, B, H_k, T, d_k, es), false},
                     {v, reach(a.vs, B, H_v, T, d_v, es), false}, {g, reach(a.gs, B, H_v, T, 1, 4), false},
                     {beta, reach(a.bs, B, H_v, T, 1, 4), false}, {op.lengths, static_cast<size_t>(B) * 4, false},
                     {S0, nS, false}, {o, reach(a.os, B, H_v, T, d_v, es), true}, {S_T, nS, true}, {workspace, workspace_bytes, true},
                     {op.saved, op.saved_bytes, true}};
  if (!aligned16(workspace) || !aligned16(op.saved) || !disjoint(r, 11, S0, S_T)) return VLA_ERR_INVALID_ARG;
  if (op.saved != nullptr && op.saved_bytes < vla_delta_saved_bytes(B, H_v, T, d_k, d_v, io_dtype)) return VLA_ERR_WORKSPACE;
  if (T == 0 && S_T == nullptr) return VLA_OK;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.S0 = S0; a.o = o; a.S_T = S_T;
  a.lengths = op.lengths;
  a.B = B; a.H_k = H_k; a.H_v = H_v; a.T = T;
  a.scale = op.scale;
  a.n_seg = 1;
  a.seg_tokens = T;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (op.saved != nullptr) {
    a.n_kept = kept_states(T);
    a.kept = static_cast<float*>(op.saved);
    a.rows = reinterpret_cast<float*>(static_cast<char*>(op.saved) + kept_bytes(static_cast<long long>(B) * H_v, T, d_k, d_v));
  }
  const long long heads = static_cast<long long>(B) * H_v;
  if (T < 16 && op.saved == nullptr && fits_launch(heads * (d_v / 16), 256)) return launched(vla::launch_delta_step(a, d_k, d_v, io_dtype, s));
  Segments seg = delta_segments(heads, T, d_k, d_v, io_dtype, op.segments);
  if (seg.n == 1 || workspace == nullptr || workspace_bytes < seg.bytes) return launched(launch_blocks(a, d_k, d_v, io_dtype, false, s));
  a.n_seg = seg.n;
  a.seg_tokens = seg.tokens;
  a.first_done = seg.first;
  a.n_slots = seg.slots;
  a.seg_map = static_cast<float*>(workspace);
  a.seg_S = reinterpret_cast<float*>(static_cast<char*>(workspace) + seg.map_bytes);
  hipError_t err = launch_blocks(a, d_k, d_v, io_dtype, true, s);
  if (err == hipSuccess) err = vla::launch_delta_combine(a, d_k, d_v, false, s);
  if (err != hipSuccess) return launched(err);
  a.S0 = a.seg_S;
  a.seg_S = nullptr;
  a.seg_states = true;
  return launched(launch_blocks(a, d_k, d_v, io_dtype, false, s));
}

int vla_delta_decode_step(const void* q, const void* k, const void* v, const float* g, const float* beta, float* S, void* o, int B,
                          int H_k, int H_v, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts, void* stream) {
  if (S == nullptr) return VLA_ERR_INVALID_ARG;
  return vla_delta_forward(q, k, v, g, beta, S, o, S, B, H_k, H_v, 1, d_k, d_v, io_dtype, opts, nullptr, 0, stream);
}

int vla_delta_backward(const void* q, const void* k, const void* v, const float* g, const float* beta, const void* dO, const float* dS_T,
                       void* dq, void* dk, void* dv, float* dg, float* dbeta, float* dS0, int B, int H_k, int H_v, int T, int d_k,
                       int d_v, int io_dtype, const vla_delta_opts* opts, void* workspace, size_t workspace_bytes, void* stream) {
  const vla_delta_opts op = delta_opts(opts, d_k);
  const int st = check_delta(B, H_k, H_v, T, d_k, d_v, io_dtype, op);
  if (st != VLA_OK) return st;
  const void* needed[] = {q, k, v, g, beta, dO, dq, dk, dv, dg, dbeta, op.saved};
  for (const void* p : needed) {
    if (T > 0 && p == nullptr) return VLA_ERR_INVALID_ARG;
  }
  const void* ptrs[] = {q, k, v, dO, dS_T, dq, dk, dv, dS0, op.saved, workspace};
  for (const void* p : ptrs) {
    if (!aligned16(p)) return VLA_ERR_INVALID_ARG;
  }
  const size_t es = io_dtype == VLA_BF16 ? 2 : 4;
  const int per16 = static_cast<int>(16 / es);
  vla::DeltaArgs a{};
  if (!rows_of(op.q, H_k, T, d_k, per16, &a.qs) || !rows_of(op.k, H_k, T, d_k, per16, &a.ks) || !rows_of(op.v, H_v, T, d_v, per16, &a.vs) ||
      !rows_of(op.o, H_v, T, d_v, per16, &a.os) || !rows_of(op.dq, H_k, T, d_k, per16, &a.dqs) || !rows_of(op.dk, H_k, T, d_k, per16, &a.dks) ||
      !rows_of(op.dv, H_v, T, d_v, per16, &a.dvs) || !gate_rows(op.g, H_v, T, &a.gs) || !gate_rows(op.beta, H_v, T, &a.bs) ||
      !tokens_apart(a.qs, T, d_k) || !tokens_apart(a.ks, T, d_k) || !tokens_apart(a.vs, T, d_v) || !tokens_apart(a.os, T, d_v) ||
      !rows_apart(a.dqs, B, H_k, T, d_k) || !rows_apart(a.dks, B, H_k, T, d_k) || !rows_apart(a.dvs, B, H_v, T, d_v)) {
    return VLA_ERR_INVALID_ARG;
  }
  for (const vla::Rows* r : {&a.qs, &a.ks, &a.vs, &a.os, &a.dqs, &a.dks, &a.dvs}) {
    if (!rows_near(*r, es)) return VLA_ERR_UNSUPPORTED;
  }
  const long long heads = static_cast<long long>(B) * H_v;
  if (!fits_launch(heads * kept_states(T), 4 * d_k)) return VLA_ERR_UNSUPPORTED;
  const BackwardParts parts = backward_parts(heads, T, d_k, d_v, io_dtype, H_v != H_k, op.segments);
  const size_t nS = static_cast<size_t>(heads) * d_v * d_k * 4, nG = static_cast<size_t>(heads) * T * 4;
  const size_t saved = vla_delta_saved_bytes(B, H_v, T, d_k, d_v, io_dtype);
  const Range r[] = {{q, reach(a.qs, B, H_k, T, d_k, es), false}, {k, reach(a.ks, B, H_k, T, d_k, es), false},
                     {v, reach(a.vs, B, H_v, T, d_v, es), false}, {g, reach(a.gs, B, H_v, T, 1, 4), false},
                     {beta, reach(a.bs, B, H_v, T, 1, 4), false}, {op.lengths, static_cast<size_t>(B) * 4, false},
                     {dO, reach(a.os, B, H_v, T, d_v, es), false}, {dS_T, nS, false}, {op.saved, saved, false},
                     {dq, reach(a.dqs, B, H_k, T, d_k, es), true}, {dk, reach(a.dks, B, H_k, T, d_k, es), true},
                     {dv, reach(a.dvs, B, H_v, T, d_v, es), true}, {dg, nG, true}, {dbeta, nG, true}, {dS0, nS, true},
                     {workspace, parts.bytes, true}};
  if (!disjoint(r, 16, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  if (op.saved_bytes < saved || (parts.bytes > 0 && (workspace == nullptr || workspace_bytes < parts.bytes))) return VLA_ERR_WORKSPACE;
  if (T == 0 && dS0 == nullptr) return VLA_OK;
  char* ws = static_cast<char*>(workspace);
  const auto at = [&](size_t offset) { return reinterpret_cast<float*>(ws + offset); };
  const hipStream_t s = static_cast<hipStream_t>(stream);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.dO = dO; a.S0 = dS_T; a.S_T = dS0; a.dv = dv;
  a.lengths = op.lengths;
  a.B = B; a.H_k = H_k; a.H_v = H_v; a.T = T;
  a.scale = op.scale;
  a.kept = at(parts.kept);
  a.rows = at(parts.rows);
  a.n_kept = kept_states(T);
  a.n_seg = parts.seg.n;
  a.seg_tokens = parts.seg.tokens;
  a.first_done = parts.seg.first;
  a.n_slots = parts.seg.slots;
  // W, dv, the state's gradient at the places that are kept
  vla::DeltaArgs chain = a;
  hipError_t err = hipSuccess;
  if (a.n_seg > 1) {
    chain.seg_map = at(parts.seg_map);
    chain.seg_S = at(parts.seg_S);
    err = launch_reverse(chain, d_k, d_v, io_dtype, true, s);
    if (err == hipSuccess) err = vla::launch_delta_combine(chain, d_k, d_v, true, s);
    chain.S0 = chain.seg_S;
    chain.seg_S = nullptr;
    chain.seg_states = true;
  }
  if (err == hipSuccess) err = launch_reverse(chain, d_k, d_v, io_dtype, false, s);
  if (err != hipSuccess || T == 0) return launched(err);
  // the other gradients
  a.kept_state = static_cast<const float*>(op.saved);
  a.R = reinterpret_cast<const float*>(static_cast<const char*>(op.saved) + kept_bytes(heads, T, d_k, d_v));
  a.dq = dq; a.dk = dk; a.dg = dg; a.dbeta = dbeta;
  a.dk_part = at(parts.dk);
  a.dq_part = H_v != H_k ? at(parts.dq) : nullptr;
  err = launch_grad(a, d_k, d_v, io_dtype, s);
  if (err == hipSuccess && H_v != H_k) err = vla::launch_delta_shared(a, d_k, io_dtype, s);
  return launched(err);
}

// ---- norm of queries and keys with the position rotation

void vla_norm_default_opts(vla_norm_opts* opts) {
  if (opts == nullptr) return;
  *opts = vla_norm_opts{};
  opts->eps = 1e-6f;
}

size_t vla_qk_norm_rope_workspace_bytes(int d) {
  return vla::layer_head_size(d) ? static_cast<size_t>(vla::kNormPartials) * 2 * d * 4 : 0;
}

}  // extern "C"

namespace {

// What the two directions check and fill in alike.
int norm_args(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos, const float* sin, int B, int T,
              int H_q, int H_k, int d, int io_dtype, const vla_norm_opts* opts, vla_norm_opts* op, vla::NormArgs* a) {
  vla_norm_default_opts(op);
  if (opts != nullptr) *op = *opts;
  if (B <= 0 || T < 0 || H_q < 0 || H_k < 0 || H_q + H_k <= 0 || d <= 0) return VLA_ERR_INVALID_ARG;
  if (io_dtype != VLA_F32 && io_dtype != VLA_BF16) return VLA_ERR_INVALID_ARG;
  if (op->weight_dtype != VLA_F32 && op->weight_dtype != VLA_BF16) return VLA_ERR_INVALID_ARG;
  if (!(op->eps > 0.0f) || !(op->eps <= 3.4e38f) || op->places < 0 || op->offset < 0) return VLA_ERR_INVALID_ARG;
  const int rot = op->rot == 0 ? (cos != nullptr ? d : 0) : op->rot;
  if (rot < 0 || rot > d || rot % 8 != 0) return VLA_ERR_INVALID_ARG;
  if (rot > 0 && (cos == nullptr || sin == nullptr || op->places <= 0)) return VLA_ERR_INVALID_ARG;
  if (!vla::layer_head_size(d)) return VLA_ERR_UNSUPPORTED;
  if (static_cast<long long>(B) * T > 0x7fffff00LL || H_q > 32767 || H_k > 32767) return VLA_ERR_UNSUPPORTED;
  if (T > 0 && ((H_q > 0 && q == nullptr) || (H_k > 0 && k == nullptr))) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {q, k, q_weight, k_weight, cos, sin};
  for (const void* p : ptrs) {
    if (!aligned16(p)) return VLA_ERR_INVALID_ARG;
  }
  *a = vla::NormArgs{};
  const int per16 = io_dtype == VLA_BF16 ? 8 : 4;
  if (!rows_of(op->q, H_q, T, d, per16, &a->xs[0]) || !rows_of(op->k, H_k, T, d, per16, &a->xs[1]) ||
      !rows_of(op->q_out, H_q, T, d, per16, &a->ys[0]) || !rows_of(op->k_out, H_k, T, d, per16, &a->ys[1])) {
    return VLA_ERR_INVALID_ARG;
  }
  a->x[0] = q; a->x[1] = k; a->w[0] = q_weight; a->w[1] = k_weight;
  a->cos = cos; a->sin = sin;
  a->positions = op->positions;
  a->H[0] = H_q; a->H[1] = H_k;
  a->B = B; a->T = T; a->rot = rot; a->offset = op->offset;
  a->places = rot > 0 ? op->places : 0x7fffffff;
  if (rot == 0) a->positions = nullptr;   // nothing is looked up
  if (rot == 0) a->offset = 0;
  a->eps = op->eps;
  a->inv_n = op->l2 ? 1.0f : 1.0f / static_cast<float>(d);
  a->w_bf16 = op->weight_dtype == VLA_BF16;
  return VLA_OK;
}

}  // namespace

extern "C" {

int vla_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos, const float* sin,
                     void* q_out, void* k_out, int B, int T, int H_q, int H_k, int d, int io_dtype, const vla_norm_opts* opts,
                     void* stream) {
  vla_norm_opts op;
  vla::NormArgs a;
  const int st = norm_args(q, k, q_weight, k_weight, cos, sin, B, T, H_q, H_k, d, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  if (T == 0) return VLA_OK;
  if ((H_q > 0 && q_out == nullptr) || (H_k > 0 && k_out == nullptr) || !aligned16(q_out) || !aligned16(k_out)) return VLA_ERR_INVALID_ARG;
  if (!rows_apart(a.ys[0], B, H_q, T, d) || !rows_apart(a.ys[1], B, H_k, T, d)) return VLA_ERR_INVALID_ARG;
  const size_t es = io_dtype == VLA_BF16 ? 2 : 4, ws = op.weight_dtype == VLA_BF16 ? 2 : 4, table = static_cast<size_t>(op.places) * (a.rot / 2) * 4;
  const Range r[] = {{q, reach(a.xs[0], B, H_q, T, d, es), false}, {k, reach(a.xs[1], B, H_k, T, d, es), false},
                     {q_weight, d * ws, false}, {k_weight, d * ws, false}, {a.rot ? cos : nullptr, table, false},
                     {a.rot ? sin : nullptr, table, false}, {a.positions, static_cast<size_t>(B) * T * 4, false},
                     {q_out, reach(a.ys[0], B, H_q, T, d, es), true}, {k_out, reach(a.ys[1], B, H_k, T, d, es), true}};
  if (!disjoint(r, 9, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.y[0] = q_out; a.y[1] = k_out;
  return launched(vla::launch_qk_norm_rope(a, d, io_dtype, op.interleaved != 0, static_cast<hipStream_t>(stream)));
}

int vla_qk_norm_rope_backward(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos,
                              const float* sin, const void* dq_out, const void* dk_out, void* dq, void* dk, void* dq_weight,
                              void* dk_weight, int B, int T, int H_q, int H_k, int d, int io_dtype, const vla_norm_opts* opts,
                              void* workspace, size_t workspace_bytes, void* stream) {
  vla_norm_opts op;
  vla::NormArgs a;
  const int st = norm_args(q, k, q_weight, k_weight, cos, sin, B, T, H_q, H_k, d, io_dtype, opts, &op, &a);
  if (st != VLA_OK) return st;
  const int per16 = io_dtype == VLA_BF16 ? 8 : 4;
  if (!rows_of(op.dq, H_q, T, d, per16, &a.dxs[0]) || !rows_of(op.dk, H_k, T, d, per16, &a.dxs[1])) return VLA_ERR_INVALID_ARG;
  if (T > 0 && ((H_q > 0 && (dq_out == nullptr || dq == nullptr)) || (H_k > 0 && (dk_out == nullptr || dk == nullptr)))) return VLA_ERR_INVALID_ARG;
  const void* ptrs[] = {dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace};
  for (const void* p : ptrs) {
    if (!aligned16(p)) return VLA_ERR_INVALID_ARG;
  }
  if (!rows_apart(a.dxs[0], B, H_q, T, d) || !rows_apart(a.dxs[1], B, H_k, T, d)) return VLA_ERR_INVALID_ARG;
  const bool sums = dq_weight != nullptr || dk_weight != nullptr;
  const size_t need = vla_qk_norm_rope_workspace_bytes(d);
  if (sums && (workspace == nullptr || workspace_bytes < need)) return VLA_ERR_WORKSPACE;
  const size_t es = io_dtype == VLA_BF16 ? 2 : 4, ws = op.weight_dtype == VLA_BF16 ? 2 : 4, table = static_cast<size_t>(op.places) * (a.rot / 2) * 4;
  const size_t nq = reach(a.xs[0], B, H_q, T, d, es), nk = reach(a.xs[1], B, H_k, T, d, es);
  const Range r[] = {{q, nq, false}, {k, nk, false}, {q_weight, d * ws, false}, {k_weight, d * ws, false},
                     {a.rot ? cos : nullptr, table, false}, {a.rot ? sin : nullptr, table, false},
                     {a.positions, static_cast<size_t>(B) * T * 4, false},
                     {dq_out, reach(a.ys[0], B, H_q, T, d, es), false}, {dk_out, reach(a.ys[1], B, H_k, T, d, es), false},
                     {dq, reach(a.dxs[0], B, H_q, T, d, es), true}, {dk, reach(a.dxs[1], B, H_k, T, d, es), true},
                     {dq_weight, d * ws, true}, {dk_weight, d * ws, true},
                     {sums ? workspace : nullptr, need, true}};
  if (!disjoint(r, 14, nullptr, nullptr)) return VLA_ERR_INVALID_ARG;
  a.dy[0] = dq_out; a.dy[1] = dk_out; a.dx[0] = dq; a.dx[1] = dk;
  a.dw[0] = dq_weight; a.dw[1] = dk_weight;
  a.dw_part = sums ? static_cast<float*>(workspace) : nullptr;
  if (T == 0 && !sums) return VLA_OK;
  return launched(vla::launch_qk_norm_rope_backward(a, d, io_dtype, op.interleaved != 0, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

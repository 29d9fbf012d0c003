/*
 * vla.h -- C ABI of the MI355X (gfx950) Variational Linear Attention forward library.
 *
 * The operation it is named for: the causal per-head VLA forward recurrence (paper Section 3.3,
 * eq. (sm), eq. (s-update), numerator of eq. (output); Algorithm 1).  For every
 * (batch b, head h) independently, starting from S = S0[b,h], A = A0[b,h], for
 * t = 1..T:
 *
 *     k^_t     = k_t / max(||k_t||, eps)                       (Section 3.1)
 *     u_t      = k^_t               (penalty direction aligned with the key, Section 7.1)
 *     z_t      = A_{t-1} u_t ;  delta_t = max(1 + u_t . z_t, eps)
 *     A_t      = A_{t-1} - z_t z_t^T / delta_t                 (eq. (sm))
 *     alpha^_t = A_t k^_t / max(||A_t k^_t||, eps)             (post-update A)
 *     e_t      = v_t - S_{t-1} k^_t
 *     S_t      = S_{t-1} + e_t alpha^_t^T                      (eq. (s-update))
 *     o_t      = S_t q_t                                       (post-update S)
 *
 * and finally S_T, A_T are written out.  The other lines of Algorithm 1 (a separate
 * penalty direction u, the periodic identity refresh, the denominator of eq. (output)
 * and the ELU+1 feature map) are off by default and switched on through vla_opts.
 *
 * Every pointer is a DEVICE pointer unless stated otherwise.  The library never
 * allocates, frees or retains memory: the caller owns every buffer for the
 * duration of the call's execution on `stream`.  Calls are asynchronous with
 * respect to the host (kernels are enqueued on `stream`, no host synchronisation)
 * and re-entrant.  All validation happens on the host before anything is enqueued: with
 * VLA_ERR_INVALID_ARG, VLA_ERR_UNSUPPORTED or VLA_ERR_WORKSPACE nothing has been launched and no
 * output has been touched.  VLA_ERR_HIP reports a launch the HIP runtime refused; in the modes
 * that run several kernels back to back, earlier kernels of the call may already be enqueued
 * then and the outputs and the workspace hold unspecified values.
 */
#ifndef VLA_H_
#define VLA_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of q, k, v and o.  The states S and A are always float32, and all
 * arithmetic is float32 regardless of the I/O type (bf16 inputs are widened
 * exactly; o is rounded to nearest-even on the final store). */
typedef enum { VLA_F32 = 0, VLA_BF16 = 1 } vla_dtype;

/* Which kernel family runs the recurrence.
 *   AUTO     : the library picks: CHUNKED when the identity refresh is switched on or the shape has no
 *              segment kernels; else TIME_PARALLEL for few heads (d = 128 and 96: B*H <= 64, 96 from
 *              T = 4096, 128 from T = 8192 (from 4096 at d = 96); d = 64: 192, 320 from T = 4096;
 *              d = 32: 512) and T >= 1024, or from T = 512 for B*H <= 32, 64, 256 heads at d = 128, 64,
 *              32 (d_k != d_v: by d_k, with 384 heads at d_k = 64 and 128 at d_k = 128 from T = 4096,
 *              1280 at d_k = 32 with d_v = 128), if the caller passed the workspace
 *              vla_forward_workspace_bytes() asks for (else CHUNKED); CHUNKED otherwise.
 *   SCAN     : one workgroup per (b,h) walks the tokens one by one with A and S
 *              resident in registers (FP32 vector ALU).
 *   CHUNKED  : tokens are processed in blocks; the block form of the same
 *              recurrence turns the matrix-vector work into dense FP32 matrix
 *              products (MFMA).  Same result up to float32 rounding order.  A second block kernel
 *              carries the options of Algorithm 1.
 *   TWO_PHASE: phase 1 runs the A recurrence and writes k^_t, alpha^_t to the
 *              workspace; phase 2 runs the S recurrence with the rows of S spread
 *              over several workgroups (for small B*H).  Allowed because A never
 *              reads S (eq. (sm)); Algorithm 2 takes k^, alpha^ as given inputs.
 *   TIME_PARALLEL: TWO_PHASE with the sequence cut into segments that run concurrently (for small
 *              B*H and long T).  Without the refresh, A at a segment boundary is the explicit
 *              inverse (A_0^{-1} + sum of u u^T up to there)^{-1} of Section 3.2 / eq. (penalty) (u = k^
 *              unless opts->u is given): one Gram matrix per segment, summed in float64 or, where no A_0
 *              is given and (tokens / lambda0) u_scale^2 is at most about 2e6, in fixed point with an error
 *              of about 1e-6 of A in the worst case, and inverted in float64; S at a boundary follows by
 *              composing the per-segment affine maps S -> S P + Q of eq. (s-update); the key sum of the
 *              normalised read-out at a boundary is a prefix sum.
 *              Inside a segment the recurrence is the same exact block form.  Same result up to float32
 *              rounding.
 */
typedef enum {
  VLA_MODE_AUTO = 0,
  VLA_MODE_SCAN = 1,
  VLA_MODE_CHUNKED = 2,
  VLA_MODE_TWO_PHASE = 3,
  VLA_MODE_TIME_PARALLEL = 4
} vla_mode;

typedef enum {
  VLA_OK = 0,
  VLA_ERR_INVALID_ARG = 1, /* null required pointer, non-positive size, misaligned pointer, bad enum */
  VLA_ERR_UNSUPPORTED = 2, /* valid request this build has no kernel for (head sizes, mode, option) */
  VLA_ERR_WORKSPACE = 3,   /* workspace missing or smaller than vla_forward_workspace_bytes() */
  VLA_ERR_HIP = 4          /* the HIP runtime reported an error at launch */
} vla_status;

/* Options; pass NULL for the defaults in brackets.  Always initialise the struct with
 * vla_default_opts() and then change fields: later library versions may append fields.
 *
 * The fields after `mode` switch on the remaining lines of Algorithm 1 (paper, pseudocode appendix).
 * SCAN and CHUNKED carry all of them; TWO_PHASE and TIME_PARALLEL carry all but the identity refresh
 * (asking for them with refresh_period > 0 returns VLA_ERR_UNSUPPORTED, and AUTO then selects CHUNKED): with
 * the refresh A_t is no longer the inverse of a prefix sum, which the segment boundaries rest on.
 * feature_map on its own changes no routing. */
typedef struct vla_opts {
  float lambda0; /* [0.1]  A_0 = I / lambda0, used only when A0 == NULL (Section 3.2) */
  float eps;     /* [1e-4] floor of every denominator: ||k||, delta, ||A k^||, ||u|| and the
                    read-out denominator (Section 5.4) */
  int mode;      /* [VLA_MODE_AUTO] a vla_mode */
  const void* u; /* [NULL] device, [B, H, T, d_k], io_dtype: raw penalty directions u~_t of
                    eq. (penalty); the recurrence uses u_t = u_scale * u~_t / max(||u~_t||, eps).
                    NULL: u_t = k^_t (Section 7.1) */
  float u_scale; /* [1.0]  1/sqrt(d_h) reproduces the scaling in Algorithm 1 */
  int refresh_period;   /* [0 = off] > 0: A += refresh_eta * I after the rank-1 update (and before the
                           write direction is formed) at every step whose 1-based index
                           step_offset + t is a multiple of refresh_period (Algorithm 1 uses 20) */
  float refresh_eta;    /* [1e-3] */
  int step_offset;      /* [0] tokens already processed by earlier calls of a split sequence; only
                           the refresh schedule depends on it */
  int normalise_output; /* [0] 1: o_t = S_t q_t / max(q_t . zkey_t, eps) with the running key sum
                           zkey_t = zkey_0 + sum_{s<=t} k_s of eq. (output); k_s is the key as used
                           (after feature_map, before L2 normalisation) */
  int feature_map;      /* [0] 1: q and k are replaced by ELU(x) + 1 elementwise on load (Section 3.3) */
  const float* zkey0;   /* [NULL = 0] device, [B, H, d_k] float32: key sum carried in from earlier calls */
  float* zkey_T;        /* [NULL = not wanted] device, [B, H, d_k] float32: key sum after the last token;
                           may alias zkey0 */
  int segments;         /* [0 = the library chooses] TIME_PARALLEL only: number of time segments (at most
                           256; capped at one per 16 tokens).  Sizes the workspace, so pass the same
                           value to vla_forward_workspace_bytes() and vla_forward() */
} vla_opts;

/* Fills *opts with the defaults above. */
void vla_default_opts(vla_opts* opts);

/* Bytes of device workspace vla_forward needs for these arguments (0 for the
 * modes that need none).  Returns 0 as well when the arguments are invalid --
 * vla_forward will then report the error.  Pass the options of the call itself: with `segments` left at 0
 * the number of segments, and so the size, also depends on whether u, normalise_output or the zkey
 * pointers are set (a workspace sized for other options may be refused with VLA_ERR_WORKSPACE). */
size_t vla_forward_workspace_bytes(int B, int H, int T, int d_k, int d_v, int io_dtype,
                                   const vla_opts* opts);

/*
 * vla_forward -- run the recurrence above for all B*H heads over T tokens.
 *
 *   q, k   [B, H, T, d_k]   io_dtype, contiguous, read-only
 *   v      [B, H, T, d_v]   io_dtype, contiguous, read-only
 *   S0     [B, H, d_v, d_k] float32 row-major, or NULL for S_0 = 0     (Algorithm 1)
 *   A0     [B, H, d_k, d_k] float32 row-major, or NULL for I / lambda0 (Algorithm 1).
 *          Must be symmetric positive definite (precondition, not checked).
 *          Values of all five are finite.  From an infinite or NaN one on, a head's results are NaN or infinite, without
 *          a rule for which; so they may be where a product or sum of the recurrence leaves float32 or comes within
 *          0.4 % of its largest value (3.39e38).  Other heads are not touched.
 *   o      [B, H, T, d_v]   io_dtype, written
 *   S_T    [B, H, d_v, d_k] float32, written; NULL if not wanted; may be S0 itself
 *   A_T    [B, H, d_k, d_k] float32, written; NULL if not wanted; may be A0 itself
 *          No written buffer (o, S_T, A_T, opts->zkey_T, the workspace) may overlap another buffer of
 *          the call, in whole or in part -- the byte ranges are compared on the host and an overlap
 *          returns VLA_ERR_INVALID_ARG -- with three exceptions: S_T == S0, A_T == A0 and
 *          zkey_T == zkey0 (the same pointer: the state is then updated in place).
 *   B, H   >= 1;  T >= 0 (T == 0 copies the initial state to S_T / A_T)
 *   d_k, d_v in {16, 32, 64, 96, 128}, any pair (S is d_v x d_k).  SCAN and CHUNKED for every pair and
 *          every option (with d_k != d_v the waves of a head share out the d_v / 16 row tiles of S);
 *          TWO_PHASE and TIME_PARALLEL for d_k >= 32 with any d_v (every option but the identity
 *          refresh); AUTO routes by d_k as above
 *   opts   host pointer or NULL
 *   workspace, workspace_bytes: device scratch of at least
 *          vla_forward_workspace_bytes(...) bytes (may be NULL/0 when that is 0)
 *   stream a hipStream_t passed as void*; NULL is the default stream
 *
 * All device pointers must be 16-byte aligned.  Returns a vla_status.
 * Running [0,T1) and then [T1,T) with the carried S_T, A_T gives the same result
 * as one call over [0,T) (the fixed-size state is the whole memory, Section 7.4).
 */
int vla_forward(const void* q, const void* k, const void* v, const float* S0, const float* A0,
                void* o, float* S_T, float* A_T, int B, int H, int T, int d_k, int d_v,
                int io_dtype, const vla_opts* opts, void* workspace, size_t workspace_bytes,
                void* stream);

/*
 * vla_forward_static -- vla_forward for callers that cannot allocate device memory or have none to pass as a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, same kernels and same results as vla_forward, without the workspace pair: the modes that need
 * a workspace (TWO_PHASE, TIME_PARALLEL, and AUTO where it resolves to them) use an array of
 * 64 MiB (67,108,864 bytes) that is part of the library's device image -- every GPU the library runs on holds
 * its own copy from the first use of the library on it until the process ends.  The call allocates and frees
 * nothing.
 *
 *   - A request whose vla_forward_workspace_bytes() exceeds 64 MiB returns VLA_ERR_WORKSPACE (with a
 *     message on stderr) when TWO_PHASE or TIME_PARALLEL was asked for by name; AUTO runs CHUNKED instead,
 *     as vla_forward does when it is given no workspace.
 *   - The device that owns the buffers and `stream` must be the current device.  The first call on a device
 *     looks the array's address up once (hipGetSymbolAddress; VLA_ERR_HIP if that fails): make that call
 *     before a stream capture begins.
 *   - All calls on one GPU share that GPU's array: two calls that need it and may overlap in time (different
 *     streams, or graphs replayed concurrently) race on it.  Calls on one stream are ordered and safe.
 *     Nothing in the array has to start at zero and nothing is kept in it between calls.
 */
int vla_forward_static(const void* q, const void* k, const void* v, const float* S0, const float* A0,
                       void* o, float* S_T, float* A_T, int B, int H, int T, int d_k, int d_v,
                       int io_dtype, const vla_opts* opts, void* stream);

/*
 * vla_decode_step -- one token of the same recurrence for every head, on a state that stays where it is
 * (generation: Section 7.4, the fixed-size state S, A is the whole memory).  Equivalent to vla_forward with
 * T = 1, S0 = S_T = S and A0 = A_T = A, but organised for the memory traffic that dominates a single step
 * (2 d^2 floats of state read and written per head against 10 d^2 flop).
 *
 *   q, k   [B, H, d_k]      io_dtype, contiguous, read-only
 *   v      [B, H, d_v]      io_dtype, contiguous, read-only
 *   S      [B, H, d_v, d_k] float32 row-major, updated in place (required)
 *   A      [B, H, d_k, d_k] float32 row-major, updated in place (required; symmetric positive definite)
 *   o      [B, H, d_v]      io_dtype, written; must not overlap any input
 *   d_k, d_v in {16, 32, 64, 96, 128}, any pair, with or without the optional lines of Algorithm 1
 *   opts   host pointer or NULL.  eps and the optional lines of Algorithm 1 are honoured as in vla_forward
 *          with T = 1: u [B, H, d_k] (io_dtype) with u_scale, the identity refresh (this call is step
 *          step_offset + 1 of the schedule), normalise_output with zkey0 / zkey_T [B, H, d_k] (may alias),
 *          feature_map.  lambda0, mode and segments are not used.
 *   stream a hipStream_t passed as void*; NULL is the default stream
 *
 * All device pointers must be 16-byte aligned.  Asynchronous, allocates nothing.  Returns a vla_status.
 */
int vla_decode_step(const void* q, const void* k, const void* v, float* S, float* A, void* o, int B,
                    int H, int d_k, int d_v, int io_dtype, const vla_opts* opts, void* stream);

/* Human-readable name of a vla_status (static storage, never NULL). */
const char* vla_status_string(int status);

/* Library version: major*10000 + minor*100 + patch. */
int vla_version(void);

/* Which concrete mode AUTO resolves to for these arguments when the workspace asked for by
 * vla_forward_workspace_bytes() is passed (a vla_mode, never AUTO), or -1 if the arguments are
 * invalid/unsupported.  Host-only, launches nothing. */
int vla_resolve_mode(int B, int H, int T, int d_k, int d_v, int io_dtype, const vla_opts* opts);

/*
 * ---- Operators around the recurrence -------------------------------------------------------------------------
 *
 * The gated delta rule (the sister recurrence: the same residual write on a state of the same layout, a decay and a write
 * strength in place of A) and the norm of queries and keys with the position rotation (what comes before either
 * recurrence).  The rules above hold for them: device pointers, nothing allocated or kept, asynchronous on `stream`, all
 * validation on the host before anything is launched, no written buffer overlapping another one of the call (by the range of addresses
 * that its strides span: slices of one buffer that alternate in memory are refused as outputs).
 */

/* Element strides of a [B, H, T, d] (gates: [B, H, T]) tensor.  All zero: contiguous.  The last dimension of d elements is always
 * contiguous; strides of q, k, v, o and of their gradients are multiples of 16 bytes (of the gates: any), none is negative,
 * and a written tensor's rows do not overlap.  A read tensor may repeat its rows over b and h (stride 0), a gate also over t, but not
 * by three zeros; for the gated delta rule its tokens are less than 2^31 / 32 bytes apart. */
typedef struct vla_strides {
  long long b, h, t;
} vla_strides;

/* Always initialise with vla_delta_default_opts() and then change fields: later versions may append fields. */
typedef struct vla_delta_opts {
  float scale;        /* [0 = 1 / sqrt(d_k)] factor of the read-out */
  const int* lengths; /* [NULL = T] device, [B]: tokens of each sequence (values outside 0..T count as the nearer end).  Later tokens
                         are not part of it: whatever they hold, even NaN, their o is 0, the states are those after the last
                         token of the sequence, and their gradients are 0 */
  vla_strides q, k, v, o, g, beta; /* [contiguous]; dO of the backward pass has the strides of o */
  vla_strides dq, dk, dv;          /* [contiguous] of the backward pass's outputs; dg and dbeta are contiguous */
  void* saved;        /* [NULL = not wanted] device, vla_delta_saved_bytes(): what vla_delta_forward keeps for vla_delta_backward
                         (the state at every 256th token, and d_v float32 numbers for every token and value head); written by the first, read by
                         the second */
  size_t saved_bytes;
  int segments;       /* [0 = the library chooses] time segments that vla_delta_forward and vla_delta_backward cut long sequences of few heads
                         into (1: none; each call by itself).  Sizes the workspace, so pass the same value to vla_delta_workspace_bytes() */
} vla_delta_opts;

void vla_delta_default_opts(vla_delta_opts* opts);

/* Bytes of device workspace that vla_delta_forward (backward: vla_delta_backward) wants for these arguments; 0 when it wants none and
 * when they are invalid.  A forward call with a smaller one, or none, runs every sequence from its start to its end (the same
 * results up to float32 rounding, slower for few heads); a backward call returns VLA_ERR_WORKSPACE. */
size_t vla_delta_workspace_bytes(int B, int H_k, int H_v, int T, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts, int backward);
/* Bytes of opts->saved. */
size_t vla_delta_saved_bytes(int B, int H_v, int T, int d_k, int d_v, int io_dtype);

/*
 * vla_delta_forward -- the gated delta rule.  For every batch row b and value head h, with the key head h / (H_v / H_k), from S = S0[b,h]:
 *
 *     S'_t = exp(g_t) S_{t-1};   S_t = S'_t + beta_t (v_t - S'_t k_t) k_t^T;   o_t = scale S_t q_t
 *
 *   q, k   [B, H_k, T, d_k]   io_dtype by strides; ||k_t|| <= 1 (vla_qk_norm_rope with l2) and 0 <= beta_t <= 2 keep the state bounded;
 *                             neither is checked
 *   v, o   [B, H_v, T, d_v]   io_dtype by strides; o written
 *   g      [B, H_v, T]        float32, the logarithm of the decay; -infinity forgets the state
 *   beta   [B, H_v, T]        float32
 *   S0     [B, H_v, d_v, d_k] float32 or NULL (zero);  S_T the same, written, or NULL; may be S0 itself
 *   H_v a multiple of H_k;  T >= 0 (T == 0 copies S0 to S_T);  d_k, d_v in {16, 32, 64, 96, 128}, any pair
 *
 * Sums, decays and the state are float32 whatever io_dtype; products of the state with q, k and the writes are formed from parts
 * that carry all of its bits (bf16: the read-out, which is rounded to bf16, from 16 of them).  q, k, v, o, S0 and S_T are
 * 16-byte aligned.  Running [0, T1) and then [T1, T) with the carried S_T gives the same result as one call up to rounding.
 * Tokens go through the matrix unit 16 at a time: an infinite or NaN value reaches, besides all that follows it, the outputs of up to
 * 15 tokens before it (never those of another head or sequence).
 */
int vla_delta_forward(const void* q, const void* k, const void* v, const float* g, const float* beta, const float* S0, void* o,
                      float* S_T, int B, int H_k, int H_v, int T, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts,
                      void* workspace, size_t workspace_bytes, void* stream);

/* One token on a state that stays where it is: vla_delta_forward with T = 1 and S0 = S_T = S (all strides are those of [B, H, 1, d]). */
int vla_delta_decode_step(const void* q, const void* k, const void* v, const float* g, const float* beta, float* S, void* o, int B,
                          int H_k, int H_v, int d_k, int d_v, int io_dtype, const vla_delta_opts* opts, void* stream);

/*
 * vla_delta_backward -- the gradients of vla_delta_forward's inputs, given those of o and S_T, its inputs and what it saved.
 *   dO      [B, H_v, T, d_v] io_dtype;  dS_T [B, H_v, d_v, d_k] float32 or NULL (zero)
 *   dq, dk  [B, H_k, T, d_k] io_dtype, summed over the value heads that share a key head, in a fixed order
 *   dv      [B, H_v, T, d_v] io_dtype;  dg, dbeta [B, H_v, T] float32;  dS0 [B, H_v, d_v, d_k] float32 or NULL (not wanted)
 * The same inputs and saved states give the same bits.  dq, dk and dv are rounded to io_dtype once (bf16: dk from 16 bits of each factor).  dg is the sum of the differences dO_i . O_i - v_i . dV_i over up to 256 tokens and of
 * <dS, S> behind them, and exact to float32's rounding of these terms: where strong decays make it far smaller than they are, what is
 * left of their rounding (1e-7 of them) shows.  A decay that is 0 in float32 (g < -104) ends the sums: its dg is 0, and nothing behind it
 * counts for the tokens before it.
 */
int vla_delta_backward(const void* q, const void* k, const void* v, const float* g, const float* beta, const void* dO, const float* dS_T,
                       void* dq, void* dk, void* dv, float* dg, float* dbeta, float* dS0, int B, int H_k, int H_v, int T, int d_k,
                       int d_v, int io_dtype, const vla_delta_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

typedef struct vla_norm_opts {
  float eps;            /* [1e-6] */
  int l2;               /* [0] 0: x / sqrt(mean x^2 + eps) (RMS); 1: x / sqrt(sum x^2 + eps) (unit length) */
  int interleaved;      /* [0] pairs of the rotation: 0: columns i and i + rot / 2; 1: columns 2i and 2i + 1 */
  int rot;              /* [0 = d, or none without tables] columns that are rotated, the first ones; a multiple of 8 */
  int places;           /* [0] rows of the tables */
  int offset;           /* [0] position of token 0 where positions is NULL */
  int weight_dtype;     /* [VLA_F32] of both weights */
  const int* positions; /* [NULL = offset + t] device, [B, T].  A position that the tables do not hold gives rows of NaN */
  vla_strides q, k;         /* [contiguous] */
  vla_strides q_out, k_out; /* [contiguous]; in the backward pass of dq_out, dk_out */
  vla_strides dq, dk;       /* [contiguous] */
} vla_norm_opts;

/* Fills *opts with the values in brackets. */
void vla_norm_default_opts(vla_norm_opts* opts);

/*
 * vla_qk_norm_rope -- every head's row x of q (k): y = Rot_p(w * x r), r = 1 / sqrt(n^-1 sum x^2 + eps), n = d (RMS) or 1 (l2).
 *   q, k          [B, H_q, T, d], [B, H_k, T, d] io_dtype by strides (views of a projection [B, T, H d] as they are); H_q or H_k
 *                 may be 0 with a NULL tensor
 *   weights       [d], opts->weight_dtype, or NULL (ones)
 *   cos, sin      [places, rot / 2] float32, or NULL without a rotation (opts->rot 0)
 *   q_out, k_out  as q, k; written, by default contiguous, which is what the recurrences take
 * Float32 arithmetic; one rounding, to io_dtype.  d in {16, 32, 64, 96, 128}; all pointers but positions 16-byte aligned.
 */
int vla_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos, const float* sin,
                     void* q_out, void* k_out, int B, int T, int H_q, int H_k, int d, int io_dtype, const vla_norm_opts* opts,
                     void* stream);
/* Its gradients: dq, dk, and those of the weights (opts->weight_dtype [d], summed over all rows in float32 in a fixed order; NULL: not
 * wanted).  The workspace is needed where one of the latter is wanted. */
size_t vla_qk_norm_rope_workspace_bytes(int d);
int vla_qk_norm_rope_backward(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos,
                              const float* sin, const void* dq_out, const void* dk_out, void* dq, void* dk, void* dq_weight,
                              void* dk_weight, int B, int T, int H_q, int H_k, int d, int io_dtype, const vla_norm_opts* opts,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * ---- Operators on rows of channels ---------------------------------------------------------------------------
 *
 * Tensors [B, T, n]: n channels of T tokens, the rows that a projection gives (the heads of the recurrences above side by side).  Their strides are
 * a vla_strides whose h is 0; the rules above hold for them (16-byte pieces, written rows apart, all zero: contiguous; read rows may repeat).  n is a multiple
 * of 8.  `lengths` as in vla_delta_opts: what lies past the end of a sequence may hold anything (NaN too) and has no effect; outputs and gradients there
 * are 0.
 */

typedef struct vla_conv_opts {
  int silu;            /* [1] 1: y = pre / (1 + exp(-pre)); 0: y = pre */
  int weight_dtype;    /* [VLA_F32] of weight and bias, and of their gradients */
  const int* lengths;  /* [NULL = T] device, [B] */
  vla_strides x, y;    /* [contiguous] of y and of dy */
  vla_strides dx;      /* [contiguous] */
} vla_conv_opts;
void vla_conv_default_opts(vla_conv_opts* opts);

/*
 * vla_causal_conv -- the short causal convolution of every channel: pre_t = bias + sum_j weight[.,j] x_{t-width+1+j}, j < width.
 *
 *   x, y     [B, T, n] io_dtype by strides
 *   weight   [n, width] weight_dtype, width 2, 3 or 4;  bias [n] or NULL (zero)
 *   state    [B, width-1, n] io_dtype: the rows before token 0, oldest first, or NULL (zero)
 *   state_T  the same, written: the rows before the token that comes next; or NULL; may be state itself
 *
 * Float32 sums, one rounding.  Running [0, T1) and then [T1, T) with the carried state gives the same bits as one call.
 */
int vla_causal_conv(const void* x, const void* weight, const void* bias, const void* state, void* y, void* state_T, int B, int T, int n,
                    int width, int io_dtype, const vla_conv_opts* opts, void* stream);
/* One token, x and y [B, n] (strides: b alone); the state moves on in place.  No lengths. */
int vla_causal_conv_step(const void* x, const void* weight, const void* bias, void* state, void* y, int B, int n, int width, int io_dtype,
                         const vla_conv_opts* opts, void* stream);
/* Its gradients, given those of y and state_T (NULL: zero).  dweight, dbias, dstate: NULL if not wanted; the first two are summed in
 * float32 in a fixed order and need the workspace. */
size_t vla_causal_conv_workspace_bytes(int B, int T, int n, int width, int io_dtype);
int vla_causal_conv_backward(const void* x, const void* weight, const void* bias, const void* state, const void* dy, const void* dstate_T,
                             void* dx, void* dweight, void* dbias, void* dstate, int B, int T, int n, int width, int io_dtype,
                             const vla_conv_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

typedef struct vla_scan_opts {
  int softplus;               /* [1] 1: dt = log(1 + exp(delta + delta_bias)); 0: dt = delta + delta_bias */
  int groups;                 /* [1] of channels that share B and C: n / groups neighbouring ones, a multiple of 8 */
  const int* lengths;         /* [NULL = T] device, [B] */
  vla_strides u, delta, z, y; /* [contiguous] of y and of dy */
  vla_strides B, C;           /* [contiguous [B, T, groups, N]]; h: from group to group */
  vla_strides du, ddelta, dz; /* [contiguous]; the gradients of B and C are contiguous [B, T, groups, N] */
  void* saved;                /* [NULL = not wanted] device, vla_selective_scan_saved_bytes(): the state at every 8th token (N / 2 bytes for every
                                 token and channel), written by vla_selective_scan, read by vla_selective_scan_backward */
  size_t saved_bytes;
  int segments;               /* [0 = the library chooses] time segments that long sequences of few channels are cut into (1: none).  Sizes the
                                 workspace, so pass the same value to vla_selective_scan_workspace_bytes() */
} vla_scan_opts;
void vla_scan_default_opts(vla_scan_opts* opts);

/* Bytes of workspace of vla_selective_scan (backward: of vla_selective_scan_backward); 0 when it wants none and when the arguments are
 * invalid.  A forward call with a smaller one, or none, runs every sequence from its start to its end; a backward call returns
 * VLA_ERR_WORKSPACE. */
size_t vla_selective_scan_workspace_bytes(int B, int T, int n, int N, int io_dtype, const vla_scan_opts* opts, int backward);
/* Bytes of opts->saved. */
size_t vla_selective_scan_saved_bytes(int B, int T, int n, int N, int io_dtype, const vla_scan_opts* opts);

/*
 * vla_selective_scan -- the selective state space scan.  For every batch row, channel c with its group, and state s, from h = h0:
 *
 *     h_t[c,s] = exp(dt_t[c] A[c,s]) h_{t-1}[c,s] + dt_t[c] u_t[c] Bm_t[s];   y_t[c] = (sum_s Cm_t[s] h_t[c,s] + D[c] u_t[c]) z_t[c] sigmoid(z_t[c])
 *
 *   u, delta, z, y  [B, T, n]         io_dtype by strides; z NULL: no gate
 *   Bm, Cm          [B, T, groups, N] io_dtype by strides
 *   A               [n, N]            float32 (finite; negative for a state that decays);  D, delta_bias [n] float32 or NULL (zero)
 *   h0, h_T         [B, n, N]         float32; h0 NULL: zero; h_T written, or NULL; may be h0 itself
 *   N in {8, 16, 32, 64};  T >= 0 (T == 0 copies h0 to h_T)
 *
 * Float32 arithmetic and states; one rounding, to io_dtype.  Running [0, T1) and then [T1, T) with the carried h_T gives the same
 * result as one call up to rounding.
 */
int vla_selective_scan(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                       const float* delta_bias, const float* h0, void* y, float* h_T, int B, int T, int n, int N, int io_dtype,
                       const vla_scan_opts* opts, void* workspace, size_t workspace_bytes, void* stream);
/* One token, u, delta, z, y [B, n], Bm, Cm [B, groups, N]; h [B, n, N] is updated in place.  No lengths. */
int vla_selective_scan_step(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                            const float* delta_bias, float* h, void* y, int B, int n, int N, int io_dtype, const vla_scan_opts* opts,
                            void* stream);
/*
 * vla_selective_scan_backward -- the gradients of its inputs, given those of y and h_T (NULL: zero) and what it saved.  du, ddelta, dz
 * (NULL without z), dBm, dCm: io_dtype, each rounded once; dA, dD, ddelta_bias, dh0: float32, the last three NULL if not wanted.  The sums over
 * tokens, channels and sequences are float32 in a fixed order: the same inputs give the same bits.
 */
int vla_selective_scan_backward(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm, const float* D, const void* z,
                                const float* delta_bias, const void* dy, const float* dh_T, void* du, void* ddelta, float* dA, void* dBm,
                                void* dCm, float* dD, void* dz, float* ddelta_bias, float* dh0, int B, int T, int n, int N, int io_dtype,
                                const vla_scan_opts* opts, void* workspace, size_t workspace_bytes, void* stream);

typedef struct vla_residual_opts {
  float eps;              /* [1e-6] of both norms */
  int group;              /* [0 = n] columns of a group of the norm of y (a head), a multiple of 8 that divides n */
  int activation;         /* [0] of the gate: 0: g / (1 + exp(-g)); 1: 1 / (1 + exp(-g)) */
  int stream_dtype;       /* [VLA_F32] of x, s and their gradients: VLA_F32 or io_dtype */
  int weight_dtype;       /* [VLA_F32] of post_weight, scale, weight and their gradients */
  vla_strides x, y, gate; /* [contiguous] */
  vla_strides s, h;       /* [contiguous] of the outputs and of their gradients */
  vla_strides dx, dy, dgate;
} vla_residual_opts;
void vla_residual_default_opts(vla_residual_opts* opts);

/*
 * vla_residual_norm -- what stands between a block and the next one:
 *
 *     s = x + scale * act(gate) * post_weight * N(y);   h = weight * N(s);   N(v) = v / sqrt(mean v^2 + eps)
 *
 * with the mean over a group of columns of y, and over the row of s.
 *
 *   x                   [B, T, n] stream_dtype: the residual stream, or NULL (zero)
 *   y                   [B, T, n] io_dtype: the block's output, or NULL: h = weight * N(x) alone (then s, gate, post_weight and scale are NULL)
 *   gate                [B, T, n] io_dtype or NULL (no gate);  scale [n] or NULL (ones);  post_weight [n] or NULL: y without a norm
 *   s                   [B, T, n] stream_dtype, written; may be x itself (the same strides)
 *   weight, h           [n], [B, T, n] io_dtype, written; both NULL: no second norm
 *
 * Float32 arithmetic; h comes from s before its rounding.  n <= 8192.
 */
int vla_residual_norm(const void* x, const void* y, const void* gate, const void* post_weight, const void* scale, const void* weight, void* s,
                      void* h, int B, int T, int n, int io_dtype, const vla_residual_opts* opts, void* stream);
/* Its gradients, given those of s (of x, where y is NULL) and h (NULL: zero); each NULL if not wanted.  Those of the weights are summed over the rows
 * in float32 in a fixed order and need the workspace. */
size_t vla_residual_norm_workspace_bytes(int n);
int vla_residual_norm_backward(const void* x, const void* y, const void* gate, const void* post_weight, const void* scale, const void* weight,
                               const void* ds, const void* dh, void* dx, void* dy, void* dgate, void* dpost_weight, void* dscale, void* dweight,
                               int B, int T, int n, int io_dtype, const vla_residual_opts* opts, void* workspace, size_t workspace_bytes,
                               void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_H_ */

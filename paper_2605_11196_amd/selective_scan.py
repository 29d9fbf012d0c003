"""The selective state space scan on torch tensors (vla_selective_scan, its step and its backward pass of include/vla.h)."""
import ctypes
import functools

from . import binding
from .binding import VlaError, VlaScanOpts
from .rows import (_all_aligned, _check_lengths, _check_rows, _check_vector, _fits, _io, _kind, _laid_groups, _laid_rows, _like, _no_tangents, _p,
                   _plan, _plans, _record, _together, _wants_gradients)


def _grouped(x, dims):
    """B or C with its dimension of groups."""
    return x.unsqueeze(-2) if x.dim() == dims else x


def _check(torch, u, delta, A, B, C, D, z, delta_bias, state, state_name, lengths, tokens):
    """Shapes of a call over tokens (tokens 1) or of one token (0); B and C with their groups; state: the given state or gradient of it."""
    dev, shape, dtype = u.device, u.shape, u.dtype
    _fits("sizes", *shape, *A.shape, *B.shape)
    if not u.is_cuda:
        raise ValueError("u must be a GPU tensor (no CPU path exists)")
    if len(shape) != 2 + tokens:
        raise ValueError(f"expected u as {'[B,T,n]' if tokens else '[B,n]'}")
    n = shape[-1]
    _check_rows(torch, "delta", delta, shape, dtype, dev)
    _check_rows(torch, "z", z, shape, dtype, dev)
    if A.dim() != 2:
        raise ValueError("expected A as [n,N]")
    _check_vector(torch, "A", A, (n, A.shape[1]), dev, (torch.float32,))
    _check_vector(torch, "D", D, (n,), dev, (torch.float32,))
    _check_vector(torch, "delta_bias", delta_bias, (n,), dev, (torch.float32,))
    G = B.shape[-2] if B.dim() == 3 + tokens else 0
    if G < 1 or n % G:
        raise ValueError(f"expected B and C as {'[B,T,N] or [B,T,G,N]' if tokens else '[B,N] or [B,G,N]'} with G a divisor of the {n} channels")
    for name, x in (("B", B), ("C", C)):
        _check_rows(torch, name, x, (*shape[:-1], G, A.shape[1]), dtype, dev)
    if state is not None and (state.dtype != torch.float32 or tuple(state.shape) != (shape[0], n, A.shape[1]) or not state.is_contiguous()
                              or state.device != dev):
        raise ValueError(f"{state_name} must be a contiguous float32 tensor of shape {(shape[0], n, A.shape[1])} on {dev}")
    _check_lengths(torch, lengths, shape[0], dev)


def _key(u, delta, A, B, C, D, z, delta_bias, state, lengths, softplus, segments=0):
    return ("scan", u.shape, u.stride(), u.dtype, u.device, delta.shape, delta.stride(), delta.dtype, delta.device, A.shape, A.stride(), A.dtype,
            A.device, B.shape, B.stride(), B.dtype, B.device, C.shape, C.stride(), C.dtype, C.device, _kind(D), _kind(z), _kind(delta_bias), _kind(state),
            _kind(lengths), bool(softplus), segments)


def _inputs(key, u, delta, A, B, C, D, z, delta_bias, lengths, softplus, segments=0):
    """The inputs as the kernels take them, kept until the call, and its options."""
    given = u, delta, A, B, C, D, z, delta_bias, lengths
    plan = _plans.get(key)
    if plan is not None and _all_aligned(u, delta, A, B, C, D, z, delta_bias):
        op = VlaScanOpts.from_buffer_copy(plan)
        if lengths is not None:
            op.lengths = lengths.data_ptr()
        return given, op
    _fits("segments", segments)
    op = VlaScanOpts(1 if softplus else 0, B.shape[-2])
    op.segments = segments
    (u, op.u), (delta, op.delta) = _laid_rows(u), _laid_rows(delta)
    if z is not None:
        z, op.z = _laid_rows(z)
    (B, op.B), (C, op.C) = _laid_groups(B), _laid_groups(C)
    A, D, delta_bias = _together(A), None if D is None else _together(D), None if delta_bias is None else _together(delta_bias)
    lengths = None if lengths is None else lengths.contiguous()
    kept = u, delta, A, B, C, D, z, delta_bias, lengths
    if plan is None:
        _plan(key, given, kept, op)
    if lengths is not None:
        op.lengths = lengths.data_ptr()
    return kept, op


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(B, T, n, N, io, groups, segments, backward):
    """vla_selective_scan_workspace_bytes, which depends on nothing else."""
    op = VlaScanOpts(1, groups)
    op.segments = segments
    return binding.load_library().vla_selective_scan_workspace_bytes(B, T, n, N, io, ctypes.byref(op), backward)


def _aligned(h):
    """A contiguous state (or None) at a 16-byte boundary."""
    return h.clone() if h is not None and h.data_ptr() & 15 else h


def _forward(torch, kept, op, h0, save, handle, outside):
    """kept, op: of _inputs(), the inputs checked; handle, outside: of binding._on_stream(), in whose context this runs.
    (y, h_T, what the backward pass needs or None)."""
    u, delta, A, Bm, Cm, D, z, delta_bias, _ = kept
    B, T, n = u.shape
    N, dev, io = A.shape[1], u.device, _io(torch, u)
    lib = binding.load_library()
    h0 = _aligned(h0)
    y = _like(torch, u)
    h_T = torch.empty((B, n, N), dtype=torch.float32, device=dev)
    saved = None
    if save:
        op.saved_bytes = lib.vla_selective_scan_saved_bytes(B, T, n, N, io, ctypes.byref(op))
        saved = torch.empty((max(op.saved_bytes, 16),), dtype=torch.uint8, device=dev)
        op.saved = saved.data_ptr()
    need = _workspace_bytes(B, T, n, N, io, op.groups, op.segments, 0)
    ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
    _record(outside, y, h_T, saved)
    rc = lib.vla_selective_scan(u.data_ptr(), delta.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _p(D), _p(z), _p(delta_bias), _p(h0),
                                y.data_ptr(), h_T.data_ptr(), B, T, n, N, io, ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_selective_scan")
    return y, h_T, saved


def selective_scan_forward(u, delta, A, B, C, D=None, z=None, h0=None, *, delta_bias=None, softplus=True, lengths=None, save_for_backward=False,
                           segments=0, stream=None):
    """h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t;  y_t = (C_t . h_t + D u_t) z_t sigmoid(z_t);  dt = softplus(delta + delta_bias)  for every channel.

    u, delta and the gate z (or None) [B,T,n] on the GPU (float32 or bfloat16, n a multiple of 8; views with a contiguous last dimension
    are read as they are), B, C [B,T,N] or, for G groups of neighbouring channels, [B,T,G,N], of u's type; A [n,N] with N 8, 16, 32 or
    64, D and delta_bias [n] (or None) and h0 [B,n,N] (or None: zero) float32.  softplus False: dt = delta + delta_bias.  lengths: int32
    [B], tokens of each sequence; y is zero beyond.  Returns (y, h_T), and with save_for_backward also what
    selective_scan_backward needs (N / 2 bytes for every token and channel).  Workspace, outputs and work are on `stream` (default: torch's current one).
    """
    import torch

    B, C = _grouped(B, u.dim()), _grouped(C, u.dim())
    key = _key(u, delta, A, B, C, D, z, delta_bias, h0, lengths, softplus, segments)
    if key not in _plans:
        _check(torch, u, delta, A, B, C, D, z, delta_bias, h0, "h0", lengths, 1)
    handle, context, outside = binding._on_stream(torch, u.device, stream)
    with context:
        kept, op = _inputs(key, u, delta, A, B, C, D, z, delta_bias, lengths, softplus, segments)
        y, h_T, saved = _forward(torch, kept, op, h0, save_for_backward, handle, outside)
    return (y, h_T, saved) if save_for_backward else (y, h_T)


def selective_scan_step(u, delta, A, B, C, h, D=None, z=None, *, delta_bias=None, softplus=True, stream=None):
    """One token: u, delta, z [B,n], B, C [B,N] or [B,G,N]; h [B,n,N] float32, contiguous and 16-byte aligned, is updated in place.  Returns
    y [B,n].  Without a gradient: for generation, under torch.no_grad() where an input asks for one."""
    import torch

    _no_tangents(torch, u, delta, A, B, C, h, D, z, delta_bias)
    if _wants_gradients(torch, u, delta, A, B, C, h, D, z, delta_bias):
        raise ValueError("selective_scan_step has no gradient: call it under torch.no_grad(), or selective_scan with one token")
    B, C = _grouped(B, u.dim()), _grouped(C, u.dim())
    key = _key(u, delta, A, B, C, D, z, delta_bias, h, None, softplus)
    if key not in _plans:
        _check(torch, u, delta, A, B, C, D, z, delta_bias, h, "h", None, 0)
    if h.data_ptr() & 15:
        raise ValueError("h must be 16-byte aligned: it is updated in place")
    handle, context, outside = binding._on_stream(torch, u.device, stream)
    with context:
        kept, op = _inputs(key, u, delta, A, B, C, D, z, delta_bias, None, softplus)
        u, delta, A, B, C, D, z, delta_bias, _ = kept
        batch, n = u.shape
        y = _like(torch, u)
        _record(outside, y)
        rc = binding.load_library().vla_selective_scan_step(u.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(), _p(D), _p(z),
                                                            _p(delta_bias), h.data_ptr(), y.data_ptr(), batch, n, A.shape[1], _io(torch, u),
                                                            ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_selective_scan_step")
    if not h.is_inference():
        torch.autograd.graph.increment_version(h)     # a graph that saved h must not use what it holds now
    return y


def _gradients(torch, u, delta, A, Bm, Cm, D, z, delta_bias, saved, dy, dh_T, lengths, softplus, segments, wanted, stream):
    """selective_scan_backward on these tensors, B and C with their groups; wanted: whether the gradients of D, delta_bias and h0 are."""
    key = _key(u, delta, A, Bm, Cm, D, z, delta_bias, dh_T, lengths, softplus, segments)
    if key not in _plans:
        _check(torch, u, delta, A, Bm, Cm, D, z, delta_bias, dh_T, "dh_T", lengths, 1)
    _check_rows(torch, "dy", dy, u.shape, u.dtype, u.device)
    if saved.dtype != torch.uint8 or saved.dim() != 1 or not saved.is_contiguous() or saved.device != u.device:
        raise ValueError(f"saved must be what selective_scan_forward returned: a contiguous uint8 tensor on {u.device}")
    handle, context, outside = binding._on_stream(torch, u.device, stream)
    with context:
        kept, op = _inputs(key, u, delta, A, Bm, Cm, D, z, delta_bias, lengths, softplus, segments)
        u, delta, A, Bm, Cm, D, z, delta_bias, _ = kept
        B, T, n = u.shape
        G, N, dev, io = Bm.shape[2], A.shape[1], u.device, _io(torch, u)
        lib = binding.load_library()
        (dy, op.y), dh_T, saved = _laid_rows(dy), _aligned(dh_T), _together(saved)
        op.saved, op.saved_bytes = saved.data_ptr(), saved.numel()
        du, ddelta = _like(torch, u), _like(torch, u)
        dz = _like(torch, u) if z is not None else None
        dB, dC = _like(torch, Bm), _like(torch, Cm)
        dA = _like(torch, A)
        dD = _like(torch, D) if wanted[0] and D is not None else None
        dbias = _like(torch, delta_bias) if wanted[1] and delta_bias is not None else None
        dh0 = torch.empty((B, n, N), dtype=torch.float32, device=dev) if wanted[2] else None
        need = _workspace_bytes(B, T, n, N, io, G, segments, 1)
        ws = torch.empty((max(need, 16),), dtype=torch.uint8, device=dev)
        _record(outside, du, ddelta, dz, dB, dC, dA, dD, dbias, dh0)
        rc = lib.vla_selective_scan_backward(u.data_ptr(), delta.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _p(D), _p(z), _p(delta_bias),
                                             dy.data_ptr(), _p(dh_T), du.data_ptr(), ddelta.data_ptr(), dA.data_ptr(), dB.data_ptr(), dC.data_ptr(),
                                             _p(dD), _p(dz), _p(dbias), _p(dh0), B, T, n, N, io, ctypes.byref(op), ws.data_ptr(), ws.numel(), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_selective_scan_backward")
    return du, ddelta, dA, dB, dC, dD, dz, dbias, dh0


def selective_scan_backward(u, delta, A, B, C, D, z, saved, dy, dh_T=None, *, delta_bias=None, softplus=True, lengths=None, segments=0, stream=None):
    """The gradients (du, ddelta, dA, dB, dC, dD, dz, ddelta_bias, dh0) of selective_scan_forward's inputs (None where there is no D, z or
    delta_bias), given those of y and h_T (None: zero), the same inputs and what it saved."""
    import torch

    shape = B.shape, C.shape
    B, C = _grouped(B, u.dim()), _grouped(C, u.dim())
    grads = list(_gradients(torch, u, delta, A, B, C, D, z, delta_bias, saved, dy, dh_T, lengths, softplus, segments, (True, True, True), stream))
    grads[3], grads[4] = grads[3].view(shape[0]), grads[4].view(shape[1])
    return tuple(grads)


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class SelectiveScan(torch.autograd.Function):
            @staticmethod
            def forward(ctx, u, delta, A, B, C, D, z, delta_bias, h0, lengths, key, softplus):
                handle, context, outside = binding._on_stream(torch, u.device, None)
                with context:
                    kept, op = _inputs(key, u, delta, A, B, C, D, z, delta_bias, lengths, softplus)
                    y, h_T, saved = _forward(torch, kept, op, h0, True, handle, outside)
                ctx.save_for_backward(*kept, saved)      # the inputs as the kernels read them
                ctx.softplus = softplus
                ctx.set_materialize_grads(False)
                return y, h_T

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dy, dh_T):
                # hooks (offload, checkpoints) may give other tensors than the saved ones: addresses and strides are those of these
                u, delta, A, B, C, D, z, delta_bias, lengths, saved = ctx.saved_tensors
                dy = torch.zeros_like(u) if dy is None else dy
                dh_T = None if dh_T is None else dh_T.contiguous()
                need = ctx.needs_input_grad
                grads = _gradients(torch, u, delta, A, B, C, D, z, delta_bias, saved, dy, dh_T, lengths, ctx.softplus, 0, (need[5], need[7], need[8]),
                                   None)
                return (*grads, None, None, None)

        _function = SelectiveScan
    return _function


def selective_scan(u, delta, A, B, C, D=None, z=None, h0=None, *, delta_bias=None, softplus=True, lengths=None, stream=None):
    """selective_scan_forward as a differentiable function: (y, h_T), with gradients for u, delta, A, B, C, D, z, delta_bias and h0 (once,
    in reverse mode, on the current stream).  Until then the states at every 8th token are kept: N / 2 bytes for every token and channel."""
    import torch

    _no_tangents(torch, u, delta, A, B, C, D, z, h0, delta_bias)
    if not _wants_gradients(torch, u, delta, A, B, C, D, z, h0, delta_bias):
        return selective_scan_forward(u, delta, A, B, C, D, z, h0, delta_bias=delta_bias, softplus=softplus, lengths=lengths, stream=stream)
    if stream is not None:
        raise ValueError("with gradients the work goes to the current stream: leave stream at None")
    B, C = _grouped(B, u.dim()), _grouped(C, u.dim())
    key = _key(u, delta, A, B, C, D, z, delta_bias, h0, lengths, softplus)
    if key not in _plans:
        _check(torch, u, delta, A, B, C, D, z, delta_bias, h0, "h0", lengths, 1)
    return _autograd().apply(u, delta, A, B, C, D, z, delta_bias, h0, lengths, key, softplus)

"""The gated delta rule on torch tensors (vla_delta_forward, vla_delta_decode_step and vla_delta_backward of include/vla.h)."""
import ctypes
import functools

from . import binding
from .binding import VlaDeltaOpts, VlaError, VlaStrides
from .qk_norm import _fits, _io, _keep_plan, _kind, _laid_out, _like, _no_tangents, _p, _steps, _strides, _together


def _gate(x):
    """A gate [B,H,T] and its strides: any that do not repeat one value over everything."""
    if x.is_contiguous():
        return x, None
    s = _steps(x)
    return (x, VlaStrides(*s)) if any(s) else (x.contiguous(), None)


def _check(torch, q, k, v, g, beta, state, state_name, lengths, tokens):
    """Shapes of a call over tokens (tokens 1) or of one token (0); state: the given state or gradient of it, or None."""
    dev, dtype, shape, v_shape = q.device, q.dtype, q.shape, v.shape
    _fits("sizes", *shape, *v_shape)
    if not (q.is_cuda and k.is_cuda and v.is_cuda):
        raise ValueError("q, k, v must be GPU tensors (no CPU path exists)")
    if k.dtype != dtype or v.dtype != dtype or k.device != dev or v.device != dev:
        raise ValueError("q, k, v must share a dtype and a device")
    if len(shape) != 3 + tokens or k.shape != shape or len(v_shape) != len(shape) or v_shape[0] != shape[0] or v_shape[2:-1] != shape[2:-1]:
        raise ValueError(f"expected q, k and v as {'[B,H,T,d]' if tokens else '[B,H,d]'} with one batch and length, q and k of one shape")
    H_k, H_v = shape[1], v_shape[1]
    if H_k < 1 or H_v % H_k:
        raise ValueError(f"the value heads ({H_v}) must be a multiple of the key heads ({H_k})")
    gate = v_shape[:-1]
    if g.dtype != torch.float32 or beta.dtype != torch.float32 or g.shape != gate or beta.shape != gate or g.device != dev or beta.device != dev:
        raise ValueError(f"g and beta must be float32 tensors of shape {tuple(gate)} on {dev}")
    if state is not None and (state.dtype != torch.float32 or state.shape != (shape[0], H_v, v_shape[-1], shape[-1]) or not state.is_contiguous()
                              or state.device != dev):
        raise ValueError(f"{state_name} must be a contiguous float32 tensor of shape {(shape[0], H_v, v_shape[-1], shape[-1])} on {dev}")
    if lengths is not None and (lengths.dtype != torch.int32 or lengths.shape != shape[:1] or lengths.device != dev):
        raise ValueError(f"lengths must be an int32 tensor of shape {tuple(shape[:1])} on {dev}")


def _aligned(S):
    """A contiguous state (or None) at a 16-byte boundary."""
    return S.clone() if S is not None and S.data_ptr() & 15 else S


def _scale(scale):
    """The option's value, where 0 stands for the default."""
    if scale is None:
        return 0.0
    if scale == 0:
        raise ValueError("scale must not be 0 (None: 1 / sqrt(d_k))")
    return scale


# Options of calls whose tensors go to the kernels as they are, by the shapes, layouts and types of these: a call like an earlier one is
# neither checked nor laid out again (4 of 16 us).
_plans = {}


def _key(q, k, v, g, beta, S0, lengths, scale, segments=0):
    return (q.shape, q.stride(), q.dtype, q.device, k.shape, k.stride(), k.dtype, k.device, v.shape, v.stride(), v.dtype, v.device, g.shape,
            g.stride(), g.dtype, g.device, beta.shape, beta.stride(), beta.dtype, beta.device, _kind(S0), _kind(lengths), scale, segments)


def _inputs(key, q, k, v, g, beta, scale, lengths, segments=0):
    """The inputs as the kernels take them, kept until the call, and its options."""
    given = q, k, v, g, beta, lengths
    plan = _plans.get(key)
    if plan is not None and not (q.data_ptr() | k.data_ptr() | v.data_ptr()) & 15:
        op = VlaDeltaOpts.from_buffer_copy(plan)
        if lengths is not None:
            op.lengths = lengths.data_ptr()
        return given, op
    op = VlaDeltaOpts(_scale(scale))
    _fits("segments", segments)
    op.segments = segments
    (q, op.q), (k, op.k), (v, op.v) = _laid_out(q), _laid_out(k), _laid_out(v)
    (g, g_strides), (beta, beta_strides) = _gate(g), _gate(beta)
    if g_strides is not None:
        op.g = g_strides
    if beta_strides is not None:
        op.beta = beta_strides
    if lengths is not None:
        lengths = lengths.contiguous()
    kept = q, k, v, g, beta, lengths
    if plan is None:
        _keep_plan(_plans, key, kept, given, op)
    if lengths is not None:
        op.lengths = lengths.data_ptr()
    return kept, op


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(B, H_k, H_v, T, dk, dv, io, segments, backward):
    """vla_delta_workspace_bytes, which depends on nothing else."""
    op = VlaDeltaOpts()
    op.segments = segments
    return binding.load_library().vla_delta_workspace_bytes(B, H_k, H_v, T, dk, dv, io, ctypes.byref(op), backward)


def _forward(torch, kept, op, S0, save, handle, outside):
    """kept, op: of _inputs(), the inputs checked; handle, outside: of binding._on_stream(), in whose context this runs.
    (o, S_T, what the backward pass needs or None)."""
    q, k, v, g, beta, _ = kept
    B, H_k, T, dk = q.shape
    H_v, dv, dev, io = v.shape[1], v.shape[3], q.device, _io(torch, q)
    lib = binding.load_library()
    S0 = _aligned(S0)
    o = _like(torch, v)
    if not o.is_contiguous():
        op.o = _strides(o)
    S_T = torch.empty((B, H_v, dv, dk), dtype=torch.float32, device=dev)
    saved = None
    if save:
        op.saved_bytes = lib.vla_delta_saved_bytes(B, H_v, T, dk, dv, io)
        saved = torch.empty((max(op.saved_bytes, 16),), dtype=torch.uint8, device=dev)
        op.saved = saved.data_ptr()
    need = _workspace_bytes(B, H_k, H_v, T, dk, dv, io, op.segments, 0)
    ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
    if outside is not None:
        for t in (o, S_T, saved):
            if t is not None:
                t.record_stream(outside)
    rc = lib.vla_delta_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _p(S0), o.data_ptr(), S_T.data_ptr(), B, H_k,
                               H_v, T, dk, dv, io, ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_delta_forward")
    return o, S_T, saved


def gated_delta_forward(q, k, v, g, beta, S0=None, *, scale=None, lengths=None, save_for_backward=False, segments=0, stream=None):
    """S' = exp(g_t) S;  S <- S' + beta_t (v_t - S' k_t) k_t^T;  o_t = scale S q_t  for every value head.

    q, k [B,H_k,T,d_k], v [B,H_v,T,d_v] on the GPU (float32 or bfloat16; views with a contiguous last dimension are read as they are),
    g (logarithm of the decay) and beta [B,H_v,T] float32, S0 [B,H_v,d_v,d_k] float32 or None (zero).  Value head h reads key head
    h // (H_v // H_k).  scale: default 1 / sqrt(d_k).  lengths: int32 [B], tokens of each sequence; o is zero beyond.
    Returns (o, S_T), o with v's order of dimensions, and with save_for_backward also what gated_delta_backward needs.
    Workspace, outputs and work are on `stream` (default: torch's current one).
    """
    import torch

    scale = None if scale is None else float(scale)
    key = _key(q, k, v, g, beta, S0, lengths, scale, segments)
    if key not in _plans:
        _check(torch, q, k, v, g, beta, S0, "S0", lengths, 1)
    binding.load_library()
    handle, context, outside = binding._on_stream(torch, q.device, stream)
    with context:
        kept, op = _inputs(key, q, k, v, g, beta, scale, lengths, segments)
        o, S_T, saved = _forward(torch, kept, op, S0, save_for_backward, handle, outside)
    return (o, S_T, saved) if save_for_backward else (o, S_T)


def gated_delta_decode_step(q, k, v, g, beta, S, *, scale=None, stream=None):
    """One token for every head: q, k [B,H_k,d_k], v [B,H_v,d_v], g, beta [B,H_v] float32; S [B,H_v,d_v,d_k] float32, contiguous and
    16-byte aligned, is updated in place.  Returns o [B,H_v,d_v].  Without a gradient: for generation, under torch.no_grad() where an
    input asks for one."""
    import torch

    _no_tangents(torch, q, k, v, g, beta, S)
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or g.requires_grad or beta.requires_grad
                                    or S.requires_grad):
        raise ValueError("gated_delta_decode_step has no gradient: call it under torch.no_grad(), or gated_delta with one token")
    scale = None if scale is None else float(scale)
    key = _key(q, k, v, g, beta, S, None, scale)
    plan = _plans.get(key)
    if plan is None:
        _check(torch, q, k, v, g, beta, S, "S", None, 0)
    handle, context, outside = binding._on_stream(torch, q.device, stream)
    with context:
        if plan is None or (q.data_ptr() | k.data_ptr() | v.data_ptr()) & 15:
            given = q, k, v, g, beta
            q, k, v, g, beta = kept = _together(q), _together(k), _together(v), g.contiguous(), beta.contiguous()
            op = VlaDeltaOpts(_scale(scale))
            if plan is None:
                _keep_plan(_plans, key, kept, given, op)
        else:
            op = VlaDeltaOpts.from_buffer_copy(plan)
        (B, H_k, dk), (_, H_v, dv) = q.shape, v.shape
        o = torch.empty_like(v)
        if outside is not None:
            o.record_stream(outside)
        rc = binding.load_library().vla_delta_decode_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), S.data_ptr(),
                                                          o.data_ptr(), B, H_k, H_v, dk, dv, _io(torch, q), ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_delta_decode_step")
    if not S.is_inference():
        torch.autograd.graph.increment_version(S)     # a graph that saved S must not use what it holds now
    return o


def _backward(torch, kept, op, saved, do, dS_T, state, handle, outside):
    """kept, op, handle, outside: as for _forward().  The gradients, with state also that of S0."""
    q, k, v, g, beta, _ = kept
    B, H_k, T, dk = q.shape
    H_v, dv, dev, io = v.shape[1], v.shape[3], q.device, _io(torch, q)
    lib = binding.load_library()
    (do, op.o), dS_T = _laid_out(do), _aligned(dS_T)
    dq, dk_, dv_ = _like(torch, q), _like(torch, k), _like(torch, v)
    dg, dbeta = (torch.empty((B, H_v, T), dtype=torch.float32, device=dev) for _ in range(2))
    dS0 = torch.empty((B, H_v, dv, dk), dtype=torch.float32, device=dev) if state else None
    op.dq, op.dk, op.dv = _strides(dq), _strides(dk_), _strides(dv_)
    saved = _together(saved)
    op.saved, op.saved_bytes = saved.data_ptr(), saved.numel()
    need = _workspace_bytes(B, H_k, H_v, T, dk, dv, io, op.segments, 1)
    ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
    outputs = (dq, dk_, dv_, dg, dbeta, dS0)
    if outside is not None:
        for t in outputs[:6 if state else 5]:
            t.record_stream(outside)
    rc = lib.vla_delta_backward(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), do.data_ptr(), _p(dS_T), dq.data_ptr(),
                                dk_.data_ptr(), dv_.data_ptr(), dg.data_ptr(), dbeta.data_ptr(), _p(dS0), B, H_k, H_v, T, dk, dv, io,
                                ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_delta_backward")
    return outputs


def _gradients(torch, q, k, v, g, beta, saved, do, dS_T, scale, lengths, segments, state, stream):
    """gated_delta_backward on these tensors; state: as for _backward()."""
    key = _key(q, k, v, g, beta, dS_T, lengths, scale, segments)
    if key not in _plans:
        _check(torch, q, k, v, g, beta, dS_T, "dS_T", lengths, 1)
    if do.shape != v.shape or do.dtype != v.dtype or do.device != v.device:
        raise ValueError("do must match v in shape, dtype and device")
    if saved.dtype != torch.uint8 or saved.dim() != 1 or not saved.is_contiguous() or saved.device != q.device:
        raise ValueError(f"saved must be what gated_delta_forward returned: a contiguous uint8 tensor on {q.device}")
    handle, context, outside = binding._on_stream(torch, q.device, stream)
    with context:
        kept, op = _inputs(key, q, k, v, g, beta, scale, lengths, segments)
        return _backward(torch, kept, op, saved, do, dS_T, state, handle, outside)


def gated_delta_backward(q, k, v, g, beta, saved, do, dS_T=None, *, scale=None, lengths=None, segments=0, stream=None):
    """The gradients (dq, dk, dv, dg, dbeta, dS0) of gated_delta_forward's inputs, given those of o and S_T (None: zero), the same inputs
    and what it saved.  dg, dbeta and dS0 are float32."""
    import torch

    scale = None if scale is None else float(scale)
    return _gradients(torch, q, k, v, g, beta, saved, do, dS_T, scale, lengths, segments, True, stream)


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class GatedDelta(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, v, g, beta, S0, key, scale, lengths):
                handle, context, outside = binding._on_stream(torch, q.device, None)
                with context:
                    kept, op = _inputs(key, q, k, v, g, beta, scale, lengths)
                    o, S_T, saved = _forward(torch, kept, op, S0, True, handle, outside)
                ctx.save_for_backward(*kept, saved)      # the inputs as the kernels read them
                ctx.scale = scale
                ctx.set_materialize_grads(False)
                return o, S_T

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, do, dS_T):
                # hooks (offload, checkpoints) may give other tensors than the saved ones: addresses and strides are those of these
                q, k, v, g, beta, lengths, saved = ctx.saved_tensors
                do = torch.zeros_like(v) if do is None else do
                dS_T = None if dS_T is None else dS_T.contiguous()
                grads = _gradients(torch, q, k, v, g, beta, saved, do, dS_T, ctx.scale, lengths, 0, ctx.needs_input_grad[5], None)
                return (*grads, None, None, None)

        _function = GatedDelta
    return _function


def gated_delta(q, k, v, g, beta, S0=None, *, scale=None, lengths=None, stream=None):
    """gated_delta_forward as a differentiable function: (o, S_T), with gradients for q, k, v, g, beta and S0 (once, in reverse mode, on
    the current stream)."""
    import torch

    _no_tangents(torch, q, k, v, g, beta, S0)
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or g.requires_grad or beta.requires_grad
                                    or S0 is not None and S0.requires_grad):
        if stream is not None:
            raise ValueError("with gradients the work goes to the current stream: leave stream at None")
        scale = None if scale is None else float(scale)
        key = _key(q, k, v, g, beta, S0, lengths, scale)
        if key not in _plans:
            _check(torch, q, k, v, g, beta, S0, "S0", lengths, 1)
        return _autograd().apply(q, k, v, g, beta, S0, key, scale, lengths)
    return gated_delta_forward(q, k, v, g, beta, S0, scale=scale, lengths=lengths, stream=stream)

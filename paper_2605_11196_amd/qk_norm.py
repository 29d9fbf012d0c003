"""Norm of queries and keys for each head with the position rotation, on torch tensors (vla_qk_norm_rope of include/vla.h)."""
import ctypes

from . import binding
from .binding import VLA_BF16, VLA_F32, VlaError, VlaNormOpts, VlaStrides


def _io(torch, x):
    if x.dtype == torch.float32:
        return VLA_F32
    if x.dtype == torch.bfloat16:
        return VLA_BF16
    raise ValueError(f"unsupported dtype {x.dtype}")


def _fits(what, *numbers):
    """ctypes cuts what an int of the library does not hold."""
    for n in numbers:
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{what} must fit 32 bits, not {n}")


def _no_tangents(torch, *tensors):
    """Refuses tensors of forward mode, whose tangents would be lost."""
    ad = torch.autograd.forward_ad
    if getattr(ad, "_current_level", -1) >= 0 and any(x is not None and ad.unpack_dual(x).tangent is not None for x in tensors):
        raise NotImplementedError("gradients in reverse mode alone: no jvp for forward mode")


def _steps(x):
    """The strides of the first three dimensions; 0 where a dimension has one entry and its stride says nothing."""
    return [step if n > 1 else 0 for step, n in zip(x.stride(), x.shape[:3])]


def _laid_out(x):
    """x and its strides for the C call, or a contiguous copy where it is not laid out as the kernels take it: the last dimension
    together, the other strides multiples of 16 bytes and not all zero for rows that repeat, tokens apart but not too far, 16-byte
    alignment."""
    aligned = not x.data_ptr() & 15
    if x.is_contiguous():
        return (x if aligned else x.clone()), _CONTIGUOUS
    s, size = _steps(x), x.element_size()
    if (aligned and x.stride(-1) == 1 and not any(step * size & 15 for step in s) and any(s)
            and (x.shape[2] <= 1 or x.shape[-1] <= s[2] < 2 ** 26 // size)):
        return x, VlaStrides(*s)
    return x.contiguous(), _CONTIGUOUS


_CONTIGUOUS = VlaStrides(0, 0, 0)


def _strides(x):
    return VlaStrides(*_steps(x))


def _like(torch, x):
    """An empty tensor with x's shape and order of dimensions, without gaps."""
    y = torch.empty_like(x)
    return y if y.stride(-1) == 1 else torch.empty_like(x, memory_format=torch.contiguous_format)


def _check(torch, q, k, q_weight, k_weight, cos, sin, positions, norm):
    dev, dtype, shape, k_shape = q.device, q.dtype, q.shape, k.shape
    _fits("sizes", *shape, *k_shape)
    if not (q.is_cuda and k.is_cuda):
        raise ValueError("q and k must be GPU tensors (no CPU path exists)")
    if k.dtype != dtype or len(shape) != 4 or len(k_shape) != 4 or shape[0] != k_shape[0] or shape[2:] != k_shape[2:] or k.device != dev:
        raise ValueError("expected q [B,H_q,T,d] and k [B,H_k,T,d] of one dtype on one device")
    if norm not in ("rms", "l2"):
        raise ValueError(f"norm must be 'rms' or 'l2', not {norm!r}")
    d = shape[3]
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (w.shape != (d,) or w.dtype not in (torch.float32, torch.bfloat16) or w.device != dev):
            raise ValueError(f"{name} must be a float32 or bfloat16 tensor of shape {(d,)} on {dev}")
    if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
        raise ValueError("q_weight and k_weight must share a dtype")
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        table = cos.shape
        _fits("sizes", *table)
        if (cos.dtype != torch.float32 or sin.dtype != torch.float32 or len(table) != 2 or sin.shape != table or cos.device != dev
                or sin.device != dev or not 0 < 2 * table[1] <= d or table[0] < 1):
            raise ValueError(f"cos and sin must be float32 tensors [positions, rot / 2] on {dev}")
    if positions is not None and (positions.dtype != torch.int32 or positions.shape != (shape[0], shape[2]) or positions.device != dev):
        raise ValueError(f"positions must be an int32 tensor of shape {(shape[0], shape[2])} on {dev}")


# Options of calls whose tensors go to the kernels as they are, by the shapes, layouts and types of these: a call like an earlier one is
# neither checked nor laid out again (5 of 17 us for a token of a layer).
_plans = {}


def _keep_plan(plans, key, kept, given, op):
    """Keeps op, which has no addresses yet, where nothing was copied."""
    if all(x is y for x, y in zip(kept, given)):
        if len(plans) >= 1024:
            plans.clear()
        plans[key] = bytes(op)


def _kind(x):
    return None if x is None else (x.shape, x.stride(), x.dtype, x.device)


def _together(x):
    """x contiguous and 16-byte aligned."""
    x = x.contiguous()
    return x.clone() if x.data_ptr() & 15 else x


def _key(q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved):
    return (q.shape, q.stride(), q.dtype, q.device, k.shape, k.stride(), k.dtype, k.device, _kind(q_weight), _kind(k_weight), _kind(cos), _kind(sin),
            _kind(positions), eps, norm, bool(interleaved))


def _call(torch, key, q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved):
    """What both directions share: the tensors as the kernels take them, which have to live until the call, and the options."""
    given = q, k, q_weight, k_weight, cos, sin, positions
    if not 0 <= offset < 2 ** 31:
        _fits("offset", offset)
    plan = _plans.get(key)
    if plan is not None and not (q.data_ptr() | k.data_ptr() | (_p(q_weight) or 0) | (_p(k_weight) or 0) | (_p(cos) or 0) | (_p(sin) or 0)) & 15:
        op = VlaNormOpts.from_buffer_copy(plan)
        op.offset = offset
        if positions is not None:
            op.positions = positions.data_ptr()
        return given, op
    op = VlaNormOpts(eps, norm == "l2", bool(interleaved))
    (q, op.q), (k, op.k) = _laid_out(q), _laid_out(k)
    if q_weight is not None:
        q_weight = _together(q_weight)
    if k_weight is not None:
        k_weight = _together(k_weight)
    weight = k_weight if q_weight is None else q_weight
    if weight is not None and weight.dtype == torch.bfloat16:
        op.weight_dtype = VLA_BF16
    if cos is not None:
        cos, sin = _together(cos), _together(sin)
        op.places, half = cos.shape
        op.rot = 2 * half
    if positions is not None:
        positions = positions.contiguous()
    kept = q, k, q_weight, k_weight, cos, sin, positions
    if plan is None:
        _keep_plan(_plans, key, kept, given, op)
    op.offset = offset
    if positions is not None:
        op.positions = positions.data_ptr()
    return kept, op


def _p(x):
    return None if x is None else x.data_ptr()


def _forward(torch, kept, op, handle, outside):
    """kept, op: of _call(), the inputs checked; handle, outside: of binding._on_stream(), in whose context this runs.  (q, k) after the
    norm and the rotation."""
    q, k = kept[0], kept[1]
    B, H_q, T, d = q.shape
    q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
    if outside is not None:
        q_out.record_stream(outside)
        k_out.record_stream(outside)
    rc = binding.load_library().vla_qk_norm_rope(
        q.data_ptr(), k.data_ptr(), _p(kept[2]), _p(kept[3]), _p(kept[4]), _p(kept[5]), q_out.data_ptr(), k_out.data_ptr(), B, T, H_q, k.shape[1],
        d, _io(torch, q), ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_qk_norm_rope")
    return q_out, k_out


def _backward(torch, kept, op, dq_out, dk_out, wanted, handle, outside):
    """kept, op, handle, outside: as for _forward().  The gradients (dq, dk, dq_weight, dk_weight), of the weights those that are wanted."""
    q, k, q_weight, k_weight = kept[:4]
    B, H_q, T, d = q.shape
    dev = q.device
    lib = binding.load_library()
    (dq_out, op.q_out), (dk_out, op.k_out) = _laid_out(dq_out), _laid_out(dk_out)
    dq, dk = _like(torch, q), _like(torch, k)
    op.dq, op.dk = _strides(dq), _strides(dk)
    dwq = torch.empty_like(q_weight) if wanted[0] and q_weight is not None else None
    dwk = torch.empty_like(k_weight) if wanted[1] and k_weight is not None else None
    need = lib.vla_qk_norm_rope_workspace_bytes(d) if dwq is not None or dwk is not None else 0
    ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
    if outside is not None:
        for t in (dq, dk, dwq, dwk):
            if t is not None:
                t.record_stream(outside)
    rc = lib.vla_qk_norm_rope_backward(
        q.data_ptr(), k.data_ptr(), _p(q_weight), _p(k_weight), _p(kept[4]), _p(kept[5]), dq_out.data_ptr(), dk_out.data_ptr(),
        dq.data_ptr(), dk.data_ptr(), _p(dwq), _p(dwk), B, T, H_q, k.shape[1], d, _io(torch, q), ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_qk_norm_rope_backward")
    return dq, dk, dwq, dwk


def _gradients(torch, q, k, q_weight, k_weight, cos, sin, positions, how, dq_out, dk_out, wanted, stream):
    """qk_norm_rope_backward on these tensors; wanted: as for _backward()."""
    key = _key(q, k, q_weight, k_weight, cos, sin, positions, *how)
    if key not in _plans:
        _check(torch, q, k, q_weight, k_weight, cos, sin, positions, how[2])
    for x, y in ((q, dq_out), (k, dk_out)):
        if y.shape != x.shape or y.dtype != x.dtype or y.device != x.device:
            raise ValueError("dq_out and dk_out must match q and k in shape, dtype and device")
    handle, context, outside = binding._on_stream(torch, q.device, stream)
    with context:
        kept, op = _call(torch, key, q, k, q_weight, k_weight, cos, sin, positions, *how)
        return _backward(torch, kept, op, dq_out, dk_out, wanted, handle, outside)


def qk_norm_rope_backward(q, k, q_weight, k_weight, cos, sin, dq_out, dk_out, *, positions=None, offset=0, eps=1e-6, norm="rms",
                          interleaved=False, stream=None):
    """The gradients of qk_norm_rope's q, k, q_weight and k_weight (None where there is no weight; summed in float32 and of the weights'
    type), given those of its outputs."""
    import torch

    how = (int(offset), float(eps), norm, interleaved)
    return _gradients(torch, q, k, q_weight, k_weight, cos, sin, positions, how, dq_out, dk_out, (True, True), stream)


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class QkNormRope(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, key, how):
                handle, context, outside = binding._on_stream(torch, q.device, None)
                with context:
                    kept, op = _call(torch, key, q, k, q_weight, k_weight, cos, sin, positions, *how)
                    ctx.save_for_backward(*kept)     # the inputs as the kernels read them
                    ctx.how = how
                    ctx.set_materialize_grads(False)
                    return _forward(torch, kept, op, handle, outside)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dq_out, dk_out):
                # hooks (offload, checkpoints) may give other tensors than the saved ones: addresses and strides are those of these
                q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
                dq_out = torch.zeros_like(q) if dq_out is None else dq_out
                dk_out = torch.zeros_like(k) if dk_out is None else dk_out
                grads = _gradients(torch, q, k, q_weight, k_weight, cos, sin, positions, ctx.how, dq_out, dk_out, ctx.needs_input_grad[2:4], None)
                return (*grads, None, None, None, None, None)

        _function = QkNormRope
    return _function


def qk_norm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, *, positions=None, offset=0, eps=1e-6, norm="rms",
                 interleaved=False, stream=None):
    """Norm of every query and key head and the position rotation in one pass.

    q [B,H_q,T,d], k [B,H_k,T,d] on the GPU (float32 or bfloat16), any views with a contiguous last dimension, such as the slices
    of a fused projection [B,T,H d] with tokens and heads swapped.  norm: "rms" (by the root of the mean square) or "l2" (unit length).
    q_weight, k_weight: [d] or None.  cos, sin: float32 [positions, rot / 2], the tables of the rotation of the first rot
    columns (None: no rotation).  Token t is at positions[b, t] (int32), or at offset + t.  Returns contiguous (q, k), which
    vla_forward and gated_delta take; differentiable in q, k and the weights (once, in reverse mode, on the current stream).
    """
    import torch

    _no_tangents(torch, q, k, q_weight, k_weight, cos, sin)
    how = (int(offset), float(eps), norm, interleaved)
    train = torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or q_weight is not None and q_weight.requires_grad
                                         or k_weight is not None and k_weight.requires_grad)
    if train and stream is not None:
        raise ValueError("with gradients the work goes to the current stream: leave stream at None")
    key = _key(q, k, q_weight, k_weight, cos, sin, positions, *how)
    if key not in _plans:
        _check(torch, q, k, q_weight, k_weight, cos, sin, positions, norm)
    if train:
        return _autograd().apply(q, k, q_weight, k_weight, cos, sin, positions, key, how)
    handle, context, outside = binding._on_stream(torch, q.device, stream)
    with context:
        kept, op = _call(torch, key, q, k, q_weight, k_weight, cos, sin, positions, *how)
        return _forward(torch, kept, op, handle, outside)

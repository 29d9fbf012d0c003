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


def _steps(x):
    """The strides of the first three dimensions; 0 where a dimension has one entry and its stride says nothing."""
    return [step if n > 1 else 0 for step, n in zip(x.stride(), x.shape[:3])]


def _rows(x):
    """x, or a contiguous copy where it is not laid out as the kernels take it: the last dimension together, the other strides
    multiples of 16 bytes and not all zero for rows that repeat, tokens apart but not too far, 16-byte alignment."""
    per16 = 16 // x.element_size()
    s = _steps(x)
    fits = (x.stride(-1) == 1 and not any(step % per16 for step in s) and (any(s) or x.is_contiguous())
            and (x.shape[2] <= 1 or x.shape[-1] <= s[2] < 2 ** 26 // x.element_size()))
    if fits and x.data_ptr() % 16 == 0:
        return x
    return x.clone() if x.is_contiguous() else x.contiguous()


def _strides(x):
    return VlaStrides(*_steps(x))


def _like(torch, x):
    """An empty tensor with x's shape and order of dimensions, without gaps."""
    y = torch.empty_like(x)
    return y if y.stride(-1) == 1 else torch.empty_like(x, memory_format=torch.contiguous_format)


def _check(torch, q, k, q_weight, k_weight, cos, sin, positions, norm):
    if not (q.is_cuda and k.is_cuda):
        raise ValueError("q and k must be GPU tensors (no CPU path exists)")
    if k.dtype != q.dtype or q.dim() != 4 or k.dim() != 4 or (k.shape[0], *k.shape[2:]) != (q.shape[0], *q.shape[2:]) or k.device != q.device:
        raise ValueError("expected q [B,H_q,T,d] and k [B,H_k,T,d] of one dtype on one device")
    if norm not in ("rms", "l2"):
        raise ValueError(f"norm must be 'rms' or 'l2', not {norm!r}")
    d = q.shape[-1]
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (w.shape != (d,) or w.dtype not in (torch.float32, torch.bfloat16) or w.device != q.device):
            raise ValueError(f"{name} must be a float32 or bfloat16 tensor of shape {(d,)} on {q.device}")
    if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
        raise ValueError("q_weight and k_weight must share a dtype")
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        for name, t in (("cos", cos), ("sin", sin)):
            if t.dtype != torch.float32 or t.dim() != 2 or t.shape != cos.shape or t.device != q.device or not 0 < 2 * t.shape[1] <= d or t.shape[0] < 1:
                raise ValueError(f"{name} must be a float32 tensor [positions, rot / 2] on {q.device}")
    if positions is not None and (positions.dtype != torch.int32 or tuple(positions.shape) != (q.shape[0], q.shape[2]) or positions.device != q.device):
        raise ValueError(f"positions must be an int32 tensor of shape {(q.shape[0], q.shape[2])} on {q.device}")


def _call(torch, q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved):
    """The arguments that both directions share, ready for the C call: tensors that have to live until it, and the options."""
    q, k = _rows(q), _rows(k)
    same = lambda x: None if x is None else x.contiguous()
    kept = [q, k, same(q_weight), same(k_weight), same(cos), same(sin), same(positions)]
    for i in (2, 3, 4, 5):
        if kept[i] is not None and kept[i].data_ptr() % 16:
            kept[i] = kept[i].clone()
    op = VlaNormOpts(eps=eps, l2=norm == "l2", interleaved=bool(interleaved), offset=offset)
    if cos is not None:
        op.rot, op.places = 2 * cos.shape[1], cos.shape[0]
    weight = q_weight if q_weight is not None else k_weight
    op.weight_dtype = VLA_BF16 if weight is not None and weight.dtype == torch.bfloat16 else VLA_F32
    if positions is not None:
        op.positions = kept[6].data_ptr()
    op.q, op.k = _strides(q), _strides(k)
    return kept, op


def _p(x):
    return None if x is None else x.data_ptr()


def _forward(q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved, stream):
    import torch

    _check(torch, q, k, q_weight, k_weight, cos, sin, positions, norm)
    io, (B, H_q, T, d), H_k, dev = _io(torch, q), q.shape, k.shape[1], q.device
    lib = binding.load_library()
    handle, context, outside = binding._on_stream(torch, dev, stream)
    with context:
        kept, op = _call(torch, q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved)
        q_out, k_out = (torch.empty(x.shape, dtype=q.dtype, device=dev) for x in (q, k))
        if outside is not None:
            q_out.record_stream(outside)
            k_out.record_stream(outside)
        rc = lib.vla_qk_norm_rope(*(_p(x) for x in kept[:6]), _p(q_out), _p(k_out), B, T, H_q, H_k, d, io, ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_qk_norm_rope")
    return q_out, k_out


def qk_norm_rope_backward(q, k, q_weight, k_weight, cos, sin, dq_out, dk_out, *, positions=None, offset=0, eps=1e-6, norm="rms",
                          interleaved=False, stream=None):
    """The gradients of qk_norm_rope's q, k, q_weight and k_weight (the last two float32, None where there is no weight), given
    those of its outputs."""
    import torch

    _check(torch, q, k, q_weight, k_weight, cos, sin, positions, norm)
    if any(y.shape != x.shape or y.dtype != x.dtype or y.device != x.device for x, y in ((q, dq_out), (k, dk_out))):
        raise ValueError("dq_out and dk_out must match q and k in shape, dtype and device")
    io, (B, H_q, T, d), H_k, dev = _io(torch, q), q.shape, k.shape[1], q.device
    lib = binding.load_library()
    handle, context, outside = binding._on_stream(torch, dev, stream)
    with context:
        kept, op = _call(torch, q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved)
        dq_out, dk_out, dq, dk = _rows(dq_out), _rows(dk_out), _like(torch, q), _like(torch, k)
        op.q_out, op.k_out, op.dq, op.dk = (_strides(x) for x in (dq_out, dk_out, dq, dk))
        dw = [None if w is None else torch.empty((d,), dtype=torch.float32, device=dev) for w in (q_weight, k_weight)]
        need = lib.vla_qk_norm_rope_workspace_bytes(d) if q_weight is not None or k_weight is not None else 0
        ws = torch.empty((need,), dtype=torch.uint8, device=dev) if need else None
        if outside is not None:
            for t in (dq, dk, *dw):
                if t is not None:
                    t.record_stream(outside)
        rc = lib.vla_qk_norm_rope_backward(*(_p(x) for x in kept[:6]), _p(dq_out), _p(dk_out), _p(dq), _p(dk), _p(dw[0]), _p(dw[1]), B, T,
                                           H_q, H_k, d, io, ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_qk_norm_rope_backward")
    return dq, dk, dw[0], dw[1]


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class QkNormRope(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, how):
                ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
                ctx.how = how
                return _forward(q, k, q_weight, k_weight, cos, sin, positions, how["offset"], how["eps"], how["norm"], how["interleaved"], None)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dq_out, dk_out):
                q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
                dq, dk, dwq, dwk = qk_norm_rope_backward(q, k, q_weight, k_weight, cos, sin, dq_out, dk_out, positions=positions, **ctx.how)
                cast = lambda g, w: g if g is None else g.to(w.dtype)
                return dq, dk, cast(dwq, q_weight), cast(dwk, k_weight), None, None, None, None

        _function = QkNormRope
    return _function


def qk_norm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, *, positions=None, offset=0, eps=1e-6, norm="rms",
                 interleaved=False, stream=None):
    """Norm of every query and key head and the position rotation in one pass.

    q [B,H_q,T,d], k [B,H_k,T,d] on the GPU (float32 or bfloat16), any views with a contiguous last dimension, such as the slices
    of a fused projection [B,T,H d] with tokens and heads swapped.  norm: "rms" (by the root of the mean square) or "l2" (unit length).
    q_weight, k_weight: [d] or None.  cos, sin: float32 [positions, rot / 2], the tables of the rotation of the first rot
    columns (None: no rotation).  Token t is at positions[b, t] (int32), or at offset + t.  Returns contiguous (q, k), which
    vla_forward and gated_delta take; differentiable in q, k and the weights (on the current stream).
    """
    import torch

    offset, eps = int(offset), float(eps)
    if torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in (q, k, q_weight, k_weight)):
        if stream is not None:
            raise ValueError("with gradients the work goes to the current stream: leave stream at None")
        how = dict(offset=offset, eps=eps, norm=norm, interleaved=interleaved)
        return _autograd().apply(q, k, q_weight, k_weight, cos, sin, positions, how)
    return _forward(q, k, q_weight, k_weight, cos, sin, positions, offset, eps, norm, interleaved, stream)

"""The norms around a block with its gate and residual scale on torch tensors (vla_residual_norm of include/vla.h)."""
import ctypes

from . import binding
from .binding import VLA_BF16, VLA_F32, VlaError, VlaResidualOpts
from .rows import (_all_aligned, _check_rows, _check_vector, _fits, _io, _kind, _laid_rows, _like, _no_tangents, _p, _plan, _plans, _record,
                   _together, _wants_gradients)

_ACTIVATIONS = {"silu": 0, "sigmoid": 1}


def _check(torch, x, y, weight, post_weight, gate, scale, groups, activation):
    row = x if y is None else y
    if row is None:
        raise ValueError("one of x and y has to be given")
    dev, shape = row.device, row.shape
    _fits("sizes", *shape)
    if not row.is_cuda:
        raise ValueError("x and y must be GPU tensors (no CPU path exists)")
    if len(shape) != 3:
        raise ValueError("expected rows as [B,T,n]")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be 'silu' or 'sigmoid', not {activation!r}")
    if y is None and not (post_weight is None and gate is None and scale is None):
        raise ValueError("post_weight, gate and scale go with y")
    if y is None and weight is None:
        raise ValueError("without y there is a norm alone: weight has to be given")
    if x is not None and y is not None:
        if x.shape != shape or x.device != dev or x.dtype not in (y.dtype, torch.float32):
            raise ValueError(f"x must be a float32 or {str(y.dtype).replace('torch.', '')} tensor of shape {tuple(shape)} on {dev}")
    _check_rows(torch, "gate", gate, shape, row.dtype, dev)
    if groups < 1 or shape[-1] % groups:
        raise ValueError(f"groups ({groups}) must divide the {shape[-1]} columns")
    given = [w for w in (weight, post_weight, scale) if w is not None]
    types = (torch.float32, torch.bfloat16) if not given else (given[0].dtype,) if given[0].dtype in (torch.float32, torch.bfloat16) else ()
    for name, w in (("weight", weight), ("post_weight", post_weight), ("scale", scale)):
        _check_vector(torch, name, w, (shape[-1],), dev, types or (torch.float32, torch.bfloat16))


def _key(x, y, weight, post_weight, gate, scale, groups, eps, activation):
    return ("residual", _kind(x), _kind(y), _kind(weight), _kind(post_weight), _kind(gate), _kind(scale), groups, eps, activation)


def _inputs(torch, key, x, y, weight, post_weight, gate, scale, groups, eps, activation):
    """The inputs as the kernels take them, kept until the call, and its options."""
    given = x, y, weight, post_weight, gate, scale
    plan = _plans.get(key)
    if plan is not None and _all_aligned(*given):
        return given, VlaResidualOpts.from_buffer_copy(plan)
    row = x if y is None else y
    op = VlaResidualOpts(eps, 0 if groups == 1 else row.shape[-1] // groups, _ACTIVATIONS[activation])
    op.stream_dtype = _io(torch, row if x is None else x)
    if x is not None:
        x, op.x = _laid_rows(x)
    if y is not None:
        y, op.y = _laid_rows(y)
    if gate is not None:
        gate, op.gate = _laid_rows(gate)
    weight, post_weight, scale = (None if w is None else _together(w) for w in (weight, post_weight, scale))
    for w in (weight, post_weight, scale):
        if w is not None:
            op.weight_dtype = VLA_BF16 if w.dtype == torch.bfloat16 else VLA_F32
    kept = x, y, weight, post_weight, gate, scale
    if plan is None:
        _plan(key, given, kept, op)
    return kept, op


def _forward(torch, kept, op, handle, outside):
    """(s, h), None where the call has no such output."""
    x, y, weight, post_weight, gate, scale = kept
    row = x if y is None else y
    B, T, n = row.shape
    s = None if y is None else _like(torch, y if x is None else x)
    h = None if weight is None else _like(torch, row)
    _record(outside, s, h)
    rc = binding.load_library().vla_residual_norm(_p(x), _p(y), _p(gate), _p(post_weight), _p(scale), _p(weight), _p(s), _p(h), B, T, n,
                                                  _io(torch, row), ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_residual_norm")
    return s, h


def _gradients(torch, x, y, weight, post_weight, gate, scale, how, ds, dh, wanted, stream):
    """residual_norm_backward on these tensors; wanted: whether the gradients of x, y, weight, post_weight, gate and scale are."""
    key = _key(x, y, weight, post_weight, gate, scale, *how)
    if key not in _plans:
        _check(torch, x, y, weight, post_weight, gate, scale, how[0], how[2])
    row, streamed = x if y is None else y, y if x is None else x
    _check_rows(torch, "ds", ds, row.shape, streamed.dtype, row.device)
    _check_rows(torch, "dh", dh, row.shape, row.dtype, row.device)
    if dh is not None and weight is None:
        raise ValueError("dh goes with weight")
    handle, context, outside = binding._on_stream(torch, row.device, stream)
    with context:
        (x, y, weight, post_weight, gate, scale), op = _inputs(torch, key, x, y, weight, post_weight, gate, scale, *how)
        B, T, n = row.shape
        lib = binding.load_library()
        if ds is not None:
            ds, op.s = _laid_rows(ds)
        if dh is not None:
            dh, op.h = _laid_rows(dh)
        rows = [None if t is None or not w else _like(torch, t) for t, w in zip((x, y, gate), wanted[:2] + wanted[4:5])]
        sums = [None if t is None or not w else torch.empty_like(t) for t, w in zip((post_weight, scale, weight), (wanted[3], wanted[5], wanted[2]))]
        need = lib.vla_residual_norm_workspace_bytes(n) if any(t is not None for t in sums) else 0
        ws = torch.empty((need,), dtype=torch.uint8, device=row.device) if need else None
        _record(outside, *rows, *sums)
        rc = lib.vla_residual_norm_backward(_p(x), _p(y), _p(gate), _p(post_weight), _p(scale), _p(weight), _p(ds), _p(dh), *(_p(t) for t in rows),
                                            *(_p(t) for t in sums), B, T, n, _io(torch, row), ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_residual_norm_backward")
    return rows[0], rows[1], sums[2], sums[0], rows[2], sums[1]


def residual_norm_backward(x, y, weight, ds, dh, *, post_weight=None, groups=1, gate=None, activation="silu", scale=None, eps=1e-6, stream=None):
    """The gradients (dx, dy, dweight, dpost_weight, dgate, dscale) of residual_norm's inputs (None where there is no such input; the weights'
    summed in float32 and of the weights' type), given those of s and h (None: zero)."""
    import torch

    how = (int(groups), float(eps), activation)
    return _gradients(torch, x, y, weight, post_weight, gate, scale, how, ds, dh, (True,) * 6, stream)


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class ResidualNorm(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, y, weight, post_weight, gate, scale, key, how):
                row = x if y is None else y
                handle, context, outside = binding._on_stream(torch, row.device, None)
                with context:
                    kept, op = _inputs(torch, key, x, y, weight, post_weight, gate, scale, *how)
                    ctx.save_for_backward(*kept)      # the inputs as the kernels read them
                    ctx.how = how
                    ctx.set_materialize_grads(False)
                    return _forward(torch, kept, op, handle, outside)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, ds, dh):
                # hooks (offload, checkpoints) may give other tensors than the saved ones: addresses and strides are those of these
                return (*_gradients(torch, *ctx.saved_tensors, ctx.how, ds, dh, ctx.needs_input_grad[:6], None), None, None)

        _function = ResidualNorm
    return _function


def residual_norm(x, y=None, weight=None, *, post_weight=None, groups=1, gate=None, activation="silu", scale=None, eps=1e-6, stream=None):
    """What stands between a block and the next one, in one pass:  s = x + scale * act(gate) * post_weight * N(y);  h = weight * N(s).

    x: the residual stream [B,T,n] or None (zero), y: the block's output [B,T,n] on the GPU (float32 or bfloat16, n a multiple of 8 up to
    8192; views with a contiguous last dimension are read as they are); x may be float32 with y bfloat16; s has x's type and h y's (without y: x's).  N divides by the
    root of the mean square + eps, of the row, and of y over each of `groups` groups of neighbouring columns (heads).  gate [B,T,n] of y's
    type goes through activation ("silu" or "sigmoid"); post_weight, scale and weight [n] share a type.  What is None is left out: without
    post_weight y has no norm, without weight h is None, without y the call is h = weight * N(x), and s is x.  Returns
    (s, h); differentiable in all tensors (once, in reverse mode, on the current stream).
    """
    import torch

    _no_tangents(torch, x, y, weight, post_weight, gate, scale)
    how = (int(groups), float(eps), activation)
    train = _wants_gradients(torch, x, y, weight, post_weight, gate, scale)
    if train and stream is not None:
        raise ValueError("with gradients the work goes to the current stream: leave stream at None")
    key = _key(x, y, weight, post_weight, gate, scale, *how)
    if key not in _plans:
        _check(torch, x, y, weight, post_weight, gate, scale, how[0], activation)
    if train:
        s, h = _autograd().apply(x, y, weight, post_weight, gate, scale, key, how)
    else:
        handle, context, outside = binding._on_stream(torch, (x if y is None else y).device, stream)
        with context:
            kept, op = _inputs(torch, key, x, y, weight, post_weight, gate, scale, *how)
            s, h = _forward(torch, kept, op, handle, outside)
    return (x if y is None else s), h

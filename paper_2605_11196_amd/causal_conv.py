"""The short causal convolution of channels on torch tensors (vla_causal_conv of include/vla.h)."""
import ctypes
import functools

from . import binding
from .binding import VLA_BF16, VlaConvOpts, VlaError
from .rows import (_all_aligned, _check_lengths, _check_rows, _check_vector, _fits, _io, _kind, _laid_rows, _like, _no_tangents, _p, _plan, _plans,
                   _record, _together, _wants_gradients)

_ACTIVATIONS = {"silu": 1, None: 0}


def _check(torch, x, weight, bias, state, lengths, activation, tokens):
    """Shapes of a call over tokens (tokens 1) or of one token (0)."""
    dev, shape = x.device, x.shape
    _fits("sizes", *shape, *weight.shape)
    if not x.is_cuda:
        raise ValueError("x must be a GPU tensor (no CPU path exists)")
    if len(shape) != 2 + tokens:
        raise ValueError(f"expected x as {'[B,T,n]' if tokens else '[B,n]'}")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be 'silu' or None, not {activation!r}")
    B, n = shape[0], shape[-1]
    if weight.dim() != 2:
        raise ValueError("expected weight as [n,width]")
    types = torch.float32, torch.bfloat16
    _check_vector(torch, "weight", weight, (n, weight.shape[1]), dev, types)
    _check_vector(torch, "bias", bias, (n,), dev, (weight.dtype,))
    _check_rows(torch, "state", state, (B, weight.shape[1] - 1, n), x.dtype, dev)
    if not tokens and not state.is_contiguous():
        raise ValueError("state must be contiguous: it is updated in place")
    _check_lengths(torch, lengths, B, dev)


def _key(x, weight, bias, state, lengths, activation):
    return ("conv", x.shape, x.stride(), x.dtype, x.device, weight.shape, weight.stride(), weight.dtype, weight.device, _kind(bias), _kind(state),
            _kind(lengths), activation)


def _inputs(torch, key, x, weight, bias, state, lengths, activation):
    """The inputs as the kernels take them, kept until the call, and its options."""
    given = x, weight, bias, state, lengths
    plan = _plans.get(key)
    if plan is not None and _all_aligned(x, weight, bias, state):
        op = VlaConvOpts.from_buffer_copy(plan)
        if lengths is not None:
            op.lengths = lengths.data_ptr()
        return given, op
    op = VlaConvOpts(_ACTIVATIONS[activation])
    x, op.x = _laid_rows(x)
    weight, bias, state = _together(weight), None if bias is None else _together(bias), None if state is None else _together(state)
    if weight.dtype == torch.bfloat16:
        op.weight_dtype = VLA_BF16
    lengths = None if lengths is None else lengths.contiguous()
    kept = x, weight, bias, state, lengths
    if plan is None:
        _plan(key, given, kept, op)
    if lengths is not None:
        op.lengths = lengths.data_ptr()
    return kept, op


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(B, T, n, width, io):
    """vla_causal_conv_workspace_bytes, which depends on nothing else."""
    return binding.load_library().vla_causal_conv_workspace_bytes(B, T, n, width, io)


def _forward(torch, kept, op, handle, outside):
    x, weight, bias, state, _ = kept
    B, T, n = x.shape
    width = weight.shape[1]
    y = _like(torch, x)
    state_T = torch.empty((B, width - 1, n), dtype=x.dtype, device=x.device)
    _record(outside, y, state_T)
    rc = binding.load_library().vla_causal_conv(x.data_ptr(), weight.data_ptr(), _p(bias), _p(state), y.data_ptr(), state_T.data_ptr(), B, T, n, width,
                                                _io(torch, x), ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_causal_conv")
    return y, state_T


def causal_conv_step(x, weight, state, bias=None, *, activation="silu", stream=None):
    """One token: x [B,n], state [B,width-1,n] of x's type, contiguous and 16-byte aligned, moves on in place.  Returns y [B,n].  Without a
    gradient: for generation, under torch.no_grad() where an input asks for one."""
    import torch

    _no_tangents(torch, x, weight, state, bias)
    if _wants_gradients(torch, x, weight, state, bias):
        raise ValueError("causal_conv_step has no gradient: call it under torch.no_grad(), or causal_conv with one token")
    key = _key(x, weight, bias, state, None, activation)
    if key not in _plans:
        _check(torch, x, weight, bias, state, None, activation, 0)
    handle, context, outside = binding._on_stream(torch, x.device, stream)
    with context:
        B, n = x.shape
        (x, weight, bias, moved, _), op = _inputs(torch, key, x, weight, bias, state, None, activation)
        if moved is not state:
            raise ValueError("state must be 16-byte aligned: it is updated in place")
        y = _like(torch, x)
        _record(outside, y)
        rc = binding.load_library().vla_causal_conv_step(x.data_ptr(), weight.data_ptr(), _p(bias), state.data_ptr(), y.data_ptr(), B, n,
                                                         weight.shape[1], _io(torch, x), ctypes.byref(op), handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_causal_conv_step")
    if not state.is_inference():
        torch.autograd.graph.increment_version(state)     # a graph that saved the state must not use what it holds now
    return y


def _gradients(torch, x, weight, bias, state, dy, dstate_T, lengths, activation, wanted, stream):
    """causal_conv_backward on these tensors; wanted: whether the gradients of weight, bias and state are."""
    key = _key(x, weight, bias, state, lengths, activation)
    if key not in _plans:
        _check(torch, x, weight, bias, state, lengths, activation, 1)
    _check_rows(torch, "dy", dy, x.shape, x.dtype, x.device)
    width = weight.shape[1]
    _check_rows(torch, "dstate_T", dstate_T, (x.shape[0], width - 1, x.shape[2]), x.dtype, x.device)
    handle, context, outside = binding._on_stream(torch, x.device, stream)
    with context:
        (x, weight, bias, state, lengths), op = _inputs(torch, key, x, weight, bias, state, lengths, activation)
        B, T, n = x.shape
        lib, io = binding.load_library(), _io(torch, x)
        dy, op.y = _laid_rows(dy)
        dstate_T = None if dstate_T is None else _together(dstate_T)
        dx = _like(torch, x)
        dweight = torch.empty_like(weight) if wanted[0] else None
        dbias = torch.empty_like(bias) if wanted[1] and bias is not None else None
        dstate = torch.empty_like(state) if wanted[2] and state is not None else None
        need = _workspace_bytes(B, T, n, width, io) if dweight is not None or dbias is not None else 0
        ws = torch.empty((need,), dtype=torch.uint8, device=x.device) if need else None
        _record(outside, dx, dweight, dbias, dstate)
        rc = lib.vla_causal_conv_backward(x.data_ptr(), weight.data_ptr(), _p(bias), _p(state), dy.data_ptr(), _p(dstate_T), dx.data_ptr(),
                                          _p(dweight), _p(dbias), _p(dstate), B, T, n, width, io, ctypes.byref(op), _p(ws), need, handle)
    if rc != 0:
        raise VlaError(rc, binding.status_string(rc), "vla_causal_conv_backward")
    return dx, dweight, dbias, dstate


def causal_conv_backward(x, weight, bias, state, dy, dstate_T=None, *, activation="silu", lengths=None, stream=None):
    """The gradients (dx, dweight, dbias, dstate) of causal_conv's inputs (None where there is no such input), given those of its outputs
    (dstate_T None: zero); the weights' are summed in float32 and of the weights' type."""
    import torch

    return _gradients(torch, x, weight, bias, state, dy, dstate_T, lengths, activation, (True, True, True), stream)


_function = None


def _autograd():
    global _function
    if _function is None:
        import torch

        class CausalConv(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, weight, bias, state, lengths, key, activation):
                handle, context, outside = binding._on_stream(torch, x.device, None)
                with context:
                    kept, op = _inputs(torch, key, x, weight, bias, state, lengths, activation)
                    ctx.save_for_backward(*kept)      # the inputs as the kernels read them
                    ctx.activation = activation
                    ctx.set_materialize_grads(False)
                    return _forward(torch, kept, op, handle, outside)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dy, dstate_T):
                # hooks (offload, checkpoints) may give other tensors than the saved ones: addresses and strides are those of these
                x, weight, bias, state, lengths = ctx.saved_tensors
                dy = torch.zeros_like(x) if dy is None else dy
                grads = _gradients(torch, x, weight, bias, state, dy, dstate_T, lengths, ctx.activation, ctx.needs_input_grad[1:4], None)
                return (*grads, None, None, None)

        _function = CausalConv
    return _function


def causal_conv(x, weight, bias=None, state=None, *, activation="silu", lengths=None, stream=None):
    """y_t = act(bias + sum_j weight[:, j] x_{t - width + 1 + j}) for every channel: what stands before a recurrence.

    x [B,T,n] on the GPU (float32 or bfloat16, n a multiple of 8; views with a contiguous last dimension, such as slices of a fused projection,
    are read as they are), weight [n,width] (2 to 4 taps) and bias [n] float32 or bfloat16, state [B,width-1,n]: the rows before the first
    token (None: zero).  activation: "silu" or None.  lengths: int32 [B], tokens of each sequence; y is zero beyond.  Returns
    (y, state_T), which the next call or causal_conv_step continues from; differentiable in x, weight, bias and state (once, in reverse
    mode, on the current stream).
    """
    import torch

    _no_tangents(torch, x, weight, bias, state)
    train = _wants_gradients(torch, x, weight, bias, state)
    if train and stream is not None:
        raise ValueError("with gradients the work goes to the current stream: leave stream at None")
    key = _key(x, weight, bias, state, lengths, activation)
    if key not in _plans:
        _check(torch, x, weight, bias, state, lengths, activation, 1)
    if train:
        return _autograd().apply(x, weight, bias, state, lengths, key, activation)
    handle, context, outside = binding._on_stream(torch, x.device, stream)
    with context:
        kept, op = _inputs(torch, key, x, weight, bias, state, lengths, activation)
        return _forward(torch, kept, op, handle, outside)

"""What the operators on rows of channels [B,T,n] share on the side of torch: layouts, checks, options that are kept."""
from .binding import VlaStrides
from .qk_norm import _fits, _io, _kind, _no_tangents, _p, _together  # noqa: F401

_CONTIGUOUS = VlaStrides(0, 0, 0)


def _laid_rows(x):
    """x [B,T,n] (or [B,n]) and its strides for the C call, or a contiguous copy where it is not laid out as the kernels take it: the last
    dimension together, the others in steps of 16 bytes that are not all zero, tokens not too far apart, 16-byte alignment."""
    aligned = not x.data_ptr() & 15
    if x.is_contiguous():
        return (x if aligned else x.clone()), _CONTIGUOUS
    size, step = x.element_size(), [s if n > 1 else 0 for s, n in zip(x.stride(), x.shape[:-1])]
    if aligned and x.stride(-1) == 1 and not any(s * size & 15 for s in step) and any(step) and step[-1] * size < 2 ** 26:
        return x, VlaStrides(step[0], 0, step[1] if len(step) > 1 else 0)
    return x.contiguous(), _CONTIGUOUS


def _laid_groups(x):
    """The same for [B,T,G,N] (or [B,G,N]), whose strides go from sequence to sequence, from group to group and from token to token."""
    aligned = not x.data_ptr() & 15
    if x.is_contiguous():
        return (x if aligned else x.clone()), _CONTIGUOUS
    size, step = x.element_size(), [s if n > 1 else 0 for s, n in zip(x.stride(), x.shape[:-1])]
    if aligned and x.stride(-1) == 1 and not any(s * size & 15 for s in step) and any(step):
        return x, VlaStrides(step[0], step[-1], step[1] if len(step) > 2 else 0)
    return x.contiguous(), _CONTIGUOUS


def _check_vector(torch, name, w, shape, dev, dtypes):
    if w is not None and (tuple(w.shape) != shape or w.dtype not in dtypes or w.device != dev):
        types = " or ".join(str(d).replace("torch.", "") for d in dtypes)
        raise ValueError(f"{name} must be a {types} tensor of shape {shape} on {dev}")


def _check_lengths(torch, lengths, B, dev):
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (B,) or lengths.device != dev):
        raise ValueError(f"lengths must be an int32 tensor of shape {(B,)} on {dev}")


def _check_rows(torch, name, x, shape, dtype, dev):
    if x is not None and (x.shape != shape or x.dtype != dtype or x.device != dev):
        raise ValueError(f"{name} must be a {str(dtype).replace('torch.', '')} tensor of shape {tuple(shape)} on {dev}")


def _wants_gradients(torch, *tensors):
    return torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in tensors)


def _record(outside, *tensors):
    """Marks outputs that may be read on the stream that is current outside."""
    if outside is not None:
        for x in tensors:
            if x is not None:
                x.record_stream(outside)


# Options of calls whose tensors go to the kernels as they are, by the shapes, layouts and types of these: a call like an earlier one is
# neither checked nor laid out again.
_plans = {}


def _plan(key, given, kept, op):
    """Keeps op, which has no addresses yet, where nothing was copied."""
    if all(x is y for x, y in zip(given, kept)):
        if len(_plans) >= 1024:
            _plans.clear()
        _plans[key] = bytes(op)


def _all_aligned(*tensors):
    low = 0
    for x in tensors:
        if x is not None:
            low |= x.data_ptr()
    return not low & 15


def _like(torch, x):
    """An uninitialised contiguous tensor of x's shape and type (a third less time than torch.empty with all of them given)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)

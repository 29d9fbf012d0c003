"""The operators on rows of channels in 64 bits, and what the roundings of a float32 computation of them are measured by.

`magnitude=True` gives every sum with its terms' absolute values (and gradients of that form, which add absolute values of all that the
true ones add): a float32 computation whose terms each go through k roundings is off by at most about k 2^-24 of it.
"""
import torch

UNIT = 2.0 ** -24     # half a step of float32
EPS = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}   # of the results' own rounding beyond the float32 one


def close(got, want, magnitude, k, what=""):
    """got within k roundings of `magnitude`, and its own rounding (twice where that follows a rounding to bfloat16 in autograd)."""
    want, magnitude = want.double().cpu(), magnitude.double().cpu()
    tol = EPS[got.dtype] * want.abs() + (1 + EPS[got.dtype]) * k * UNIT * magnitude + 1e-37
    off = (got.detach().double().cpu() - want).abs()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((off / tol)[bad].max()), [int(i[0]) for i in bad.nonzero(as_tuple=True)])


def double(x):
    return None if x is None else x.detach().double().cpu()


def _valued(value, slope, x):
    """`value` with the derivative `slope` to x."""
    return value.detach() + slope.detach() * (x - x.detach())


def _silu(z, magnitude):
    """z sigmoid(z).  The sizes of value and slope: the sigmoid's exponential has an argument that is off by |z| half steps, so that it is off by
    (1 + |z|) of them times a small number; the slope is sigmoid(z) (1 + z (1 - sigmoid(z))), whose two terms cancel near z = -1.28, so that its
    size is sigmoid(z) (1 + |z| (1 - sigmoid(z)))."""
    s = torch.sigmoid(z)
    return _valued((z * s).abs() * (1 + z.abs()), s * (1 + z.abs() * (1 - s)) * (1 + z.abs()), z) if magnitude else z * s


def conv(x, weight, bias, state, lengths, silu, magnitude=False):
    B, T, n = x.shape
    W = weight.shape[1]
    if magnitude:
        signed = conv(x.detach(), weight.detach(), double(bias), double(state), lengths, False)[0]
        x, weight = x.abs(), weight.abs()
        bias, state = None if bias is None else bias.abs(), None if state is None else state.abs()
    rows = torch.cat((torch.zeros(B, W - 1, n, dtype=torch.float64) if state is None else state, x), 1)
    pre = sum(weight[:, j] * rows[:, j:j + T] for j in range(W)) + (0 if bias is None else bias)
    if silu:
        if magnitude:
            s = torch.sigmoid(signed)
            # as in _silu(); and a sum that is off by k half steps of `pre` (its terms' sizes) moves the value by the slope, which is 1.1 or less,
            # and the slope by its own derivative, which is 1/2 or less, times that
            pre = _valued((1 + signed.abs()) * pre, s * (1 + signed.abs() * (1 - s)) * (1 + signed.abs()) + pre / 2, pre)
        else:
            pre = pre * torch.sigmoid(pre)
    lengths = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    live = torch.stack([torch.arange(T) < v for v in lengths]).unsqueeze(-1) if B else torch.zeros(0, T, 1, dtype=torch.bool)
    return torch.where(live, pre, 0.0), torch.stack([rows[b, v:v + W - 1] for b, v in enumerate(lengths)])


def scan(u, delta, A, B, C, D, z, delta_bias, h0, lengths, softplus=True, magnitude=False):
    """B, C [batch, T, G, N]."""
    batch, T, n = u.shape
    N, share = A.shape[1], n // B.shape[2]
    live = torch.ones(batch, T, 1, dtype=torch.bool)
    if lengths is not None:
        live = torch.arange(T)[None, :, None] < lengths.cpu().long()[:, None, None]
    clean = lambda x, m: torch.where(m, x, 0.0)
    u, delta = clean(u, live), clean(delta, live)
    B, C = clean(B, live.unsqueeze(-1)), clean(C, live.unsqueeze(-1))
    raw = delta if delta_bias is None else delta + delta_bias
    dt = clean(torch.logaddexp(raw, torch.zeros_like(raw)) if softplus else raw, live)
    if magnitude:
        u, B, C = u.abs(), B.abs(), C.abs()
        D, h0 = None if D is None else D.abs(), None if h0 is None else h0.abs()
        size = _valued(dt.abs(), torch.ones_like(dt), dt)
    else:
        size = dt
    B, C = B.repeat_interleave(share, 2), C.repeat_interleave(share, 2)
    h = torch.zeros(batch, n, N, dtype=torch.float64) if h0 is None else h0
    y = []
    for t in range(T):
        x = dt[:, t, :, None] * A
        a = torch.exp(x)
        if magnitude:
            a = _valued(a, a * A.abs(), dt[:, t, :, None].expand_as(a)) + _valued(torch.zeros_like(a), a * dt[:, t, :, None].abs(), A.expand_as(a))
        h = a * h + (size[:, t] * u[:, t]).unsqueeze(-1) * B[:, t]
        y.append((h * C[:, t]).sum(-1))
    y = torch.stack(y, 1) if T else torch.zeros(batch, 0, n, dtype=torch.float64)
    if D is not None:
        y = y + D * u
    if z is not None:
        y = y * _silu(clean(z, live), magnitude)
    return clean(y, live), h


def residual(x, y, weight, post_weight, groups, gate, activation, scale, eps):
    if y is None:
        s = x
    else:
        t = y
        if post_weight is not None:
            t = t.unflatten(-1, (groups, -1))
            t = (t * (t.square().mean(-1, keepdim=True) + eps) ** -0.5).flatten(-2) * post_weight
        if gate is not None:
            t = t * (gate * torch.sigmoid(gate) if activation == "silu" else torch.sigmoid(gate))
        if scale is not None:
            t = t * scale
        s = t if x is None else x + t
    return s, None if weight is None else s * (s.square().mean(-1, keepdim=True) + eps) ** -0.5 * weight


def residual_sizes(x, y, weight, post_weight, groups, gate, activation, scale, eps, ds, dh):
    """Sums of absolute values of what the outputs and gradients are made of: (s, h, dx, dy, dgate, dweight, dpost_weight, dscale)."""
    base = x if y is None else y
    one = torch.ones_like(base)
    wide = lambda v: v.unflatten(-1, (groups, -1)).mean(-1, keepdim=True).expand(*v.shape[:-1], groups, v.shape[-1] // groups).flatten(-2)
    r1 = one if post_weight is None else (wide(y.square()) + eps) ** -0.5
    w1, k = one if post_weight is None else post_weight.abs(), one if scale is None else scale.abs()
    sig = None if gate is None else torch.sigmoid(gate)
    act = one if gate is None else (gate * sig).abs() if activation == "silu" else sig
    slope = one if gate is None else (sig * (1 + gate.abs() * (1 - sig))) if activation == "silu" else sig
    unit = torch.zeros_like(base) if y is None else (y * r1).abs()
    t = unit * w1 * act * k
    size = t + (0 if x is None else x.abs())
    s = residual(x, y, None, post_weight, groups, gate, activation, scale, eps)[0]
    out = [size]
    d = torch.zeros_like(base) if ds is None else ds.abs()
    w2 = one if weight is None else weight.abs()
    r2 = (s.square().mean(-1, keepdim=True) + eps) ** -0.5
    # r2 is off by what the parts of the row's sum of squares are
    grown = (size.square().mean(-1, keepdim=True) + eps) * r2 ** 2
    out.append(size * r2 * w2 * grown)
    dw2 = torch.zeros_like(base)
    if dh is not None:
        dh = dh.abs()
        d = d + r2 * grown * (dh * w2 + size * r2 ** 2 * (dh * w2 * size).mean(-1, keepdim=True))
        dw2 = dh * size * r2 * grown
    through = d * k * act
    c = through * w1
    dy = r1 * (c + unit * wide(c * unit)) if post_weight is not None else c
    rows = lambda v: v.sum((0, 1))
    return out + [d, dy, d * k * unit * w1 * slope, rows(dw2), rows(through * unit), rows(d * unit * w1 * act)]

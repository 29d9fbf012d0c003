"""The norms around a block with its gate and residual scale against the definition in 64 bits (GPU)."""
import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("x", "y", "weight", "post_weight", "gate", "scale")
ALL = ("x", "y", "weight", "post_weight", "gate", "scale")


def make(B, T, n, dtype, given, *, stream=None, weights=None, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    s = dict(x=(3 * r(B, T, n)).to(DT[stream or dtype]), y=r(B, T, n).to(DT[dtype]), weight=(1 + 0.2 * r(n)).to(DT[weights or dtype]),
             post_weight=(1 + 0.2 * r(n)).to(DT[weights or dtype]), gate=r(B, T, n).to(DT[dtype]), scale=(0.5 + 0.2 * r(n)).to(DT[weights or dtype]))
    return {k: s[k].cuda() if k in given else None for k in NAMES}


def call(s, groups=1, activation="silu", **kw):
    return vla.residual_norm(s["x"], s["y"], s["weight"], post_weight=s["post_weight"], groups=groups, gate=s["gate"], activation=activation,
                             scale=s["scale"], **kw)


# Roundings: a norm's sum of squares over up to 32 columns of a lane and its lanes (40), its root, the factors, and those of the sums that go into others
K = 256

CASES = [
    # B, T, n, dtype, what is given, groups, activation, stream, weights
    (1, 1, 8, "f32", ALL, 1, "silu", None, None),
    (2, 3, 64, "bf16", ALL, 2, "silu", None, None),
    (1, 5, 72, "f32", ALL, 1, "sigmoid", None, None),
    (3, 7, 264, "bf16", ALL, 1, "silu", "f32", None),
    (2, 9, 512, "f32", ("x", "y", "weight"), 1, "silu", None, None),
    (1, 33, 960, "bf16", ("y", "post_weight", "gate"), 10, "silu", None, "f32"),
    (2, 5, 1664, "f32", ("y", "post_weight", "gate"), 13, "silu", None, None),
    (2, 6, 1664, "bf16", ALL, 1, "sigmoid", "f32", "f32"),
    (1, 4, 2048, "f32", ALL, 2, "silu", None, None),
    (2, 3, 4096, "bf16", ("x", "y", "weight", "post_weight", "scale"), 1, "silu", "f32", None),
    (1, 3, 4104, "f32", ALL, 27, "silu", None, None),
    (1, 2, 8192, "bf16", ALL, 64, "silu", None, None),
    (1, 3, 5000, "f32", ALL, 1, "silu", None, None),
    (2, 2, 8192, "f32", ALL, 8, "sigmoid", None, None),
    (4, 50, 128, "bf16", ("x", "y", "gate", "scale", "weight"), 1, "silu", None, None),
    (4, 300, 96, "f32", ("x", "weight"), 1, "silu", None, None),
    (1, 700, 40, "bf16", ("x", "y", "post_weight"), 5, "silu", "f32", "f32"),
    (1, 6, 256, "f32", ("y", "gate"), 1, "sigmoid", None, None),
]


@pytest.mark.parametrize("B,T,n,dtype,given,groups,activation,stream,weights", CASES)
def test_outputs_and_gradients(B, T, n, dtype, given, groups, activation, stream, weights):
    s = make(B, T, n, dtype, given, stream=stream, weights=weights, seed=n + T)
    leaves = {k: None if v is None else ref.double(v).requires_grad_() for k, v in s.items()}
    args = (leaves["x"], leaves["y"], leaves["weight"], leaves["post_weight"], groups, leaves["gate"], activation, leaves["scale"], 1e-6)
    out = [o for o in ref.residual(*args) if o is not None]
    ours = {k: None if v is None else v.detach().requires_grad_() for k, v in s.items()}
    got = call(ours, groups, activation)
    assert (got[1] is None) == (s["weight"] is None) and (s["y"] is not None or got[0] is ours["x"])
    seen = [o for o in got if o is not None]
    grads = [torch.randn(B, T, n).to(o.dtype).cuda() for o in seen]
    names = [k for k in NAMES if s[k] is not None]
    want = torch.autograd.grad(out, [leaves[k] for k in names], [ref.double(g) for g in grads])
    found = torch.autograd.grad(seen, [ours[k] for k in names], grads)
    detached = [None if a is None or not torch.is_tensor(a) else a.detach() for a in args]
    sizes = ref.residual_sizes(*(a if torch.is_tensor(b) else b for a, b in zip(detached, args)), ref.double(grads[0]),
                               ref.double(grads[1]) if len(grads) > 1 else None)
    of = dict(zip(("s", "h", "x", "y", "gate", "weight", "post_weight", "scale"), sizes))
    for name, o, w in zip(("s", "h"), got, [ref.double(out[0]), ref.double(out[1]) if len(out) > 1 else None]):
        if o is not None and (name == "h" or s["y"] is not None):
            ref.close(o, w, of[name], K, name)
    for name, g, w in zip(names, found, want):
        # where y is missing autograd adds the gradient of s itself, in x's type
        k = K + (B * T if name in ("weight", "post_weight", "scale") else 0)
        extra = 2 ** 16 if s["y"] is None and g.dtype == torch.bfloat16 else 0
        ref.close(g, w, of[name], k + extra, "d" + name)


def test_a_single_gradient_given():
    """The gradient of s alone, that of h alone, and gradients of some inputs alone are the same numbers as those asked for together."""
    s = make(2, 5, 264, "bf16", ALL, seed=4)
    ds, dh = torch.randn(2, 5, 264).bfloat16().cuda(), torch.randn(2, 5, 264).bfloat16().cuda()
    zero = torch.zeros_like(ds)
    for a, b in ((ds, None), (None, dh)):
        how = dict(post_weight=s["post_weight"], gate=s["gate"], scale=s["scale"], groups=3)
        one = vla.residual_norm_backward(s["x"], s["y"], s["weight"], a, b, **how)
        both = vla.residual_norm_backward(s["x"], s["y"], s["weight"], zero if a is None else a, zero if b is None else b, **how)
        assert all(torch.equal(p, q) for p, q in zip(one, both))
    leaves = {k: v.detach().requires_grad_(k in ("y", "scale")) for k, v in s.items()}
    out = call(leaves, 3)
    dy, dscale = torch.autograd.grad(out, (leaves["y"], leaves["scale"]), (ds, dh))
    every = vla.residual_norm_backward(s["x"], s["y"], s["weight"], ds, dh, **how)
    assert torch.equal(dy, every[1]) and torch.equal(dscale, every[5])


def test_rows_of_zeros_and_infinities():
    """A row of zeros is divided by the root of eps; an infinite value or a NaN reaches its row alone."""
    s = make(1, 4, 256, "f32", ("x", "y", "weight", "post_weight"), seed=9)
    want = call(s)
    s["x"][0, 1], s["y"][0, 1] = 0, 0
    s["y"][0, 2, 5] = float("inf")
    s["x"][0, 3, 7] = float("nan")
    got = call(s)
    assert (got[0][0, 1] == 0).all() and (got[1][0, 1] == 0).all()
    assert torch.equal(got[0][0, 0], want[0][0, 0]) and torch.equal(got[1][0, 0], want[1][0, 0])
    assert torch.isnan(got[1][0, 3]).all() and torch.isnan(got[0][0, 3, 7]) and torch.isnan(got[0][0, 2, 5])


def test_views_and_a_norm_for_each_head():
    """The outputs of a recurrence as rows of heads, a gate that is a slice of a projection: read as they are."""
    B, H, T, d = 2, 3, 11, 32
    n = H * d
    o = torch.randn(B, T, H, d).bfloat16().cuda().transpose(1, 2)                 # as gated_delta returns it for values of that layout
    rows = torch.randn(B, T, 2 * n).bfloat16().cuda()
    w = (1 + 0.1 * torch.randn(d)).bfloat16().cuda()
    y = o.transpose(1, 2).reshape(B, T, n)
    s, h = vla.residual_norm(None, y, post_weight=w.repeat(H), groups=H, gate=rows[..., n:])
    assert h is None
    for i in range(H):
        one, _ = vla.residual_norm(None, o[:, i].contiguous(), post_weight=w, gate=rows[..., n + i * d:n + (i + 1) * d].contiguous())
        assert torch.equal(one, s[..., i * d:(i + 1) * d])
    swapped = y.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(vla.residual_norm(None, swapped, post_weight=w.repeat(H), groups=H, gate=rows[..., n:])[0], s)


def test_no_row():
    s = make(2, 0, 64, "f32", ALL)
    leaves = {k: v.detach().requires_grad_() for k, v in s.items()}
    out = call(leaves)
    assert out[0].shape == out[1].shape == (2, 0, 64)
    grads = torch.autograd.grad(out, list(leaves.values()), [torch.zeros_like(o) for o in out])
    assert all((g == 0).all() for g in grads)

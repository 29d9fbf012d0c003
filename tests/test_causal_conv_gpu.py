"""The short causal convolution against its definition in 64 bits: outputs, windows, gradients, one token (GPU)."""
import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("x", "weight", "bias", "state")


def make(B, T, n, W, dtype, *, weights=None, bias=True, carried=True, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    w = DT[weights or dtype]
    return dict(x=r(B, T, n).to(DT[dtype]).cuda(), weight=r(n, W).to(w).cuda(), bias=r(n).to(w).cuda() if bias else None,
                state=r(B, W - 1, n).to(DT[dtype]).cuda() if carried else None)


def references(s, lengths, silu, grads=None):
    both = []
    for magnitude in (False, True):
        leaves = {k: ref.double(s[k]) for k in NAMES}
        for k in leaves:
            if leaves[k] is not None:
                leaves[k].requires_grad_()
        out = ref.conv(*(leaves[k] for k in NAMES), lengths, silu, magnitude)
        got = [x.detach() for x in out]
        if grads is not None:
            d = [ref.double(g).abs() if magnitude else ref.double(g) for g in grads]
            names = [k for k in NAMES if leaves[k] is not None]
            back = torch.autograd.grad(out, [leaves[k] for k in names], d, allow_unused=True)
            got += [(torch.zeros_like(leaves[k]) if g is None else g) for k, g in zip(names, back)]
        both.append([g.abs() if magnitude else g for g in got])
    return both


CASES = [
    # B, T, n, width, dtype, weights, silu, options
    (1, 1, 8, 2, "f32", None, True, {}),
    (2, 2, 64, 4, "bf16", None, True, {}),
    (3, 7, 72, 3, "f32", None, False, {}),
    (1, 8, 136, 4, "bf16", "f32", True, dict(carried=False)),
    (2, 17, 264, 4, "f32", None, True, dict(bias=False)),
    (1, 131, 64, 2, "bf16", None, False, dict(bias=False, carried=False)),
    (2, 200, 520, 3, "bf16", None, True, {}),
    (1, 300, 40, 4, "f32", "bf16", True, {}),
    (3, 300, 72, 4, "bf16", None, True, {}),          # runs of the same channels in a workgroup, not all as often
    (2, 500, 1024, 2, "bf16", None, True, {}),        # twice each
    (2, 50, 1032, 3, "bf16", None, True, {}),         # and not
]


@pytest.mark.parametrize("B,T,n,W,dtype,weights,silu,options", CASES)
def test_outputs_and_gradients(B, T, n, W, dtype, weights, silu, options):
    s = make(B, T, n, W, dtype, weights=weights, seed=T + n, **options)
    grads = [torch.randn(B, T, n).to(DT[dtype]).cuda(), torch.randn(B, W - 1, n).to(DT[dtype]).cuda()]
    act = "silu" if silu else None
    want, size = references(s, None, silu, grads)
    leaves = {k: x if x is None else x.detach().requires_grad_() for k, x in s.items()}
    out = vla.causal_conv(leaves["x"], leaves["weight"], leaves["bias"], leaves["state"], activation=act)
    got = [*out, *torch.autograd.grad(out, [x for x in leaves.values() if x is not None], grads)]
    names = ["y", "state_T", *("d" + k for k in NAMES if s[k] is not None)]
    for name, g, w, m in zip(names, got, want, size):
        # the taps, the bias and the activation (12); the second rounding of the slope; a sum over tokens one after the other
        ref.close(g, w, m, 2 * W + 24 + (B * T if name in ("dweight", "dbias") else 0), name)
    plain = vla.causal_conv(s["x"], s["weight"], s["bias"], s["state"], activation=act)
    assert all(torch.equal(a, b) for a, b in zip(plain, out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_lengths(dtype, W):
    B, T, n = 8, 40, 72
    s = make(B, T, n, W, dtype, seed=W)
    given = torch.tensor([40, 0, 1, 2, 3, 17, 90, -1], dtype=torch.int32)
    lengths = given.clamp(0, T)
    grads = [torch.randn(B, T, n).to(DT[dtype]).cuda(), torch.randn(B, W - 1, n).to(DT[dtype]).cuda()]
    want, size = references(s, lengths, True, grads)
    for b in range(B):
        s["x"][b, lengths[b]:] = float("nan")
        grads[0][b, lengths[b]:] = float("inf")
    y, state_T = vla.causal_conv(s["x"], s["weight"], s["bias"], s["state"], lengths=given.cuda())
    got = [y, state_T, *vla.causal_conv_backward(s["x"], s["weight"], s["bias"], s["state"], *grads, lengths=given.cuda())]
    for i, (g, w, m) in enumerate(zip(got, want, size)):
        ref.close(g, w, m, 2 * W + 24 + (B * T if i in (3, 4) else 0), str(i))
    for b in range(B):
        assert (got[0][b, lengths[b]:] == 0).all() and (got[2][b, lengths[b]:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_one_token_at_a_time_and_pieces(dtype, W):
    """Token by token, and in pieces of 1, 2, 13 and the other tokens: the same bits as the whole sequence."""
    B, T, n = 2, 30, 64
    s = make(B, T, n, W, dtype, seed=7)
    y, last = vla.causal_conv(s["x"], s["weight"], s["bias"], s["state"])
    state = s["state"].clone()
    for t in range(T):
        assert torch.equal(vla.causal_conv_step(s["x"][:, t], s["weight"], state, s["bias"]), y[:, t])
    assert torch.equal(state, last)
    state, at = s["state"], 0
    for piece in (1, 2, 13, 14):
        out, state = vla.causal_conv(s["x"][:, at:at + piece], s["weight"], s["bias"], state)
        assert torch.equal(out, y[:, at:at + piece])
        at += piece
    assert torch.equal(state, last)


def test_no_token():
    s = make(2, 0, 64, 4, "bf16")
    leaves = {k: x.detach().requires_grad_() for k, x in s.items()}
    y, state = vla.causal_conv(*leaves.values())
    assert y.shape == (2, 0, 64) and torch.equal(state, s["state"])
    g = torch.randn_like(state)
    dstate, dw = torch.autograd.grad(state, (leaves["state"], leaves["weight"]), g)
    assert torch.equal(dstate, g) and (dw == 0).all()
    assert (vla.causal_conv(s["x"], s["weight"])[1] == 0).all()


def test_views():
    """A slice of a fused projection and a sequence-major one are read as they are; other layouts are copied."""
    B, T, n = 2, 21, 64
    s = make(B, T, n, 4, "bf16", seed=3)
    want = vla.causal_conv(*s.values())
    wide = torch.randn(B, T, 3 * n).bfloat16().cuda()
    wide[..., n:2 * n] = s["x"]
    odd = torch.empty(B, T, n + 2, dtype=torch.bfloat16, device="cuda")[..., 1:-1]
    odd.copy_(s["x"])
    for x in (wide[..., n:2 * n], s["x"].transpose(0, 1).contiguous().transpose(0, 1), s["x"].transpose(1, 2).contiguous().transpose(1, 2), odd):
        assert all(torch.equal(a, b) for a, b in zip(vla.causal_conv(x, s["weight"].t().contiguous().t(), s["bias"], s["state"]), want))


def test_heads_before_a_recurrence():
    """The convolution over the fused queries, keys and values, whose heads go on to the norm and the gated delta rule as views."""
    B, T, H, d = 2, 40, 2, 32
    s = make(B, T, 3 * H * d, 4, "bf16", seed=1)
    y, _ = vla.causal_conv(*s.values())
    q, k, v = (x.view(B, T, H, d).transpose(1, 2) for x in y.split(H * d, -1))
    q, k = vla.qk_norm_rope(q, k, norm="l2")
    g, beta = -torch.rand(B, H, T, device="cuda"), torch.rand(B, H, T, device="cuda")
    o, _ = vla.gated_delta(q, k, v, g, beta)
    dense = vla.gated_delta(q, k, v.contiguous(), g, beta)[0]
    assert torch.equal(o, dense)

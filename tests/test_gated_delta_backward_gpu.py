"""Gradients of the gated delta rule against autograd through the token-by-token recurrence in float64, and against differences (GPU).

Tolerances, of the largest value of a head: products and states are float32 throughout, so that dS0, dbeta and float32 dq, dk, dv are off
by some roundings of 2^-24 times the few products that they pass: 2e-5.  dg is the difference of sums over up to 256 tokens, each term off by
about 1e-7 of terms that can be some times larger than dg: 1e-4.  bfloat16 dq, dk, dv: one rounding (2^-9) on top of products of 16-bit
parts: 6e-3."""
import pytest
import torch

import paper_2605_11196_amd as vla
from test_gated_delta_gpu import DT, close, make, oracle

pytestmark = pytest.mark.gpu
ROUNDED = {"f32": 2e-5, "bf16": 6e-3}
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dS0")
LIMIT = {"dg": 1e-4, "dbeta": 2e-5, "dS0": 2e-5}


def grads(inputs, dtype, seed, *, with_state=True, **kw):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    q, k, v, g, beta, S0 = inputs
    do = torch.randn(v.shape, generator=gen, device="cuda").to(DT[dtype])
    dS = torch.randn((v.shape[0], v.shape[1], v.shape[3], q.shape[3]), generator=gen, device="cuda") * 0.3 if with_state else None
    segments = kw.pop("segments", 0)
    o, S, saved = vla.gated_delta_forward(*inputs, save_for_backward=True, segments=segments, **kw)
    got = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS, segments=segments, **kw)
    leaves = [x.double().requires_grad_() for x in inputs if x is not None]
    ro, rS = oracle(*leaves, *([None] if S0 is None else []), scale=kw.get("scale"), lengths=kw.get("lengths"))
    outs = (ro, rS) if with_state else (ro,)
    want = torch.autograd.grad(outs, leaves, (do.double(), dS.double()) if with_state else (do.double(),), allow_unused=True)
    want = [torch.zeros_like(x) if w is None else w for w, x in zip(want, leaves)]
    return (o, S), (ro.detach(), rS.detach()), got, want


def check(inputs, dtype, seed=1, **kw):
    out, ref, got, want = grads(inputs, dtype, seed, **kw)
    close(out[1], ref[1], 1e-5, "S_T")
    for name, x, y in zip(NAMES, got, want):
        if name in ("dg", "dbeta"):
            x, y = x.unsqueeze(-1), y.unsqueeze(-1)
        close(x, y, LIMIT.get(name, ROUNDED[dtype]), name)
    return out, got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 16, 17, 31, 32, 33, 64, 65, 255, 256, 257, 300])
def test_lengths_around_the_blocks(T, dtype):
    check(make(2, 2, 2, T, 64, 64, dtype, seed=T), dtype, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_v", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("d_k", [16, 32, 64, 96, 128])
def test_head_sizes(d_k, d_v, dtype):
    check(make(1, 2, 2, 75, d_k, d_v, dtype, seed=d_k + 3 * d_v), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H_k,H_v", [(1, 4), (2, 6)])
def test_shared_key_heads(H_k, H_v, dtype):
    check(make(2, H_k, H_v, 70, 32, 64, dtype, seed=H_v, carried=False), dtype, scale=0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H_k", [2, 4])
def test_ragged_lengths(H_k, dtype):
    T = 300
    inputs = make(6, H_k, 4, T, 32, 64, dtype, seed=8)
    lengths = torch.tensor([0, 1, 40, 256, 290, T], device="cuda", dtype=torch.int32)
    out, got = check(inputs, dtype, lengths=lengths)
    for b, n in enumerate(lengths.tolist()):
        for x in got[:5]:
            assert (x[b, :, n:] == 0).all()
    q, k, v, g, beta, S0 = (x.clone() for x in inputs)
    for b, n in enumerate(lengths.tolist()):
        for x in (q, k, v, g, beta):
            x[b, :, n:] = float("nan")
    out2, _, got2, _ = grads((q, k, v, g, beta, S0), dtype, 1, lengths=lengths)
    assert all(torch.equal(x, y) for x, y in zip((*out, *got), (*out2, *got2)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_that_forget_and_no_state(dtype):
    q, k, v, g, beta, _ = make(2, 2, 2, 90, 32, 32, dtype, seed=11, rate=2.0, carried=False)
    g[0, 0] = 0
    g[1, 0, 5:20] = -60.0
    beta[0, 0, ::3] = 0
    beta[1, 1, ::5] = 2
    check((q, k, v, g, beta, None), dtype, with_state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_forgotten_state_has_no_gradient(dtype):
    q, k, v, g, beta, S0 = make(1, 1, 1, 50, 32, 32, dtype, seed=3)
    g[0, 0, 40] = float("-inf")
    _, _, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, save_for_backward=True)
    got = vla.gated_delta_backward(q, k, v, g, beta, saved, torch.randn_like(v), None)
    assert all(torch.isfinite(x).all() for x in got)
    cut = tuple(x[:, :, 40:] for x in (q, k, v, g, beta))
    zeroed = g.clone()
    zeroed[0, 0, 40] = 0
    do = torch.randn_like(v)
    got = vla.gated_delta_backward(q, k, v, g, beta, saved, do, None)
    _, _, saved2 = vla.gated_delta_forward(cut[0], cut[1], cut[2], zeroed[:, :, 40:], cut[4], None, save_for_backward=True)
    alone = vla.gated_delta_backward(cut[0], cut[1], cut[2], zeroed[:, :, 40:], cut[4], saved2, do[:, :, 40:], None)
    close(got[0][:, :, 40:], alone[0].double(), ROUNDED[dtype], "dq after the cut")
    close(got[2][:, :, 40:], alone[2].double(), ROUNDED[dtype], "dv after the cut")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_keys(dtype):
    q, k, v, g, beta, S0 = make(1, 2, 2, 100, 64, 64, dtype, seed=12)
    k = k[:, :, :1].expand_as(k).contiguous()
    check((q, k, v, torch.zeros_like(g), torch.full_like(beta, 0.9), S0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_k,d_v,T,segments", [(16, 32, 200, 3), (64, 64, 700, 5), (128, 64, 300, 4), (96, 128, 520, 8)])
def test_time_segments(d_k, d_v, T, segments, dtype):
    inputs = make(2, 1, 2, T, d_k, d_v, dtype, seed=T, rate=0.05)
    lengths = torch.tensor([T, T // 2 + 3], device="cuda", dtype=torch.int32)
    check(inputs, dtype, segments=segments, lengths=lengths)


def test_against_differences():
    """Central differences of the float64 oracle along random directions: their own error is about 1e-8 at a step of 1e-4."""
    inputs = make(1, 1, 2, 40, 16, 32, "f32", seed=21)
    q, k, v, g, beta, S0 = inputs
    do, dS = torch.randn_like(v), torch.randn_like(S0)
    _, _, saved = vla.gated_delta_forward(*inputs, save_for_backward=True)
    got = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS)

    def loss(args):
        o, S = oracle(*args)
        return (o * do.double()).sum() + (S * dS.double()).sum()

    for i, name in enumerate(NAMES):
        u = torch.randn(inputs[i].shape, device="cuda", dtype=torch.float64)
        u /= u.norm()
        args = [x.double() for x in inputs]
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-4 * u, args[i] - 1e-4 * u
        want = (loss(up) - loss(down)) / 2e-4
        assert abs((got[i].double() * u).sum() - want) <= 1e-4 * max(abs(want), got[i].double().norm() * 0.1), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_autograd_strides_and_repeatability(dtype):
    B, H_k, H_v, T, d_k, d_v = 2, 2, 4, 90, 64, 32
    q, k, v, g, beta, S0 = make(B, H_k, H_v, T, d_k, d_v, dtype, seed=30)
    do, dS = torch.randn_like(v), torch.randn_like(S0)
    _, _, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, save_for_backward=True)
    want = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS)
    rows = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    leaves = [x.detach().requires_grad_() for x in (rows(q), rows(k), rows(v), rows(g[..., None])[..., 0], beta, S0)]
    for _ in range(2):
        o, S = vla.gated_delta(*leaves)
        got = torch.autograd.grad((o, S), leaves, (rows(do), dS))
        for name, x, y in zip(NAMES, got, want):
            assert torch.equal(x, y), name
        assert got[2].stride() == leaves[2].stride()
    o, _ = vla.gated_delta(*leaves[:5])
    (o.float().sum()).backward()
    assert leaves[0].grad is not None and leaves[5].grad is None


def test_no_tokens():
    q, k, v, g, beta, S0 = make(2, 1, 2, 0, 32, 32, "f32", seed=1)
    _, _, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, save_for_backward=True)
    dS = torch.randn_like(S0)
    got = vla.gated_delta_backward(q, k, v, g, beta, saved, v, dS)
    assert torch.equal(got[5], dS)

"""Norm of queries and keys with the position rotation against the formula in float64 (GPU).

Tolerances: float32 arithmetic on up to 128 columns with one rounding at the end.  float32 outputs: the sum of squares, the reciprocal
root, three products and the turn are about ten roundings of 2^-24, so 2e-6 of the row's largest value holds with room.  bfloat16: half a
unit in the last place of a value, 2^-8 of it at most (2^-9 in the mean), with the float32 error far below: 2^-8 of the row's largest value.  Weight
gradients add up N rows in float32, parts of at most some thousand rows at a time: 1e-5 of the largest."""
import pytest
import torch

import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 2e-6, "bf16": 2.0 ** -8}


def tables(places, rot, base=10000.0):
    angle = torch.arange(places, dtype=torch.float64)[:, None] * base ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def oracle(x, w, cos, sin, place, *, eps, l2, interleaved):
    """float64; x [B,H,T,d], place [B,T] or None without a rotation"""
    x = x.double()
    n = 1 if l2 else x.shape[-1]
    y = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / n + eps)
    if w is not None:
        y = y * w.double()
    if cos is None:
        return y
    c, s = cos.double()[place][:, None], sin.double()[place][:, None]
    rot = 2 * cos.shape[1]
    first = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    second = first + 1 if interleaved else first + rot // 2
    z = y.clone()
    z[..., first] = y[..., first] * c - y[..., second] * s
    z[..., second] = y[..., first] * s + y[..., second] * c
    return z


def close(got, want, tol, what):
    assert got.shape == want.shape
    err = ((got.double() - want).abs().amax(-1) / want.abs().amax(-1).clamp_min(1e-30)).max().item() if want.numel() else 0.0
    assert err <= tol, (what, err)


def make(B, T, H_q, H_k, d, dtype, seed, fused=True):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows = torch.randn((B, T, (H_q + 2 * H_k) * d), generator=gen, device="cuda").to(DT[dtype])
    q = rows[..., :H_q * d].view(B, T, H_q, d).transpose(1, 2)
    k = rows[..., H_q * d:(H_q + H_k) * d].view(B, T, H_k, d).transpose(1, 2)
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    wq, wk = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    dq, dk = (torch.randn((B, H, T, d), generator=gen, device="cuda").to(DT[dtype]) for H in (H_q, H_k))
    return q, k, wq, wk, dq, dk


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot,interleaved,l2", [(16, 16, False, False), (16, 8, True, True), (32, 16, False, True), (64, 64, True, False),
                                                  (96, 96, False, False), (96, 48, True, True), (96, 24, False, False), (128, 128, False, True),
                                                  (128, 32, True, False), (128, 0, False, False)])
@pytest.mark.parametrize("B,T,H_q,H_k", [(2, 37, 6, 3), (5, 1, 4, 1)])
def test_forward_and_gradients(B, T, H_q, H_k, d, rot, interleaved, l2, dtype):
    q, k, wq, wk, dq, dk = make(B, T, H_q, H_k, d, dtype, seed=d + rot + T)
    cos, sin = tables(T + 20, rot) if rot else (None, None)
    how = dict(eps=1e-5, norm="l2" if l2 else "rms", interleaved=interleaved, offset=3)
    place = (torch.arange(T, device="cuda") + 3)[None].expand(B, T)
    leaves = [x.detach().requires_grad_() for x in (q, k, wq, wk)]
    out = vla.qk_norm_rope(*leaves, cos, sin, **how)
    grads = torch.autograd.grad(out, leaves, (dq, dk))
    ref_leaves = [x.detach().double().requires_grad_() for x in (q, k, wq, wk)]
    ref = [oracle(x, w, cos, sin, place, eps=1e-5, l2=l2, interleaved=interleaved) for x, w in ((ref_leaves[0], ref_leaves[2]), (ref_leaves[1], ref_leaves[3]))]
    want = torch.autograd.grad(ref, ref_leaves, (dq.double(), dk.double()))
    for i, name in enumerate(("q", "k")):
        assert out[i].is_contiguous() and out[i].dtype == DT[dtype]
        close(out[i], ref[i].detach(), TOL[dtype], name)
        close(grads[i], want[i], 4 * TOL[dtype] if dtype == "f32" else TOL[dtype], "d" + name)   # the projection cancels up to a few times
        close(grads[2 + i], want[2 + i], 1e-5, "dw" + name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(dtype):
    """(f(x + h) - f(x - h)) / 2h of the oracle along random directions: its own error is h^2 / 6 f''' + 1e-16 / h, about 1e-9 at h = 1e-4."""
    q, k, wq, wk, dq, dk = make(1, 5, 2, 1, 32, "f32", seed=9)
    cos, sin = tables(5, 32)
    place = torch.arange(5, device="cuda")[None]
    f = lambda x, w: (oracle(x, w, cos, sin, place, eps=1e-6, l2=False, interleaved=False) * dq.double()).sum()
    got = vla.qk_norm_rope_backward(q, k, wq, wk, cos, sin, dq, dk)
    for i in range(4):
        u, w = torch.randn(q.shape, device="cuda", dtype=torch.float64), torch.randn(wq.shape, device="cuda", dtype=torch.float64)
        h = 1e-4
        along_x = (f(q.double() + h * u, wq) - f(q.double() - h * u, wq)) / (2 * h)
        along_w = (f(q.double(), wq.double() + h * w) - f(q.double(), wq.double() - h * w)) / (2 * h)
        assert abs((got[0].double() * u).sum() - along_x) <= 1e-5 * (got[0].double().norm() * u.norm())
        assert abs((got[2].double() * w).sum() - along_w) <= 1e-5 * (got[2].double().norm() * w.norm())


def test_positions_per_sequence_and_outside_the_tables():
    q, k, wq, wk, dq, dk = make(3, 4, 2, 2, 64, "f32", seed=3)
    cos, sin = tables(50, 64)
    place = torch.tensor([[0, 49, 7, 7], [1, 2, 3, 4], [30, 20, 10, 0]], device="cuda", dtype=torch.int32)
    out = vla.qk_norm_rope(q, k, wq, wk, cos, sin, positions=place)
    close(out[0], oracle(q, wq, cos, sin, place.long(), eps=1e-6, l2=False, interleaved=False), TOL["f32"], "q")
    bad = place.clone()
    bad[1, 2], bad[2, 0] = -1, 50
    out2 = vla.qk_norm_rope(q, k, wq, wk, cos, sin, positions=bad)
    for a, b in zip(out, out2):
        gone = torch.isnan(b).all(-1)
        assert gone[1, :, 2].all() and gone[2, :, 0].all() and gone.sum() == 2 * b.shape[1]
        assert torch.equal(a[~gone], b[~gone])


def test_zero_rows_and_no_tokens():
    q, k, wq, wk, dq, dk = make(2, 3, 2, 1, 16, "f32", seed=4)
    q = q.clone()
    q[0, 1, 2] = 0
    out = vla.qk_norm_rope(q, k)
    assert (out[0][0, 1, 2] == 0).all()
    g = vla.qk_norm_rope_backward(q, k, None, None, None, None, dq, dk)
    want = dq[0, 1, 2].double() * 1e6 ** 0.5     # eps alone: the reciprocal root of 1e-6
    assert ((g[0][0, 1, 2].double() - want).abs() <= 1e-6 * want.abs()).all() and g[2] is None and g[3] is None
    empty = vla.qk_norm_rope(q[:, :, :0], k[:, :, :0], wq, wk)
    assert empty[0].shape == (2, 2, 0, 16)
    dx = vla.qk_norm_rope_backward(q[:, :, :0], k[:, :, :0], wq, wk, None, None, dq[:, :, :0], dk[:, :, :0])
    assert (dx[2] == 0).all() and (dx[3] == 0).all()


def test_strides_weights_in_bfloat16_and_repeatability():
    q, k, wq, wk, dq, dk = make(3, 300, 5, 2, 128, "bf16", seed=5)
    cos, sin = tables(300, 128)
    place = torch.arange(300, device="cuda")[None].expand(3, 300)
    wq16, wk16 = wq.bfloat16(), wk.bfloat16()
    a = vla.qk_norm_rope(q, k, wq16, wk16, cos, sin)
    b = vla.qk_norm_rope(q.contiguous(), k.contiguous(), wq16.float(), wk16.float(), cos, sin)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    odd = torch.randn(3, 5, 300, 130, device="cuda").bfloat16()[..., 1:129]     # rows that are not 16-byte aligned
    c = vla.qk_norm_rope(odd, k, None, None, cos, sin)
    close(c[0], oracle(odd, None, cos, sin, place, eps=1e-6, l2=False, interleaved=False), TOL["bf16"], "odd")
    repeated = q[:1].expand(3, -1, -1, -1)      # a batch that repeats one sequence
    r = vla.qk_norm_rope(repeated, k, wq16, wk16, cos, sin)
    assert torch.equal(r[0][2], a[0][0])
    g1 = vla.qk_norm_rope_backward(q, k, wq16, wk16, cos, sin, dq, dk)
    g2 = vla.qk_norm_rope_backward(q, k, wq16, wk16, cos, sin, dq.transpose(1, 2).contiguous().transpose(1, 2), dk)
    assert all(torch.equal(x, y) for x, y in zip(g1, g2))


def test_runs_on_the_given_stream():
    q, k, wq, wk, _, _ = make(2, 64, 4, 2, 64, "bf16", seed=6)
    want = vla.qk_norm_rope(q, k, wq, wk)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = vla.qk_norm_rope(q, k, wq, wk, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

"""Infinite values that a formula does not let reach a result: 0 times them, which is no number, must not come from tokens, terms or norms that are not
there (GPU)."""
import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("T,last", [(16, 15), (13, 12), (16, 9)])
def test_the_rates_gradient_where_the_last_state_overflows(dtype, N, T, last):
    """The last token's input takes the state past float32: dA is a sum of g_t a_t h_{t-1} dt_t, none of which has that state in it.  The blocks that the kernel goes
    through end behind the sequence's last token, at it, or at the tensor's end."""
    n = 72
    gen = torch.Generator().manual_seed(N + T)
    r = lambda *s: torch.randn(s, generator=gen)
    s = dict(u=r(2, T, n), delta=torch.rand((2, T, n), generator=gen), B=1 + torch.rand((2, T, 1, N), generator=gen), C=r(2, T, 1, N))
    s = {k: v.to(DT[dtype]) for k, v in s.items()}
    s["u"][:, last], s["delta"][:, last] = 3e38, 4.0
    A, h0, dh = -torch.rand((n, N), generator=gen) - 0.1, r(2, n, N), r(2, n, N)
    dy = r(2, T, n).to(DT[dtype])
    lengths = torch.full((2,), last + 1, dtype=torch.int32)
    both = []
    for magnitude in (False, True):
        a = A.double().requires_grad_()
        d = [x.double() for x in (dy, dh)]
        d[0][:, last + 1:] = 0
        out = ref.scan(*(s[k].double() if k in s else a if k == "A" else h0.double() if k == "h0" else None
                         for k in ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "h0")), lengths, False, magnitude)
        both.append(torch.autograd.grad(out, a, [x.abs() if magnitude else x for x in d])[0].abs() if magnitude
                    else torch.autograd.grad(out, a, d)[0])
    args = [s[k].cuda() if k in s else A.cuda() for k in ("u", "delta", "A", "B", "C")]
    y, h_T, saved = vla.selective_scan_forward(*args, None, None, h0.cuda(), softplus=False, lengths=lengths.cuda(), save_for_backward=True)
    assert torch.isinf(h_T).all()
    dA = vla.selective_scan_backward(*args, None, None, saved, dy.cuda(), dh.cuda(), softplus=False, lengths=lengths.cuda())[2]
    # as for the scan's other tests: 48 roundings a token, the sums over tokens and sequences
    ref.close(dA, *both, 48 * T + 64 + 2 * T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinite_input_without_a_skip(dtype):
    """Without D the read-out is C . h alone, which has a sign where B and C do: over a sequence as token by token."""
    n, N, T = 64, 16, 11
    gen = torch.Generator().manual_seed(3)
    u, delta = (torch.randn((1, T, n), generator=gen).to(DT[dtype]).cuda() for _ in range(2))
    B, C = (1 + torch.rand((1, T, N), generator=gen).to(DT[dtype]).cuda() for _ in range(2))
    A = -torch.rand((n, N), generator=gen).cuda()
    u[0, 4, 5] = float("inf")
    z = torch.ones_like(u)
    y, h = vla.selective_scan(u, delta, A, B, C, None, z)
    assert (y[0, 4:, 5] == float("inf")).all() and (h[0, 5] == float("inf")).all()
    state = torch.zeros(1, n, N, device="cuda")
    for t in range(T):
        one = vla.selective_scan_step(u[:, t], delta[:, t], A, B[:, t], C[:, t], state, None, z[:, t])
        assert torch.equal(torch.isinf(one), torch.isinf(y[:, t])) and not torch.isnan(one).any(), t
    # the gate's gradient is the sign of dy times that, the input's dt times sum g B, which is finite
    _, _, saved = vla.selective_scan_forward(u, delta, A, B, C, None, z, save_for_backward=True)
    grads = vla.selective_scan_backward(u, delta, A, B, C, None, z, saved, torch.ones_like(u))
    assert (grads[6][0, 4:, 5] == float("inf")).all() and torch.isfinite(grads[0]).all()
    dy = torch.ones_like(u)
    dy[0, 6, 9] = float("inf")
    grads = vla.selective_scan_backward(u, delta, A, B, C, None, z, saved, dy)
    assert (grads[0][0, :7, 9] == float("inf")).all() and not torch.isnan(grads[0]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [64, 1536, 4096])
def test_an_infinite_output_of_a_block_without_its_norm(dtype, n):
    """s = x + scale y: dy is scale ds, whatever y is."""
    gen = torch.Generator().manual_seed(n)
    x, y, ds = (torch.randn((1, 5, n), generator=gen).to(DT[dtype]).cuda() for _ in range(3))
    scale = (0.5 + torch.rand(n, generator=gen)).to(DT[dtype]).cuda()
    y[0, 2, 7], y[0, 3, 9] = float("inf"), float("nan")
    dx, dy, *_ = vla.residual_norm_backward(x, y, None, ds, None, scale=scale)
    assert torch.equal(dx, ds) and torch.equal(dy, (ds.float() * scale.float()).to(DT[dtype]))

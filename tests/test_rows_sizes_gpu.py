"""The operators on rows of channels at sizes where their kernels go round a loop again: more columns than a launch holds work-items for, more rows than
workgroups, more segments than are joined at once, long runs of tokens (GPU)."""
import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- more columns of a weight's gradient than workgroups of 64 in a launch

def test_gradients_of_2_28_rates():
    """One token of 2^22 channels with 64 states: dA = (e C + dh) exp(dt A) h0 dt, here with e = C = 0."""
    n, N = 2 ** 22, 64
    u = torch.ones(1, 1, n, device="cuda", dtype=torch.bfloat16)
    B = torch.zeros(1, 1, N, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    A, h0, dh = (torch.rand((1, n, N), generator=gen, device="cuda") - shift for shift in (1.5, 0.5, 0.5))
    args = u, 0.5 * u, A[0], B, B
    _, _, saved = vla.selective_scan_forward(*args, None, None, h0, softplus=False, save_for_backward=True)
    dA = vla.selective_scan_backward(*args, None, None, saved, u, dh, softplus=False)[2]
    for at in range(0, n, 2 ** 18):
        rows = slice(at, at + 2 ** 18)
        a, h, d = (x.reshape(n, N)[rows].double() for x in (A, h0, dh))
        want = d * torch.exp(0.5 * a) * h * 0.5
        # the rate times log2(e), the step, the exponential (its argument is below 2), three products
        assert ((dA[rows].double() - want).abs() <= 12 * ref.UNIT * want.abs() + 1e-37).all(), at


def test_gradients_of_2_28_channels_taps():
    """One token without a state: the last tap's gradient is dy x, the other one's 0, the bias's dy, each rounded once."""
    n = 2 ** 28
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn((1, 1, n), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    weight, bias = torch.ones(n, 2, device="cuda", dtype=torch.bfloat16), torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    dx, dweight, dbias, _ = vla.causal_conv_backward(x, weight, bias, None, dy, activation=None)
    assert torch.equal(dx, dy) and torch.equal(dbias, dy[0, 0])
    assert not dweight[:, 0].any() and torch.equal(dweight[:, 1], (dy[0, 0].float() * x[0, 0].float()).bfloat16())

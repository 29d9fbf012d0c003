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

"""Gradients of the gated delta rule where decays are strong or forget the state (GPU).

A token whose decay is 0 cuts a sequence in two: nothing passes it.  The gradients on either side are those of the parts alone, with the tolerances of
test_gated_delta_backward_gpu.py.

dg of a token is a difference of sums, of dO_i . O_i - v_i . dV_i over the tokens up to the next multiple of 256, and of <dS, S> there: off by the float32
rounding of these terms.  O, dV, S and dS are off by some roundings of 2^-24 of their size, 1e-6 with room, so dg by 1e-6 of the sum of the products'
absolute values, whatever dg itself is."""
import pytest
import torch

import paper_2605_11196_amd as vla
from test_gated_delta_backward_gpu import LIMIT, ROUNDED
from test_gated_delta_gpu import close, make, oracle

pytestmark = pytest.mark.gpu
FORGET = (float("-inf"), -20000.0, -110.0)      # below the clamp of the block kernels; no float32 number holds exp(-110)


def run(q, k, v, g, beta, S0, do, dS, segments):
    _, _, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, segments=segments, save_for_backward=True)
    return vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS, segments=segments)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("forget", FORGET)
@pytest.mark.parametrize("cut,segments", [(40, 1), (32, 3), (47, 1), (256, 1), (255, 5), (300, 5), (511, 0), (599, 1)])
def test_nothing_passes_a_token_that_forgets_the_state(cut, segments, forget, dtype):
    T = 600
    q, k, v, g, beta, S0 = make(1, 1, 2, T, 64, 64, dtype, seed=cut, rate=0.02)
    g[:, :, cut] = forget
    do, dS = torch.randn_like(v), torch.randn_like(S0)
    got = run(q, k, v, g, beta, S0, do, dS, segments)
    head = lambda x: x[:, :, :cut].contiguous()
    tail = lambda x: x[:, :, cut:].contiguous()
    before = run(head(q), head(k), head(v), head(g), head(beta), S0, head(do), None, 1)
    g0 = tail(g)
    g0[:, :, 0] = 0
    after = run(tail(q), tail(k), tail(v), g0, tail(beta), None, tail(do), dS, 1)
    for i, name in enumerate(("dq", "dk", "dv", "dbeta")):
        at = i if i < 3 else 4
        limit = 2 * LIMIT.get(name, ROUNDED[dtype])       # both sides are off
        last = (lambda x: x) if i < 3 else (lambda x: x.unsqueeze(-1))
        close(last(head(got[at])), last(before[at]).double(), limit, name + " before")
        close(last(tail(got[at])), last(after[at]).double(), limit, name + " after")
    close(got[5], before[5].double(), 2 * LIMIT["dS0"], "dS0")
    assert (got[3][:, :, cut] == 0).all()
    # a loss of the part behind the cut alone
    do[:, :, :cut] = 0
    got = run(q, k, v, g, beta, S0, do, dS, segments)
    for i in range(5):
        assert (head(got[i]) == 0).all(), i
    assert (got[5] == 0).all() and (got[3][:, :, cut] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rate", [0.01, 1.0, 5.0])
def test_the_gradient_of_a_decay_by_what_it_is_formed_from(rate, dtype):
    T, piece = 600, 256
    inputs = make(2, 1, 2, T, 32, 64, dtype, seed=int(100 * rate), rate=rate)
    inputs[3][0, 0, ::50] *= 20
    do, dS = torch.randn_like(inputs[2]), torch.randn_like(inputs[5])
    got = run(*inputs, do, dS, 0)[3]
    q, k, v, g, beta, S = (x.double().requires_grad_() for x in inputs)
    outs, states = [], []
    for first in range(0, T, piece):
        part = slice(first, first + piece)
        o, S = oracle(q[:, :, part], k[:, :, part], v[:, :, part], g[:, :, part], beta[:, :, part], S)
        outs.append(o)
        states.append(S)
    o = torch.cat(outs, 2)
    dv, dg, *dstates = torch.autograd.grad((o, S), (v, g, *states), (do.double(), dS.double()))
    reads = ((do.double() * o).abs() + (v * dv).abs()).sum(-1).detach()
    for i, first in enumerate(range(0, T, piece)):
        part = slice(first, min(T, first + piece))
        terms = reads[:, :, part].flip(-1).cumsum(-1).flip(-1) + (dstates[i] * states[i]).abs().sum((-1, -2)).detach().unsqueeze(-1)
        off = (got[:, :, part].double() - dg[:, :, part]).abs() / terms
        assert off.max() <= 1e-6, (first, off.max().item())

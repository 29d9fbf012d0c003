"""The norm and the gated delta rule together: the example, a layer's gradients, HIP graphs, and refusals of the tensor front ends (GPU)."""
import importlib.util
import os

import pytest
import torch

import paper_2605_11196_amd as vla
from test_gated_delta_gpu import make

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("gated_delta_layer", os.path.join(ROOT, "examples", "gated_delta_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_learns_and_generates():
    """Values have unit variance, so that the error starts at about 1; outputs are bfloat16 (2^-8 of the largest, through two projections)."""
    first, last, off, off_state = example().main(steps=120)
    assert last < 0.5 * first and off < 2e-2 and off_state < 2e-2


def test_a_lost_gradient_is_not_asked_for():
    q, k, v, g, beta, S0 = make(1, 2, 2, 40, 32, 32, "f32", seed=3)
    leaves = [x.detach().requires_grad_() for x in (q, k, v, g, beta, S0)]
    o, S = vla.gated_delta(*leaves)
    a = torch.autograd.grad(o.sum(), leaves, retain_graph=True)
    b = torch.autograd.grad((o, S), leaves, (torch.ones_like(o), torch.zeros_like(S)), retain_graph=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    c = torch.autograd.grad(S.sum(), leaves)
    assert (c[0] == 0).all() and (c[2] != 0).any()
    x = q.detach().requires_grad_()
    yq, yk = vla.qk_norm_rope(x, k)
    (d,) = torch.autograd.grad(yq.sum(), (x,))
    assert torch.isfinite(d).all()


def test_replays_of_a_captured_graph_match_the_eager_calls():
    """A decode step and a sequence in segments with its gradients, captured once and replayed with new inputs and other work between."""
    def inputs(seed):
        return make(2, 2, 4, 640, 64, 64, "bf16", seed=seed, rate=0.05)

    static = [x.clone() for x in inputs(1)]
    do, dS = torch.randn_like(static[2]), torch.randn_like(static[5])

    def work(q, k, v, g, beta, S0):
        o, S, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, save_for_backward=True, segments=4)
        grads = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS, segments=4)
        qn, kn = vla.qk_norm_rope(q, k, norm="l2")
        last = [x[:, :, -1].contiguous() for x in (qn, kn, v, g, beta)]
        step = vla.gated_delta_decode_step(*last, S)
        return [o, S, step, *grads]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(*static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work(*static)
    for seed in (2, 3, 4):
        fresh = inputs(seed)
        for a, b in zip(static, fresh):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = work(*fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), seed


@pytest.mark.parametrize("change", [
    dict(k=lambda x: x.float()), dict(v=lambda x: x[:, :, :-1]), dict(q=lambda x: x.half()), dict(g=lambda x: x.bfloat16()),
    dict(beta=lambda x: x[:, :1]), dict(S0=lambda x: x.double()), dict(S0=lambda x: x.transpose(2, 3)), dict(v=lambda x: x[:, :3]),
    dict(g=lambda x: x.cpu()), dict(q=lambda x: x[0])])
def test_gated_delta_refuses(change):
    names = ("q", "k", "v", "g", "beta", "S0")
    inputs = dict(zip(names, make(1, 2, 4, 6, 32, 64, "bf16", seed=1)))
    for name, f in change.items():
        inputs[name] = f(inputs[name])
    with pytest.raises(ValueError):
        vla.gated_delta_forward(**inputs)


def test_other_refusals():
    q, k, v, g, beta, S0 = make(1, 2, 4, 6, 32, 64, "bf16", seed=1)
    with pytest.raises(ValueError, match="lengths"):
        vla.gated_delta_forward(q, k, v, g, beta, lengths=torch.ones(1, device="cuda"))
    with pytest.raises(vla.VlaError):
        vla.gated_delta_forward(q[..., :24], k[..., :24], v, g, beta)      # no kernel for key heads of 24
    with pytest.raises(vla.VlaError):
        vla.gated_delta_forward(q, k, v, g, beta, scale=float("nan"))
    _, _, saved = vla.gated_delta_forward(q, k, v, g, beta, save_for_backward=True)
    with pytest.raises(vla.VlaError, match="WORKSPACE"):
        vla.gated_delta_backward(q, k, v, g, beta, saved[:64], v, None)
    with pytest.raises(ValueError, match="do"):
        vla.gated_delta_backward(q, k, v, g, beta, saved, v.float(), None)
    cos = torch.ones(8, 16, device="cuda")
    w = torch.ones(32, device="cuda")
    for kw in (dict(k=k[:, :, :-1]), dict(cos=cos), dict(cos=cos, sin=cos[:4]), dict(cos=cos.double(), sin=cos.double()), dict(norm="layer"),
               dict(q_weight=w[:16]), dict(q_weight=w, k_weight=w.bfloat16()), dict(positions=torch.zeros(1, 6, device="cuda")),
               dict(positions=torch.zeros(1, 5, device="cuda", dtype=torch.int32)), dict(cos=torch.ones(8, 20, device="cuda"), sin=torch.ones(8, 20, device="cuda"))):
        with pytest.raises(ValueError):
            vla.qk_norm_rope(**{**dict(q=q, k=k), **kw})
    with pytest.raises(vla.VlaError):
        vla.qk_norm_rope(q, k, cos=cos[:, :6], sin=cos[:, :6])      # 12 columns
    with pytest.raises(vla.VlaError):
        vla.qk_norm_rope(q, k, eps=0.0)


def test_offsets_beyond_32_bits():
    """More than 2^31 elements in a tensor, laid out with tokens before heads: the last sequence gives what it gives alone."""
    B, H, T, d = 3, 32, 180000, 128
    rows = torch.zeros((B, T, H, d), device="cuda", dtype=torch.bfloat16)
    assert rows.numel() > 2 ** 31
    rows[-1] = torch.nn.functional.normalize(torch.randn((T, H, d), device="cuda"), dim=-1)
    x = rows.transpose(1, 2)
    g = torch.full((B, H, T), -0.05, device="cuda")
    beta = torch.full((B, H, T), 0.5, device="cuda")
    o, S = vla.gated_delta_forward(x, x, x, g, beta)
    alone = vla.gated_delta_forward(x[-1:], x[-1:], x[-1:], g[-1:], beta[-1:])
    scale = alone[0].float().abs().max()
    assert ((o[-1].float() - alone[0][0].float()).abs().max() <= 1e-2 * scale) and (o[0] == 0).all()    # one rounding of bfloat16 apart at most: other segments
    assert (S[-1] - alone[1][0]).abs().max() <= 1e-5 * alone[1].abs().max()
    del o, S, alone
    q, _ = vla.qk_norm_rope(x, x[:, :1], norm="l2", eps=1e-12)
    one, _ = vla.qk_norm_rope(x[-1:], x[-1:, :1], norm="l2", eps=1e-12)
    assert torch.equal(q[-1], one[0])

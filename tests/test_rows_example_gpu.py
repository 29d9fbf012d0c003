"""The example of layers on the selective scan: it runs, and its gradients are those of the formulas (GPU)."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

import mixer_reference as ref
from test_rows_calls_gpu import near

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("selective_scan_layer", os.path.join(ROOT, "examples", "selective_scan_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_runs():
    """Prompt and single tokens round their outputs to bfloat16 at the same places, but the library's products of one row and of many sum in other orders, so
    that a number may round to its neighbour (2^-8 of itself) anywhere in two layers."""
    first, last, off, off_state = example().main(steps=3)
    assert all(map(torch.isfinite, map(torch.tensor, (first, last)))) and off < 2e-2 and off_state < 2e-2


def plain(p, x, layers, channels, states, taps):
    """The model from its formulas, with every parameter of p."""
    norm = lambda v, w: v * (v.square().mean(-1, keepdim=True) + 1e-6) ** -0.5 * w
    h = norm(x, p["norms"][0])
    for i in range(layers):
        q = {k.split(".", 2)[2]: v for k, v in p.items() if k.startswith(f"layers.{i}.")}
        a, z = F.linear(h, q["rows.weight"]).split(channels, -1)
        rows = F.pad(a, (0, 0, taps - 1, 0))
        pre = sum(q["conv"][:, j] * rows[:, j:j + a.shape[1]] for j in range(taps)) + q["conv_bias"]
        a = pre * torch.sigmoid(pre)
        Bm, Cm = F.linear(a, q["shared.weight"]).split(states, -1)
        dt = F.softplus(F.linear(a, q["delta.weight"]) + q["delta_bias"], threshold=100)
        state, y = torch.zeros(x.shape[0], channels, states, dtype=x.dtype), []
        for t in range(a.shape[1]):
            state = torch.exp(dt[:, t, :, None] * -q["log_A"].exp()) * state + (dt[:, t] * a[:, t])[..., None] * Bm[:, t, None]
            y.append((state * Cm[:, t, None]).sum(-1))
        y = F.linear((torch.stack(y, 1) + q["D"] * a) * z * torch.sigmoid(z), q["out.weight"])
        x, h = ref.residual(x, y, p["norms"][i + 1], p["posts"][i], 1, None, "silu", p["scales"][i], 1e-6)
    return h


def test_gradients_of_the_example():
    torch.manual_seed(3)
    model = example().SelectiveModel(32, 64, dtype=torch.float32)
    p = {k: v.detach().clone() for k, v in model.named_parameters()}
    x, dy = torch.randn(2, 30, 32), torch.randn(2, 30, 32)
    results = []
    for move in (torch.Tensor.double, torch.Tensor.clone):
        leaves = {k: move(v).requires_grad_() for k, v in p.items()}
        out = plain(leaves, move(x), 2, 64, 16, 4)
        results.append([out.detach(), *torch.autograd.grad(out, list(leaves.values()), move(dy))])
    model = model.cuda()
    out = model(x.cuda())[0]
    got = [out.detach(), *torch.autograd.grad(out, list(model.parameters()), dy.cuda())]
    for name, g, t, q in zip(("h", *p), got, *results):
        near(g, t, q, name)

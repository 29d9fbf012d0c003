"""The differentiable operators around the recurrence in a user's program: saved tensors that are offloaded, packed or formed again, on slices of
a fused projection (GPU).

Copies hold the same values and the kernels add up in a fixed order whatever the strides, so that the gradients have the same bits."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dense(x):
    return x.clone(memory_format=torch.contiguous_format)


def turned(x):
    """Tokens before heads, whatever the order was."""
    return x.transpose(1, 2).clone(memory_format=torch.contiguous_format).transpose(1, 2) if x.dim() >= 3 else x.clone()


def off_by_one(x):
    """Not at a 16-byte boundary."""
    room = torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)
    return room[1:].view(x.shape).copy_(x)


def hooks(name):
    if name in ("pageable", "pinned"):
        return torch.autograd.graph.save_on_cpu(pin_memory=name == "pinned")
    return torch.autograd.graph.saved_tensors_hooks(lambda x: x, {"dense": dense, "turned": turned, "off_by_one": off_by_one}[name])


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def projection(B, T, H_k, H_v, d, dtype, seed):
    """Leaves: rows of a projection, rows of its gates, S0; and the gradients of o and S_T."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows = (randn(gen, B, T, (2 * H_k + H_v) * d) * d ** -0.5).to(DT[dtype])
    gates, S0 = randn(gen, B, T, 2 * H_v), randn(gen, B, H_v, d, d) * 0.3
    return [x.requires_grad_() for x in (rows, gates, S0)], randn(gen, B, H_v, T, d).to(DT[dtype]), randn(gen, B, H_v, d, d)


def sliced(rows, gates, H_k, H_v, d):
    B, T, _ = rows.shape
    q, k, v = rows.view(B, T, -1, d).transpose(1, 2).split((H_k, H_k, H_v), 1)
    g, beta = gates.transpose(1, 2).split(H_v, 1)
    return q, k, v, -torch.nn.functional.softplus(g), torch.sigmoid(beta)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hook", ["pageable", "pinned", "dense", "turned", "off_by_one"])
def test_the_delta_rule_under_saved_tensor_hooks(hook, dtype):
    B, T, H_k, H_v, d = 3, 70, 2, 4, 32
    leaves, do, dS = projection(B, T, H_k, H_v, d, dtype, seed=1)
    lengths = torch.tensor([70, 0, 41], device="cuda", dtype=torch.int32)

    def grads():
        out = vla.gated_delta(*sliced(*leaves[:2], H_k, H_v, d), leaves[2], lengths=lengths.clone())
        return torch.autograd.grad(out, leaves, (do, dS))

    want = grads()
    with hooks(hook):
        got = grads()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_checkpointed_delta_rule(dtype):
    B, T, H_k, H_v, d = 2, 50, 1, 2, 64
    leaves, do, dS = projection(B, T, H_k, H_v, d, dtype, seed=2)

    def layer(rows, gates, S0):
        lengths = torch.tensor([13, 50]).to("cuda", torch.int32)
        return vla.gated_delta(*sliced(rows, gates, H_k, H_v, d), S0, lengths=lengths)

    want = torch.autograd.grad(layer(*leaves), leaves, (do, dS))
    out = checkpoint(layer, *leaves, use_reentrant=False)
    torch.full((64,), 3, device="cuda", dtype=torch.int32)      # takes the place of the first lengths
    got = torch.autograd.grad(out, leaves, (do, dS))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def norm_inputs(B, T, H_q, H_k, d, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows = randn(gen, B, T, (H_q + H_k) * d).to(DT[dtype])
    leaves = [x.requires_grad_() for x in (rows, 1 + 0.1 * randn(gen, d), 1 + 0.1 * randn(gen, d))]
    angle = torch.arange(64, device="cuda").unsqueeze(1) * 100.0 ** (-torch.arange(d // 4, device="cuda") * 4.0 / d)
    return leaves, (angle.cos(), angle.sin()), [randn(gen, B, H, T, d).to(DT[dtype]) for H in (H_q, H_k)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hook", ["pageable", "pinned", "dense", "turned", "off_by_one"])
def test_the_norm_under_saved_tensor_hooks(hook, dtype):
    B, T, H_q, H_k, d = 3, 21, 4, 2, 64
    leaves, tables, dy = norm_inputs(B, T, H_q, H_k, d, dtype, seed=3)
    positions = torch.randint(0, 64, (1, T), device="cuda", dtype=torch.int32)

    def grads():
        q, k = leaves[0].view(B, T, -1, d).transpose(1, 2).split((H_q, H_k), 1)
        out = vla.qk_norm_rope(q, k, *leaves[1:], *tables, positions=positions.expand(B, T), norm="l2")
        return torch.autograd.grad(out, leaves, dy)

    want = grads()
    with hooks(hook):
        got = grads()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_checkpointed_norm(dtype):
    B, T, H_q, H_k, d = 2, 16, 3, 1, 32
    leaves, tables, dy = norm_inputs(B, T, H_q, H_k, d, dtype, seed=4)
    start = torch.tensor([[5], [40]]).cuda()

    def layer(rows, *weights):
        q, k = rows.view(B, T, -1, d).transpose(1, 2).split((H_q, H_k), 1)
        positions = (start + torch.arange(T, device="cuda")).int()
        return vla.qk_norm_rope(q, k, *weights, *tables, positions=positions, interleaved=True)

    want = torch.autograd.grad(layer(*leaves), leaves, dy)
    out = checkpoint(layer, *leaves, use_reentrant=False)
    torch.full((128,), 7, device="cuda", dtype=torch.int32)     # takes the place of the first positions
    got = torch.autograd.grad(out, leaves, dy)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_a_state_that_starts_anywhere():
    """Cut out of a larger buffer; its gradient comes back from torch.cat, not at a 16-byte boundary either."""
    leaves, do, dS = projection(2, 40, 1, 2, 32, "f32", seed=5)
    inputs = sliced(*leaves[:2], 1, 2, 32)
    want = torch.autograd.grad(vla.gated_delta(*inputs, leaves[2]), leaves, (do, dS), retain_graph=True)
    S0 = off_by_one(leaves[2].detach()).requires_grad_()
    o, S = vla.gated_delta(*inputs, S0)
    joined = torch.cat((torch.zeros(1, device="cuda"), S.flatten(), o.flatten()))
    got = torch.autograd.grad(joined, (*leaves[:2], S0), torch.cat((torch.zeros(1, device="cuda"), dS.flatten(), do.flatten())))
    assert all(torch.equal(x, y) for x, y in zip(got, want))

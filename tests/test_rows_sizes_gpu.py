"""The operators on rows of channels at sizes where their kernels go round a loop again: more columns than a launch holds work-items for, more rows than
workgroups, more segments than are joined at once, long runs of tokens (GPU)."""
import ctypes

import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla
from paper_2605_11196_amd.binding import VlaScanOpts

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


# ---- more rows than the workgroups take at once

# Roundings as in test_residual_norm_gpu.py: 256 for a row.  The weights' gradients: 8 rows of a workgroup, four turns of it, and the parts of up to 1024
# workgroups, 64 by each of the 16 waves that add them.
@pytest.mark.parametrize("n,rows,each,groups,stream", [
    # each: rows that a workgroup of the backward pass takes at once
    (264, 2 * 6144 + 1001, 8, 3, None),      # four rows a workgroup forward, groups whose sums go through shared memory
    (1000, 4 * 1536 + 999, 4, 1, "f32"),     # a row on two waves, two rows a workgroup forward
    (1536, 2 * 2048 + 1537, 2, 1, None),     # three waves, a row alone forward
    (4096, 2 * 768 + 501, 1, 64, None),      # eight waves, heads of 64 columns
    (4096, 2 * 768 + 501, 1, 1, "f32"),
    (8192, 2 * 256 + 131, 1, 2, None),       # sixteen waves, groups of half a row
])
def test_norms_of_rows_that_workgroups_go_through_in_turns(n, rows, each, groups, stream):
    assert rows > 2 * each * vla.load_library().vla_residual_norm_workspace_bytes(n) // (3 * n * 4)      # a part for every workgroup of the backward pass
    gen = torch.Generator(device="cuda").manual_seed(n)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    of_stream = DT[stream or "bf16"]
    s = dict(x=(3 * r(1, rows, n)).to(of_stream), y=r(1, rows, n).bfloat16(), weight=(1 + 0.2 * r(n)).bfloat16(), post_weight=(1 + 0.2 * r(n)).bfloat16(),
             gate=r(1, rows, n).bfloat16(), scale=(0.5 + 0.2 * r(n)).bfloat16())
    ds, dh = r(1, rows, n).to(of_stream), r(1, rows, n).bfloat16()
    how = dict(post_weight=s["post_weight"], groups=groups, gate=s["gate"], scale=s["scale"])
    got = [*vla.residual_norm(s["x"], s["y"], s["weight"], **how), *vla.residual_norm_backward(s["x"], s["y"], s["weight"], ds, dh, **how)]
    leaves = {k: v.double().requires_grad_() for k, v in s.items()}
    args = leaves["x"], leaves["y"], leaves["weight"], leaves["post_weight"], groups, leaves["gate"], "silu", leaves["scale"], 1e-6
    out = ref.residual(*args)
    names = "x", "y", "weight", "post_weight", "gate", "scale"
    want = [*(o.detach() for o in out), *torch.autograd.grad(out, [leaves[k] for k in names], [ds.double(), dh.double()])]
    del out
    sizes = dict(zip(("s", "h", "x", "y", "gate", "weight", "post_weight", "scale"),
                     ref.residual_sizes(*(a.detach() if torch.is_tensor(a) else a for a in args), ds.double(), dh.double())))
    for name, g, w in zip(("s", "h", *names), got, want):
        ref.close(g, w, sizes[name], 256 + (8 + 4 + 64 + 16 if w.dim() == 1 else 0), name)


# ---- more segments than are joined at once

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,segments", [(69, 9), (125, 16), (133, 17), (285, 18), (300, 38)])
def test_many_segments(dtype, T, segments):
    """As many segments as are asked for (blocks of eight tokens, one or two each), states joined eight at a time; sequences that end in the first segment, in one
    behind the eighth, and at the end."""
    B, n, N = 4, 72, 16
    opts = VlaScanOpts(1, 1, segments=segments)
    padded = lambda size: -(-size // 256) * 256
    assert (vla.load_library().vla_selective_scan_workspace_bytes(B, T, n, N, 0, ctypes.byref(opts), 0)
            == padded(B * segments * n * N * 4) + padded(B * segments * n * 4))
    gen = torch.Generator().manual_seed(T)
    r = lambda *s: torch.randn(s, generator=gen)
    io = lambda *s: r(*s).to(DT[dtype])
    s = dict(u=io(B, T, n), delta=io(B, T, n), A=-torch.arange(1, N + 1).float() * torch.exp(0.3 * r(n, N)), B=io(B, T, 1, N), C=io(B, T, 1, N), D=r(n),
             z=io(B, T, n), delta_bias=r(n) - 3, h0=r(B, n, N))
    lengths = torch.tensor([T, 3, T - 2, T // 2 + 29], dtype=torch.int32)
    dy, dh = io(B, T, n), r(B, n, N)
    both = []
    for magnitude in (False, True):
        leaves = {k: ref.double(v).requires_grad_() for k, v in s.items()}
        out = ref.scan(*leaves.values(), lengths, True, magnitude)
        d = [torch.where(torch.arange(T)[None, :, None] < lengths[:, None, None], dy.double(), 0.0), dh.double()]
        grads = torch.autograd.grad(out, list(leaves.values()), [x.abs() for x in d] if magnitude else d)
        both.append([x.detach().abs() if magnitude else x.detach() for x in (*out, *grads)])
    cuda = {k: v.cuda() for k, v in s.items()}
    args = [cuda[k] for k in ("u", "delta", "A", "B", "C", "D", "z")]
    kw = dict(delta_bias=cuda["delta_bias"], lengths=lengths.cuda(), segments=segments)
    y, h_T, saved = vla.selective_scan_forward(*args, cuda["h0"], save_for_backward=True, **kw)
    got = [y, h_T, *vla.selective_scan_backward(*args, saved, dy.cuda(), dh.cuda(), **kw)]
    for name, g, w, m in zip(("y", "h_T", *("d" + k for k in s)), got, *both):
        # 48 roundings a token and those of the sums, as for the scan's other tests
        ref.close(g, w, m, 48 * T + n / 2 + N + 64 + B * T, name)


# ---- long runs of tokens

@pytest.mark.parametrize("B,T,n,W,dtype,run,parts", [
    # a thread's run, parts that column sums add
    (2, 16411, 1032, 4, "f32", 32, 2 * 513),
    (16, 58301, 72, 3, "bf16", 32, 1025),            # runs of the same channels in a workgroup
    (4, 65573, 2048, 4, "bf16", 256, 4 * 257),
])
def test_runs_of_many_tokens(B, T, n, W, dtype, run, parts):
    """Channels have nothing to do with each other: the reference takes some of them."""
    assert vla.load_library().vla_causal_conv_workspace_bytes(B, T, n, W, dtype == "bf16") == parts * (W + 1) * n * 4
    gen = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=DT[dtype])
    x, dy, weight, bias, state, dstate_T = r(B, T, n), r(B, T, n), r(n, W), r(n), r(B, W - 1, n), r(B, W - 1, n)
    lengths = torch.full((B,), T, dtype=torch.int32, device="cuda")
    lengths[0] = T - 3 * run - 7
    got = [*vla.causal_conv(x, weight, bias, state, lengths=lengths), *vla.causal_conv_backward(x, weight, bias, state, dy, dstate_T, lengths=lengths)]
    some = torch.tensor([0, 7, 8, n // 2 + 3, n - 9, n - 1], device="cuda")
    both = []
    for magnitude in (False, True):
        leaves = [ref.double(v).requires_grad_() for v in (x[..., some], weight[some], bias[some], state[..., some])]
        out = ref.conv(*leaves, lengths, True, magnitude)
        d = [ref.double(dy[..., some]), ref.double(dstate_T[..., some])]
        grads = torch.autograd.grad(out, leaves, [v.abs() for v in d] if magnitude else d)
        both.append([v.detach().abs() if magnitude else v.detach() for v in (*out, *grads)])
    for name, g, w, m in zip(("y", "state_T", "dx", "dweight", "dbias", "dstate"), got, *both):
        weights = name in ("dweight", "dbias")
        # the taps, the bias and the activation; a run's tokens, a workgroup's runs of a channel, parts over 16 waves and these
        k = 2 * W + 24 + (run + 256 // 9 + 1 + parts // 16 + 1 + 16 if weights else 0)
        ref.close(g[some] if weights else g[..., some], w, m, k, name)

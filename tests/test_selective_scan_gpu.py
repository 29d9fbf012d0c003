"""The selective state space scan against the recurrence in 64 bits: outputs, states, gradients, segments, one token (GPU)."""
import pytest
import torch

import mixer_reference as ref
import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "h0")


def make(B, T, n, N, dtype, *, G=1, gate=True, D=True, bias=True, carried=True, seed=0, dev="cuda"):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    io = lambda x: x.to(DT[dtype]).to(dev)
    A = -torch.arange(1, N + 1).float() * torch.exp(0.3 * r(n, N))
    return dict(u=io(r(B, T, n)), delta=io(r(B, T, n)), A=A.to(dev), B=io(r(B, T, G, N)), C=io(r(B, T, G, N)), D=r(n).to(dev) if D else None,
                z=io(r(B, T, n)) if gate else None, delta_bias=(r(n) - 3).to(dev) if bias else None, h0=r(B, n, N).to(dev) if carried else None)


def call(s, **kw):
    return vla.selective_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["h0"], delta_bias=s["delta_bias"], **kw)


def references(s, lengths=None, softplus=True, grads=None):
    """The outputs and, given those of the outputs, the inputs' gradients, in 64 bits, and what they are measured by."""
    both = []
    for magnitude in (False, True):
        leaves = {k: ref.double(s[k]) for k in NAMES}
        for k in leaves:
            if leaves[k] is not None and grads is not None:
                leaves[k].requires_grad_()
        out = ref.scan(*(leaves[k] for k in NAMES), lengths, softplus, magnitude)
        got = [x.detach() for x in out]
        if grads is not None:
            d = [ref.double(g) for g in grads]
            live = 1.0 if lengths is None else (torch.arange(s["u"].shape[1])[None, :, None] < lengths.cpu()[:, None, None])
            d[0] = torch.where(torch.as_tensor(live, dtype=torch.bool).expand_as(d[0]), d[0], 0.0)
            d = [x.abs() for x in d] if magnitude else d
            names = [k for k in NAMES if leaves[k] is not None]
            back = torch.autograd.grad(out, [leaves[k] for k in names], d, allow_unused=True)
            got += [torch.zeros_like(leaves[k]) if g is None else g for k, g in zip(names, back)]
            got = [g.abs() if magnitude else g for g in got]
        both.append(got)
    return both


# Roundings that a term of a sum goes through: a step of the decay has the product, the exponential (its argument of up to 30 comes with
# one, and counts as often), the update and the step's own (softplus: six); the sums over channels, tokens and states add theirs.
def roundings(T, n, N):
    return 48 * T + n / 2 + N + 64


CASES = [
    # B, T, n, N, G, dtype, options
    (1, 1, 8, 8, 1, "f32", {}),
    (2, 7, 64, 16, 1, "bf16", {}),
    (1, 8, 136, 16, 1, "f32", dict(gate=False)),
    (3, 9, 72, 32, 1, "bf16", dict(carried=False)),
    (2, 65, 256, 16, 2, "f32", {}),
    (1, 33, 400, 64, 1, "bf16", dict(D=False)),
    (2, 40, 48, 64, 3, "f32", dict(bias=False)),
    (1, 130, 128, 8, 1, "bf16", dict(gate=False, D=False, bias=False, carried=False)),
    (2, 100, 272, 8, 2, "f32", {}),
    (1, 200, 128, 32, 1, "f32", {}),
]


@pytest.mark.parametrize("B,T,n,N,G,dtype,options", CASES)
def test_outputs_and_gradients(B, T, n, N, G, dtype, options):
    s = make(B, T, n, N, dtype, G=G, seed=T + n, **options)
    gen = torch.Generator().manual_seed(99)
    grads = [torch.randn((B, T, n), generator=gen).to(DT[dtype]).cuda(), torch.randn((B, n, N), generator=gen).cuda()]
    want, size = references(s, grads=grads)
    leaves = {k: x if x is None else x.detach().requires_grad_() for k, x in s.items()}
    out = call(leaves)
    given = [x for x in leaves.values() if x is not None]
    got = [*out, *torch.autograd.grad(out, given, grads)]
    names = ["y", "h_T", *("d" + k for k in NAMES if s[k] is not None)]
    for name, g, w, m in zip(names, got, want, size):
        ref.close(g, w, m, roundings(T, n, N) + (B * T if name in ("dA", "dD", "ddelta_bias") else 0), name)
    plain = call(s)
    assert all(torch.equal(a, b) for a, b in zip(plain, out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("segments", [1, 2, 3, 7])
def test_segments(dtype, segments):
    B, T, n, N = 2, 101, 136, 16
    s = make(B, T, n, N, dtype, seed=5)
    lengths = torch.tensor([101, 37], dtype=torch.int32, device="cuda")
    dy, dh = torch.randn(B, T, n).to(DT[dtype]).cuda(), torch.randn(B, n, N).cuda()
    want, size = references(s, lengths, grads=[dy, dh])
    args = [s[k] for k in ("u", "delta", "A", "B", "C", "D", "z")]
    y, h_T, saved = vla.selective_scan_forward(*args, s["h0"], delta_bias=s["delta_bias"], lengths=lengths, save_for_backward=True, segments=segments)
    grads = vla.selective_scan_backward(*args, saved, dy, dh, delta_bias=s["delta_bias"], lengths=lengths, segments=segments)
    for i, (g, w, m) in enumerate(zip((y, h_T, *grads), want, size)):
        ref.close(g, w, m, roundings(T, n, N) + B * T, str(i))


def test_steps_without_softplus():
    s = make(2, 20, 64, 16, "f32", seed=3)
    s["delta"], s["delta_bias"] = s["delta"].abs() * 0.1, s["delta_bias"].abs() * 0.1
    want, size = references(s, softplus=False)
    for g, w, m in zip(call(s, softplus=False), want, size):
        ref.close(g, w, m, roundings(20, 64, 16))


@pytest.mark.parametrize("value", [-100.0, -20.0, -8.0, 0.0, 8.0, 25.0, 80.0])
def test_softplus_over_its_range(value):
    """y = dt u from a zero state with A = 0, B = C of 1 in one state: the step itself.  Below -87 the exponential is no normal number."""
    n, N = 8, 8
    d = torch.linspace(value - 1, value + 1, n).view(1, 1, n).cuda()
    B = torch.zeros(1, 1, N).cuda()
    B[..., 0] = 1
    y, h = vla.selective_scan(torch.ones_like(d), d, torch.zeros(n, N).cuda(), B, B)
    want = torch.logaddexp(ref.double(d), torch.zeros(1, dtype=torch.float64))
    # the exponential's argument times log2(e) rounded twice, the exponential, its logarithm, quotient and product
    ref.close(y, want, want * (2 + d.abs().cpu()) + (1e-30 if value < -80 else 0), 12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_and_what_lies_behind_them(dtype):
    """NaN and infinities behind the end of a sequence reach nothing; lengths out of range count as the nearer end; outputs there are 0."""
    B, T, n, N = 5, 50, 72, 16
    s = make(B, T, n, N, dtype, seed=11)
    given = torch.tensor([50, 0, 23, 99, -4], dtype=torch.int32)
    lengths = given.clamp(0, T)
    want, size = references(s, lengths, grads=None)
    for b in range(B):
        for k, bad in (("u", float("nan")), ("delta", float("inf")), ("B", float("nan")), ("C", float("inf")), ("z", float("nan"))):
            s[k][b, lengths[b]:] = bad
    dy, dh = torch.randn(B, T, n).to(DT[dtype]).cuda(), torch.randn(B, n, N).cuda()
    for b in range(B):
        dy[b, lengths[b]:] = float("nan")
    for segments in (1, 3):
        args = [s[k] for k in ("u", "delta", "A", "B", "C", "D", "z")]
        y, h_T, saved = vla.selective_scan_forward(*args, s["h0"], delta_bias=s["delta_bias"], lengths=given.cuda(), save_for_backward=True, segments=segments)
        grads = vla.selective_scan_backward(*args, saved, dy, dh, delta_bias=s["delta_bias"], lengths=given.cuda(), segments=segments)
        for g, w, m in zip((y, h_T), want, size):
            ref.close(g, w, m, roundings(T, n, N))
        assert all(torch.isfinite(g).all() for g in grads)
        for b in range(B):
            for x in (y, grads[0], grads[1], grads[3], grads[4], grads[6]):
                assert (x[b, lengths[b]:] == 0).all()
    assert torch.equal(h_T[1], s["h0"][1]) and torch.equal(grads[8][1], dh[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
def test_one_token_at_a_time(dtype, N):
    """Tokens one by one on a state in place, and a sequence continued from a carried state, against the whole sequence."""
    B, T, n, G = 3, 12, 48, 2
    s = make(B, T, n, N, dtype, G=G, seed=N)
    want, size = references(s)
    h = s["h0"].clone()
    part = {k: x if x is None or k not in ("u", "delta", "B", "C", "z") else x[:, :5] for k, x in s.items()}
    first, carried = call(part)
    for t in range(T):
        if t == 5:
            ref.close(h, carried.cpu(), size[1], 2 * roundings(5, n, N))
        y = vla.selective_scan_step(s["u"][:, t], s["delta"][:, t], s["A"], s["B"][:, t], s["C"][:, t], h, s["D"], s["z"][:, t], delta_bias=s["delta_bias"])
        ref.close(y, want[0][:, t], size[0][:, t], roundings(T, n, N), f"token {t}")
    ref.close(h, want[1], size[1], roundings(T, n, N))


def test_no_token():
    s = make(2, 0, 64, 16, "f32")
    leaves = {k: x.detach().requires_grad_() for k, x in s.items()}
    y, h = call(leaves)
    assert y.shape == (2, 0, 64) and torch.equal(h, s["h0"])
    g = torch.randn_like(h)
    (dh0, dA) = torch.autograd.grad(h, (leaves["h0"], leaves["A"]), g)
    assert torch.equal(dh0, g) and (dA == 0).all()


def test_views_of_projections():
    """Slices of fused projections, tokens and sequences swapped, and inputs that repeat over tokens are read as they are or copied."""
    B, T, n, N = 2, 19, 64, 16
    s = make(B, T, n, N, "bf16", seed=21)
    want = call(s)
    wide = torch.randn(B, T, 3 * n + 2 * N + 8).bfloat16().cuda()
    wide[..., 8:8 + N], wide[..., 8 + N:8 + 2 * N] = s["B"][:, :, 0], s["C"][:, :, 0]
    at = 8 + 2 * N
    for i, k in enumerate(("u", "delta", "z")):
        wide[..., at + i * n:at + (i + 1) * n] = s[k]
    view = dict(s, B=wide[..., 8:8 + N], C=wide[..., 8 + N:8 + 2 * N], **{k: wide[..., at + i * n:at + (i + 1) * n] for i, k in enumerate(("u", "delta", "z"))})
    assert all(torch.equal(a, b) for a, b in zip(call(view), want))
    swapped = dict(s, **{k: s[k].transpose(0, 1).contiguous().transpose(0, 1) for k in ("u", "delta", "z", "B", "C")})
    assert all(torch.equal(a, b) for a, b in zip(call(swapped), want))
    odd = torch.empty(B * T * n + 1, dtype=torch.bfloat16, device="cuda")[1:].view(B, T, n)
    odd.copy_(s["u"])
    assert all(torch.equal(a, b) for a, b in zip(call(dict(s, u=odd)), want))
    repeated = dict(s, delta=s["delta"][:, :1].expand(B, T, n), z=s["z"][:1, :1].expand(B, T, n), C=s["C"][:, :1].expand(B, T, 1, N))
    dense = {k: None if x is None else x.contiguous() for k, x in repeated.items()}
    leaves = {k: x.detach().requires_grad_() for k, x in dict(s, delta=s["delta"][:, :1], z=s["z"][:1, :1], C=s["C"][:, :1]).items()}
    seen = dict(leaves, delta=leaves["delta"].expand(B, T, n), z=leaves["z"].expand(B, T, n), C=leaves["C"].expand(B, T, 1, N))
    y, h = call(seen)
    assert all(torch.equal(a, b) for a, b in zip((y, h), call(dense)))
    g = torch.ones_like(y)
    full = {k: x.detach().requires_grad_() for k, x in dense.items()}
    ours = torch.autograd.grad(y, [leaves[k] for k in ("delta", "z", "C", "A")], g)
    theirs = torch.autograd.grad(call(full)[0], [full[k] for k in ("delta", "z", "C", "A")], g)
    sums = (theirs[0].sum(1, keepdim=True), theirs[1].sum((0, 1), keepdim=True), theirs[2].sum(1, keepdim=True), theirs[3])
    assert all(torch.equal(a, b) for a, b in zip(ours, sums))


def test_gradients_against_differences():
    """Along a random direction of all inputs: the slope of the reference in 64 bits by central differences (error h^2 of the third derivative,
    1e-8 here, and 1e-16 / h of the values)."""
    B, T, n, N = 1, 10, 16, 8
    s = make(B, T, n, N, "f32", seed=8)
    gen = torch.Generator().manual_seed(4)
    way = {k: torch.randn(x.shape, generator=gen, dtype=torch.float64) for k, x in s.items()}
    weight = [torch.randn((B, T, n), generator=gen).double(), torch.randn((B, n, N), generator=gen).double()]

    def value(h):
        out = ref.scan(*(ref.double(s[k]) + h * way[k] for k in NAMES), None)
        return sum((o * w).sum() for o, w in zip(out, weight))

    h = 1e-4
    slope = (value(h) - value(-h)) / (2 * h)
    leaves = {k: x.detach().requires_grad_() for k, x in s.items()}
    grads = torch.autograd.grad(call(leaves), [leaves[k] for k in NAMES], [w.float().cuda() for w in weight])
    parts = [(g.double().cpu() * way[k]) for g, k in zip(grads, NAMES)]
    got, size = sum(p.sum() for p in parts), sum(p.abs().sum() for p in parts)
    assert abs(got - slope) <= (roundings(T, n, N) * 4 * ref.UNIT + 1e-6) * size


def test_the_same_bits_again():
    s = make(2, 300, 256, 16, "bf16", seed=2)
    grads = [torch.randn(2, 300, 256).bfloat16().cuda(), torch.randn(2, 256, 16).cuda()]
    runs = []
    for _ in range(3):
        leaves = {k: x.detach().requires_grad_() for k, x in s.items()}
        out = call(leaves)
        runs.append([*out, *torch.autograd.grad(out, list(leaves.values()), grads)])
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_infinities_stay_in_their_channel():
    """A state that overflows, a NaN input: the other channels of the sequence and the other sequences keep their outputs."""
    s = make(2, 24, 64, 16, "f32", seed=13)
    want = call(s)
    s["u"][0, 5, 3] = float("nan")
    s["h0"][0, 7, 2] = float("inf")
    y, h = call(s)
    keep = torch.ones(64, dtype=torch.bool)
    keep[[3, 7]] = False
    assert torch.equal(y[0][:, keep], want[0][0][:, keep]) and torch.equal(h[0][keep], want[1][0][keep]) and torch.equal(y[1], want[0][1])
    assert torch.isnan(y[0, 5:, 3]).all() and torch.equal(y[0, :5, 3], want[0][0, :5, 3]) and not torch.isfinite(y[0, :, 7]).any()


def test_growing_states_that_are_zero_stay_zero():
    """A > 0 and steps whose product over a segment overflows: an empty state has nothing to grow, in segments as in one piece, and the gradients have
    nothing to go back to."""
    B, T, n, N = 1, 40, 64, 16
    s = make(B, T, n, N, "f32", D=False, gate=False, bias=False, carried=False, seed=8)
    args = dict(s, A=torch.ones(n, N).cuda(), delta=torch.full((B, T, n), 30.0).cuda(), u=torch.zeros(B, T, n).cuda())
    args["u"][:, -1] = s["u"][:, -1]
    y, h, saved = vla.selective_scan_forward(*(args[k] for k in ("u", "delta", "A", "B", "C")), softplus=False, save_for_backward=True, segments=1)
    assert torch.isfinite(y).all() and torch.isfinite(h).all() and (y[:, :-1] == 0).all() and (h != 0).all()
    cut = vla.selective_scan_forward(*(args[k] for k in ("u", "delta", "A", "B", "C")), softplus=False, segments=5)
    assert torch.equal(cut[0], y) and torch.equal(cut[1], h)
    dy = torch.zeros(B, T, n).cuda()
    dy[:, 0] = 1.0
    whole, pieces = (vla.selective_scan_backward(*(args[k] for k in ("u", "delta", "A", "B", "C")), None, None, saved, dy, softplus=False, segments=k)
                     for k in (1, 5))
    for name, a, b in zip(("du", "ddelta", "dA", "dB", "dC"), whole, pieces):
        assert torch.isfinite(a).all() and torch.equal(a, b), name

"""The gated delta rule against the token-by-token recurrence in float64 (GPU).

Tolerances, of the largest value of a head: the state is a sum of writes in float32, with decays and keys of at most unit
length, so that its error is some roundings of 2^-24 that do not grow with the length: 1e-5 holds with room.  float32 outputs the
same; bfloat16 outputs one rounding (2^-9 of a value) on top of products that carry 16 bits of the state: 6e-3."""
import pytest
import torch

import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 1e-5, "bf16": 6e-3}


def make(B, H_k, H_v, T, d_k, d_v, dtype, seed, carried=True, rate=0.3):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    q, k = (unit(rnd(B, H_k, T, d_k)).to(DT[dtype]) for _ in range(2))
    v = rnd(B, H_v, T, d_v).to(DT[dtype])
    g = -rate * torch.nn.functional.softplus(rnd(B, H_v, T))
    beta = torch.sigmoid(rnd(B, H_v, T))
    S0 = rnd(B, H_v, d_v, d_k) * 0.3 if carried else None
    return q, k, v, g, beta, S0


def oracle(q, k, v, g, beta, S0, scale=None, lengths=None):
    """float64, differentiable: (o, S_T)"""
    B, H_k, T, d_k = q.shape
    H_v, d_v = v.shape[1], v.shape[-1]
    q, k = (x.double().repeat_interleave(H_v // H_k, 1) for x in (q, k))
    v, alpha, beta = v.double(), g.double().exp(), beta.double()
    scale = d_k ** -0.5 if scale is None else scale
    S = torch.zeros((B, H_v, d_v, d_k), dtype=torch.float64, device=q.device) if S0 is None else S0.double()
    o = []
    for t in range(T):
        old = S * alpha[:, :, t, None, None]
        e = beta[:, :, t, None] * (v[:, :, t] - (old * k[:, :, t, None, :]).sum(-1))
        new = old + e[..., None] * k[:, :, t, None, :]
        out = scale * (new * q[:, :, t, None, :]).sum(-1)
        if lengths is not None:
            live = (t < lengths)[:, None, None]
            new, out = torch.where(live[..., None], new, S), torch.where(live, out, torch.zeros_like(out))
        S = new
        o.append(out)
    return (torch.stack(o, 2) if T else torch.zeros_like(v)), S


def close(got, want, tol, what, per_head=True):
    assert got.shape == want.shape, what
    if not want.numel():
        return
    dims = tuple(range(2, want.dim())) if per_head else tuple(range(want.dim()))
    err = ((got.double() - want).abs().amax(dims) / want.abs().amax(dims).clamp_min(1e-20)).max().item()
    assert err <= tol, (what, err)


def check(inputs, dtype, **kw):
    o, S = vla.gated_delta_forward(*inputs, **kw)
    ro, rS = oracle(*inputs, scale=kw.get("scale"), lengths=kw.get("lengths"))
    close(o, ro, TOL[dtype], "o")
    close(S, rS, TOL["f32"], "S_T")
    return o, S


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 200])
def test_lengths_around_the_blocks(T, dtype):
    check(make(2, 2, 2, T, 64, 64, dtype, seed=T), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_v", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("d_k", [16, 32, 64, 96, 128])
def test_head_sizes(d_k, d_v, dtype):
    for T, carried in ((83, True), (5, False)):
        check(make(1, 2, 4, T, d_k, d_v, dtype, seed=d_k + 3 * d_v + T, carried=carried), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H_k,H_v", [(1, 1), (1, 5), (3, 6)])
def test_shared_key_heads_and_scale(H_k, H_v, dtype):
    check(make(3, H_k, H_v, 70, 32, 64, dtype, seed=H_v), dtype, scale=0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ragged_lengths_hide_what_lies_beyond(dtype):
    T = 150
    inputs = make(7, 2, 4, T, 64, 32, dtype, seed=8)
    lengths = torch.tensor([0, 1, 31, 32, 97, T, T + 9], device="cuda", dtype=torch.int32)
    o, S = check(inputs, dtype, lengths=lengths)
    assert torch.equal(S[0], inputs[5][0]) and (o[0] == 0).all()
    q, k, v, g, beta, S0 = (x.clone() for x in inputs)
    for b, n in enumerate(lengths.tolist()):
        for x, fill in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (g, float("nan")), (beta, float("inf"))):
            x[b, :, max(n, 0):] = fill
    o2, S2 = vla.gated_delta_forward(q, k, v, g, beta, S0, lengths=lengths)
    assert torch.equal(o, o2) and torch.equal(S, S2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_that_forget(dtype):
    """Decays of one, strong ones, ones that leave float32 and minus infinity; beta of 0 and 2."""
    q, k, v, g, beta, S0 = make(2, 2, 2, 90, 32, 32, dtype, seed=11, rate=4.0)
    g[0, 0] = 0
    g[0, 1, ::7] = float("-inf")
    g[1, 0, 5:40] = -90.0
    g[1, 1, 60] = -1e30
    beta[0, 0, ::3] = 0
    beta[1, 1, ::5] = 2
    check((q, k, v, g, beta, S0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_keys(dtype):
    """The same key at every token: the block's triangular system at its worst for unit keys."""
    q, k, v, g, beta, S0 = make(1, 2, 2, 140, 64, 64, dtype, seed=12)
    k = k[:, :, :1].expand_as(k).contiguous()
    g = torch.zeros_like(g)
    beta = torch.ones_like(beta)
    check((q, k, v, g, beta, S0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mult", [1e-20, 1e20])
def test_small_and_large_values(mult, dtype):
    q, k, v, g, beta, S0 = make(1, 2, 2, 75, 64, 64, dtype, seed=13)
    check((q, k, (v.float() * mult).to(v.dtype), g, beta, S0 * mult), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequences_and_continuation(dtype):
    inputs = make(1, 2, 2, 2500, 64, 64, dtype, seed=14, rate=0.01)
    o, S = check(inputs, dtype)
    q, k, v, g, beta, S0 = inputs
    cut = 1011
    first = vla.gated_delta_forward(q[:, :, :cut], k[:, :, :cut], v[:, :, :cut], g[:, :, :cut], beta[:, :, :cut], S0)
    second = vla.gated_delta_forward(q[:, :, cut:], k[:, :, cut:], v[:, :, cut:], g[:, :, cut:], beta[:, :, cut:], first[1])
    close(torch.cat((first[0], second[0]), 2), o.double(), TOL[dtype], "o in two calls")
    close(second[1], S.double(), TOL["f32"], "S_T in two calls")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    q, k, v, g, beta, S0 = make(2, 2, 4, 77, 64, 96, dtype, seed=15)
    want = vla.gated_delta_forward(q, k, v, g, beta, S0)
    rows = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)       # [B, T, H, d] in memory
    wide = torch.cat((v.transpose(1, 2), v.transpose(1, 2)), -1)[..., :96].transpose(1, 2)
    got = vla.gated_delta_forward(rows(q), rows(k), wide, rows(g.unsqueeze(-1))[..., 0], rows(beta.unsqueeze(-1))[..., 0], S0)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert got[0].transpose(1, 2).is_contiguous()
    same = vla.gated_delta_forward(q[:1].expand_as(q), k, v, g[:, :1].expand_as(g), beta, S0)
    ref = vla.gated_delta_forward(q[:1].expand_as(q).contiguous(), k, v, g[:, :1].expand_as(g).contiguous(), beta, S0)
    assert torch.equal(same[0], ref[0])
    buffer = torch.zeros(q.numel() + 1, device="cuda", dtype=q.dtype)
    shifted = buffer[1:].view(q.shape).copy_(q)      # not 16-byte aligned
    assert torch.equal(vla.gated_delta_forward(shifted, k, v, g, beta, S0)[0], want[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_k,d_v,H_k,H_v", [(16, 128, 1, 3), (32, 16, 2, 2), (64, 64, 2, 8), (96, 96, 1, 1), (128, 128, 4, 8)])
def test_single_tokens(d_k, d_v, H_k, H_v, dtype):
    T = 6
    inputs = make(3, H_k, H_v, T, d_k, d_v, dtype, seed=d_k + d_v)
    ro, rS = oracle(*inputs)
    q, k, v, g, beta, S = inputs
    S = S.clone()
    for t in range(T):
        o = vla.gated_delta_decode_step(q[:, :, t], k[:, :, t], v[:, :, t], g[:, :, t], beta[:, :, t], S)
        close(o, ro[:, :, t], TOL[dtype], t)
    close(S, rS, TOL["f32"], "S")


def test_no_tokens():
    inputs = make(2, 1, 2, 0, 32, 32, "f32", seed=1)
    o, S = vla.gated_delta_forward(*inputs)
    assert o.shape == (2, 2, 0, 32) and torch.equal(S, inputs[5])
    o, S = vla.gated_delta_forward(*inputs[:5])
    assert (S == 0).all()


def test_nan_stays_in_its_head():
    q, k, v, g, beta, S0 = make(1, 2, 2, 50, 32, 32, "f32", seed=2)
    want = vla.gated_delta_forward(q, k, v, g, beta, S0)
    g = g.clone()
    g[0, 0, 20] = float("nan")
    o, S = vla.gated_delta_forward(q, k, v, g, beta, S0)
    assert torch.isnan(S[0, 0]).all() and torch.equal(S[0, 1], want[1][0, 1]) and torch.equal(o[0, 1], want[0][0, 1])


def test_runs_on_the_given_stream():
    inputs = make(2, 2, 2, 300, 64, 64, "bf16", seed=6)
    want = vla.gated_delta_forward(*inputs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = vla.gated_delta_forward(*inputs, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_k,d_v,T,segments", [(16, 16, 100, 2), (16, 96, 333, 4), (32, 64, 200, 7), (64, 64, 1000, 5), (64, 32, 97, 256), (96, 128, 300, 3),
                                                (128, 128, 500, 8), (128, 16, 129, 4)])
def test_time_segments(d_k, d_v, T, segments, dtype):
    """Cut into segments: the same results, with a given state and ragged lengths that end inside and before a segment."""
    inputs = make(3, 1, 2, T, d_k, d_v, dtype, seed=T + d_k, rate=0.05)
    lengths = torch.tensor([T, T // 2 + 3, 0], device="cuda", dtype=torch.int32)
    check(inputs, dtype, segments=segments, lengths=lengths)
    check((*inputs[:5], None), dtype, segments=segments)
    whole = vla.gated_delta_forward(*inputs, segments=1)
    cut = vla.gated_delta_forward(*inputs, segments=segments)
    close(cut[1], whole[1].double(), 2 * TOL["f32"], "S_T against one segment")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("segments", [1, 3])
def test_a_nan_reaches_back_no_further_than_its_tile(dtype, segments):
    """Outputs up to the 16 tokens that a NaN lies in, and those of other heads and sequences, do not change at all."""
    clean = make(2, 2, 4, 300, 64, 64, dtype, seed=21)
    o, S = vla.gated_delta_forward(*clean, segments=segments)
    for which, place in ((0, (1, 1, 150)), (1, (1, 1, 150)), (2, (1, 2, 150)), (3, (1, 2, 150)), (4, (1, 2, 150))):
        inputs = [x.clone() for x in clean]
        inputs[which][place] = float("nan")
        o2, S2 = vla.gated_delta_forward(*inputs, segments=segments)
        assert torch.equal(o2[0], o[0]) and torch.equal(o2[1, :2], o[1, :2]) and torch.equal(S2[1, :2], S[1, :2]) and torch.equal(S2[0], S[0])
        assert torch.equal(o2[1, 2, :144], o[1, 2, :144])
        assert o2[1, 2, 150].isnan().any()
        if which in (2, 3, 4):
            assert torch.equal(o2[1, 3], o[1, 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_start_anywhere(dtype):
    """Contiguous tensors that do not start at a 16-byte boundary, over tokens and for one."""
    inputs = make(2, 2, 2, 40, 32, 32, dtype, seed=22)
    moved = []
    for x in inputs[:3]:
        room = torch.empty(x.numel() + 3, dtype=x.dtype, device="cuda")
        moved.append(room[3:].view(x.shape).copy_(x))
    o, S = vla.gated_delta_forward(*inputs)
    o2, S2 = vla.gated_delta_forward(*moved, *inputs[3:])
    assert torch.equal(o, o2) and torch.equal(S, S2)
    one = [x[:, :, 0].contiguous() for x in inputs[:5]]
    odd = []
    for x in one[:3]:
        room = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        odd.append(room[1:].view(x.shape).copy_(x))
    a, b = S.clone(), S.clone()
    assert torch.equal(vla.gated_delta_decode_step(*one, a), vla.gated_delta_decode_step(*odd, *one[3:], b)) and torch.equal(a, b)


def test_a_scale_of_zero_is_refused():
    q, k, v, g, beta, S0 = make(1, 1, 1, 3, 16, 16, "f32", seed=23)
    with pytest.raises(ValueError, match="scale"):
        vla.gated_delta_forward(q, k, v, g, beta, S0, scale=0.0)
    with pytest.raises(ValueError, match="scale"):
        vla.gated_delta_decode_step(*(x[:, :, 0] for x in (q, k, v, g, beta)), S0, scale=0)

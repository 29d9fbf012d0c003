"""The operators on rows of channels as programs use them: one after the other in a layer, trained, over a prompt and token by token; in graphs that
are replayed; on other streams, two calls at once; with rows far apart; without memory beyond the caller's (GPU)."""
import ctypes
import threading

import pytest
import torch
import torch.nn.functional as F

import mixer_reference as ref
import paper_2605_11196_amd as vla
from paper_2605_11196_amd.binding import VlaConvOpts, VlaResidualOpts, VlaScanOpts

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- a layer

B, T, WIDTH, CHANNELS, N, TAPS = 3, 40, 64, 128, 16, 4


def parameters(seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    lin = lambda o, i: r(o, i) / i ** 0.5
    return dict(norm=1 + 0.1 * r(WIDTH), w_in=lin(2 * CHANNELS, WIDTH), conv=lin(CHANNELS, TAPS), conv_bias=0.1 * r(CHANNELS),
                w_delta=lin(CHANNELS, CHANNELS), w_bc=lin(2 * N, CHANNELS), A=-torch.arange(1, N + 1).float() * torch.exp(0.2 * r(CHANNELS, N)), D=r(CHANNELS),
                delta_bias=r(CHANNELS) - 3, w_out=lin(WIDTH, CHANNELS), post=1 + 0.1 * r(WIDTH), scale=0.5 + 0.1 * r(WIDTH), last=1 + 0.1 * r(WIDTH))


def layer(p, x, window, h0):
    """(the stream, its norm, the window, the state) behind a norm, the mixer, and the norms that follow it."""
    _, a = vla.residual_norm(x, None, p["norm"])
    a, z = F.linear(a, p["w_in"]).split(CHANNELS, -1)
    a, window = vla.causal_conv(a, p["conv"], p["conv_bias"], window)
    Bm, Cm = F.linear(a, p["w_bc"]).split(N, -1)
    y, h = vla.selective_scan(a, F.linear(a, p["w_delta"]), p["A"], Bm, Cm, p["D"], z, h0, delta_bias=p["delta_bias"])
    s, out = vla.residual_norm(x, F.linear(y, p["w_out"]), p["last"], post_weight=p["post"], groups=2, scale=p["scale"])
    return s, out, window, h


def token(p, x, window, h):
    """layer() of one token x [B, WIDTH]; the window and the state move on in place."""
    _, a = vla.residual_norm(x[:, None], None, p["norm"])
    a, z = F.linear(a[:, 0], p["w_in"]).split(CHANNELS, -1)
    a = vla.causal_conv_step(a, p["conv"], window, p["conv_bias"])
    Bm, Cm = F.linear(a, p["w_bc"]).split(N, -1)
    y = vla.selective_scan_step(a, F.linear(a, p["w_delta"]), p["A"], Bm, Cm, h, p["D"], z, delta_bias=p["delta_bias"])
    s, out = vla.residual_norm(x[:, None], F.linear(y, p["w_out"])[:, None], p["last"], post_weight=p["post"], groups=2, scale=p["scale"])
    return s[:, 0], out[:, 0]


def plain_layer(p, x, window, h0):
    _, a = ref.residual(x, None, p["norm"], None, 1, None, "silu", None, 1e-6)
    a, z = F.linear(a, p["w_in"]).split(CHANNELS, -1)
    rows = torch.cat((window, a), 1)
    pre = sum(p["conv"][:, j] * rows[:, j:j + a.shape[1]] for j in range(TAPS)) + p["conv_bias"]
    a, window = pre * torch.sigmoid(pre), rows[:, -(TAPS - 1):]
    Bm, Cm = F.linear(a, p["w_bc"]).split(N, -1)
    dt, h, y = F.softplus(F.linear(a, p["w_delta"]) + p["delta_bias"], threshold=100), h0, []
    for t in range(a.shape[1]):
        h = torch.exp(dt[:, t, :, None] * p["A"]) * h + (dt[:, t] * a[:, t])[..., None] * Bm[:, t, None]
        y.append((h * Cm[:, t, None]).sum(-1))
    y = (torch.stack(y, 1) + p["D"] * a) * z * torch.sigmoid(z)
    s, out = ref.residual(x, F.linear(y, p["w_out"]), p["last"], p["post"], 2, None, "silu", p["scale"], 1e-6)
    return s, out, window, h


def inputs(seed=1):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=gen) for s in ((B, T, WIDTH), (B, TAPS - 1, CHANNELS), (B, CHANNELS, N))]


def near(got, truth, plain, what):
    """`plain` makes the same sums of the same terms in float32, one after the other or in another order, and each of its steps rounds as often; the errors of
    both are made of independent roundings of the same sizes, so that their norms differ by a small factor: 4 holds the order of sums, one step instead of
    half of one in the exponentials, and an exponent's own rounding.  2^-22 of the norm is for results that `plain` has by chance."""
    error = lambda x: (x.detach().double().cpu() - truth).norm()
    assert error(got) <= 4 * error(plain) + 2.0 ** -22 * truth.norm(), (what, float(error(got)), float(error(plain)), float(truth.norm()))


def test_a_layer_over_a_prompt_in_pieces_token_by_token_and_its_gradients():
    p, given = parameters(), inputs()
    gen = torch.Generator().manual_seed(2)
    grads = [torch.randn(s, generator=gen) for s in ((B, T, WIDTH), (B, T, WIDTH), (B, TAPS - 1, CHANNELS), (B, CHANNELS, N))]

    def run(f, move):
        leaves = [move(x).requires_grad_() for x in (*given, *p.values())]
        out = f(dict(zip(p, leaves[3:])), *leaves[:3])
        return [o.detach() for o in out], torch.autograd.grad(out, leaves, [move(g) for g in grads])

    truth, plain, ours = run(plain_layer, torch.Tensor.double), run(plain_layer, torch.Tensor.clone), run(layer, torch.Tensor.cuda)
    names = ("s", "out", "window", "h"), ("dx", "dwindow", "dh0", *("d" + k for k in p))
    for kind in range(2):
        for name, g, t, q in zip(names[kind], ours[kind], truth[kind], plain[kind]):
            near(g, t, q, name)
    p = {k: v.cuda() for k, v in p.items()}
    x, window, h = (v.cuda() for v in given)
    with torch.no_grad():
        first, second = x[:, :13], x[:, 13:]
        a = layer(p, first, window, h)
        b = layer(p, second, *a[2:])
        pieces = [torch.cat((a[0], b[0]), 1), torch.cat((a[1], b[1]), 1), b[2], b[3]]
        window, h = window.clone(), h.clone()
        steps = [token(p, x[:, t], window, h) for t in range(T)]
        steps = [torch.stack([v[i] for v in steps], 1) for i in range(2)] + [window, h]
    for way in (pieces, steps):
        for name, g, t, q in zip(names[0], way, truth[0], plain[0]):
            near(g, t, q, name)


def test_beside_the_gated_delta_rule():
    """The convolution before the delta rule's heads and the gated norm of each head behind it, a gradient through all of them: what is read through views
    gives the same bits as contiguous copies."""
    heads, d = 4, 32
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(s, generator=gen).bfloat16().cuda()
    wide, weight, post = r(2, 50, 4 * heads * d).requires_grad_(), r(3 * heads * d, 4).requires_grad_(), (1 + 0.1 * r(heads * d)).requires_grad_()
    g, beta = (-0.1 * torch.rand(2, heads, 50, generator=gen)).cuda(), torch.rand(2, heads, 50, generator=gen).cuda()

    def run(lay):
        rows, gate = wide.split((3 * heads * d, heads * d), -1)
        rows = vla.causal_conv(lay(rows), weight)[0]
        q, k, v = (lay(x.unflatten(-1, (heads, d)).transpose(1, 2)) for x in rows.split(heads * d, -1))
        o = vla.gated_delta(q, F.normalize(k.float(), dim=-1).bfloat16(), v, g, beta)[0]
        out = vla.residual_norm(None, o.transpose(1, 2).flatten(2), None, post_weight=post, groups=heads, gate=lay(gate))[0]
        return [out.detach(), *torch.autograd.grad(out.float().square().sum(), (wide, weight, post))]

    views, copies = run(lambda x: x), run(torch.Tensor.contiguous)
    assert all(torch.isfinite(x).all() and torch.equal(x, y) for x, y in zip(views, copies))


# ---- all entry points on one set of inputs

def everything(dtype="bf16", seed=5, T=300, n=264):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    io = lambda *s: r(*s).to(DT[dtype]).cuda()
    return dict(x=io(2, T, n), u=io(2, T, n), z=io(2, T, n), delta=io(2, T, n), B=io(2, T, N), C=io(2, T, N), A=(-torch.rand(n, N, generator=gen) - 0.1).cuda(),
                D=r(n).cuda(), bias=(r(n) - 3).cuda(), h0=r(2, n, N).cuda(), weight=io(n, 4), window=io(2, 3, n), w=io(n), w1=io(n), k=io(n), dy=io(2, T, n),
                dh=r(2, n, N).cuda(), lengths=torch.tensor([T, T // 2], dtype=torch.int32).cuda())


def calls(s, stream=None):
    kw = dict(lengths=s["lengths"], stream=stream)
    y, window = vla.causal_conv(s["x"], s["weight"], s["w"], s["window"], **kw)
    args = [s[k] for k in ("u", "delta", "A", "B", "C", "D", "z")]
    o, h, saved = vla.selective_scan_forward(*args, s["h0"], delta_bias=s["bias"], save_for_backward=True, **kw)
    norm = dict(post_weight=s["w1"], groups=3, gate=s["z"], scale=s["k"], stream=stream)
    r, q = vla.residual_norm(s["x"], s["u"], s["w"], **norm)
    return [y, window, o, h, r, q, *vla.causal_conv_backward(s["x"], s["weight"], s["w"], s["window"], s["dy"], s["window"], **kw),
            *vla.selective_scan_backward(*args, saved, s["dy"], s["dh"], delta_bias=s["bias"], **kw),
            *vla.residual_norm_backward(s["x"], s["u"], s["w"], s["dy"], s["x"], **norm)]


def differentiated(s):
    leaf = {k: v.detach().requires_grad_() if v.is_floating_point() else v for k, v in s.items()}
    y, window = vla.causal_conv(leaf["x"], leaf["weight"], leaf["w"], leaf["window"], lengths=s["lengths"])
    o, h = vla.selective_scan(*(leaf[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "h0")), delta_bias=leaf["bias"], lengths=s["lengths"])
    r, q = vla.residual_norm(leaf["x"], leaf["u"], leaf["w"], post_weight=leaf["w1"], groups=3, gate=leaf["z"], scale=leaf["k"])
    out = y, window, o, h, r, q
    return [x.detach() for x in out] + [
        *torch.autograd.grad((y, window), [leaf[k] for k in ("x", "weight", "w", "window")], (s["dy"], s["window"])),
        *torch.autograd.grad((o, h), [leaf[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "bias", "h0")], (s["dy"], s["dh"])),
        *torch.autograd.grad((r, q), [leaf[k] for k in ("x", "u", "w", "w1", "z", "k")], (s["dy"], s["x"]))]


def same(got, want):
    return len(got) == len(want) and all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_on_another_stream_and_through_autograd(dtype):
    s = everything(dtype)
    want = calls(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = calls(s, side)
    by_handle = calls(s, side.cuda_stream)
    with torch.cuda.stream(side):
        also = differentiated(s)
    torch.cuda.current_stream().wait_stream(side)
    assert same(got, want) and same(also, want) and same(by_handle, want)


def test_steps_on_another_stream():
    s = everything()
    one = {k: s[k][:, 0] for k in ("x", "u", "delta", "B", "C", "z")}

    def run(stream):
        window, h = s["window"].clone(), s["h0"].clone()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        out = []
        for _ in range(3):
            out.append(vla.causal_conv_step(one["x"], s["weight"], window, s["w"], stream=stream))
            out.append(vla.selective_scan_step(one["u"], one["delta"], s["A"], one["B"], one["C"], h, s["D"], one["z"], delta_bias=s["bias"], stream=stream))
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        return [*out, window, h]

    assert same(run(torch.cuda.Stream()), run(None))


def test_two_threads_at_once():
    sets = [everything(seed=11, T=700), everything("f32", seed=12, T=90, n=72)]
    want = [calls(s) for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    got = calls(sets[i])
                    stream.synchronize()
                    if not same(got, want[i]):
                        wrong.append(i)
        except Exception as e:      # an assertion in a thread is not seen
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_repeated_call_may_have_tensors_that_start_anywhere():
    s = everything("f32", T=17)
    want = calls(s)

    def moved(x):
        room = torch.empty(x.numel() + 1, device="cuda", dtype=x.dtype)
        return room[1:].view(x.shape).copy_(x)

    for k in s:
        if k != "lengths":
            assert same(calls(dict(s, **{k: moved(s[k])})), want), k
    wide = torch.stack((s["lengths"], s["lengths"]), 1)
    assert same(calls(dict(s, lengths=wide[:, 0])), want)
    state = moved(s["window"])
    with pytest.raises(ValueError, match="16-byte"):
        vla.causal_conv_step(s["x"][:, 0], s["weight"], state, s["w"])
    with pytest.raises(ValueError, match="16-byte"):
        vla.selective_scan_step(s["u"][:, 0], s["delta"][:, 0], s["A"], s["B"][:, 0], s["C"][:, 0], moved(s["h0"]), s["D"])


# ---- graphs

def captured(f):
    """f() in a graph, after it ran eagerly on the stream that captures."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    return graph, out


@pytest.mark.parametrize("f", [calls, differentiated])
def test_forward_and_backward_in_graphs(f):
    """Two graphs, replayed in turn on new data with eager calls and synchronisations between: their workspaces are their own."""
    s, other = everything(seed=21, T=700), everything("f32", seed=22, T=60, n=72)
    (graph, out), (graph2, out2) = captured(lambda: f(s)), captured(lambda: f(other))
    for i in range(4):
        for now, seed, dtype, T, n in ((s, 31 + i, "bf16", 700, 264), (other, 41 + i, "f32", 60, 72)):
            for k, v in everything(dtype, seed=seed, T=T, n=n).items():
                now[k].copy_(v)
        graph.replay()
        graph2.replay()
        want, want2 = calls(s), calls(other)
        torch.cuda.synchronize()
        assert same(out, want) and same(out2, want2), i
        graph2.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want) and same(out2, want2), i


def test_tokens_in_a_graph():
    p = {k: v.cuda() for k, v in parameters().items()}
    x, window, h = (v.cuda() for v in inputs())
    now, eager = (x[:, 0].clone(), window.clone(), h.clone()), (window.clone(), h.clone())
    graph, out = captured(lambda: token(p, *now))
    now[1].copy_(window)
    now[2].copy_(h)
    for t in range(6):
        now[0].copy_(x[:, t])
        graph.replay()
        want = token(p, x[:, t], *eager)
        torch.cuda.synchronize()
        assert same([*out, *now[1:]], [*want, *eager]), t


# ---- rows far apart

def test_offsets_that_pass_32_bits():
    """A sequence that starts 2^31 elements behind the other, and tokens 2^16 apart that pass 2^31: as contiguous copies."""
    n, room = 72, torch.empty(2 ** 31 + 2 ** 24, dtype=torch.bfloat16, device="cuda")
    for size, steps in (((2, 9, n), (2 ** 31, 128, 1)), ((1, 33000, n), (0, 2 ** 16, 1))):
        far = room.as_strided(size, steps)
        s = everything(T=size[1], n=n)
        s = {k: v[:size[0]].contiguous() if v.dim() == 3 else v for k, v in s.items()}
        s["lengths"] = s["lengths"][:size[0]]
        want = calls(s)
        for k in ("x", "u", "z", "delta", "dy"):
            far.copy_(s[k])
            got = calls(dict(s, **{k: far}))
            assert same(got, want), (k, size)


# ---- memory

def test_the_entry_points_allocate_nothing():
    """The device's free memory before and after calls with the caller's buffers alone (a first call may load code)."""
    lib, stream, io, T, n = vla.load_library(), torch.cuda.current_stream().cuda_stream, vla.VLA_BF16, 700, 264
    s = everything(T=T, n=n)
    s["w"], s["w1"], s["k"], s["weight"] = (s[k].float() for k in ("w", "w1", "k", "weight"))
    out = {k: torch.empty_like(v) for k, v in s.items()}
    rows = [torch.empty_like(s["x"]) for _ in range(3)]
    p = lambda *names, of=s: [of[k].data_ptr() for k in names]
    scan, conv, norm = VlaScanOpts(1, 1), VlaConvOpts(1), VlaResidualOpts(eps=1e-6, stream_dtype=io)
    kept = lib.vla_selective_scan_saved_bytes(2, T, n, N, io, ctypes.byref(scan))
    saved = torch.empty(kept, dtype=torch.uint8, device="cuda")
    scan.saved, scan.saved_bytes = saved.data_ptr(), kept
    sizes = [lib.vla_selective_scan_workspace_bytes(2, T, n, N, io, ctypes.byref(scan), back) for back in (0, 1)]
    sizes += [lib.vla_causal_conv_workspace_bytes(2, T, n, 4, io), lib.vla_residual_norm_workspace_bytes(n)]
    assert min(sizes) > 0      # long sequences of few channels: cut into segments
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    y, h, extra = rows[0].data_ptr(), out["h0"].data_ptr(), rows[1].data_ptr()
    given = p("u", "delta", "A", "B", "C", "D", "z", "bias")
    grad = lambda *names: p(*names, of=out)

    def run():
        rc = lib.vla_causal_conv(*p("x", "weight", "w", "window"), y, *grad("window"), 2, T, n, 4, io, ctypes.byref(conv), stream)
        rc |= lib.vla_causal_conv_backward(*p("x", "weight", "w", "window", "dy"), None, *grad("x", "weight", "w", "window"), 2, T, n, 4, io, ctypes.byref(conv),
                                           ws.data_ptr(), sizes[2], stream)
        rc |= lib.vla_causal_conv_step(*p("x", "weight", "w"), *grad("window"), y, 2, n, 4, io, None, stream)
        rc |= lib.vla_selective_scan(*given, *p("h0"), y, h, 2, T, n, N, io, ctypes.byref(scan), ws.data_ptr(), sizes[0], stream)
        rc |= lib.vla_selective_scan_backward(*given, *p("dy", "dh"), *grad("u", "delta", "A", "B", "C", "D", "z", "bias"), h, 2, T, n, N, io, ctypes.byref(scan),
                                              ws.data_ptr(), sizes[1], stream)
        rc |= lib.vla_selective_scan_step(*given, h, y, 2, n, N, io, None, stream)
        rc |= lib.vla_residual_norm(*p("x", "u", "z", "w1", "k", "w"), y, extra, 2, T, n, io, ctypes.byref(norm), stream)
        rc |= lib.vla_residual_norm_backward(*p("x", "u", "z", "w1", "k", "w", "dy", "dy"), *grad("x", "u", "z", "w1", "k", "w"), 2, T, n, io,
                                             ctypes.byref(norm), ws.data_ptr(), sizes[3], stream)
        torch.cuda.synchronize()
        return rc

    assert run() == 0
    free = torch.cuda.mem_get_info()[0]
    for _ in range(20):
        assert run() == 0
    assert torch.cuda.mem_get_info()[0] == free

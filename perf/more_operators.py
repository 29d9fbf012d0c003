"""The selective state space scan, its short causal convolution, and the norms around a block with its gate and residual scale, as
cases to time: each operator over whole sequences, in training (forward and backward), and the recurrent ones for one token.

A case is a dict: kind ("conv", "conv_train", "conv_step", "scan", "scan_train", "scan_step", "norm" or "norm_train"), B, T (tokens),
n (channels, columns), dtype ("f32" or "bf16") and the choices of that kind.
"""
import math

import torch

own = False   # false: the plain forms below; true: this repository's kernels

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64    # tokens of a step of the plain scan
EPS = 1e-6


def _conv(kind, B, n, dtype, *, T=1, width=4, bias=True, silu=True, carried=False, ragged=False, name=None):
    c = dict(kind=kind, B=B, T=T, n=n, dtype=dtype, width=width, bias=bias, silu=silu, carried=carried, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _scan(kind, B, n, N, dtype, *, T=1, groups=1, gate=True, carried=False, ragged=False, name=None):
    c = dict(kind=kind, B=B, T=T, n=n, N=N, groups=groups, dtype=dtype, gate=gate, carried=carried, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _norm(kind, B, T, n, dtype, *, stream="same", post=False, groups=1, gate="none", scale=False, pre=True, name=None):
    c = dict(kind=kind, B=B, T=T, n=n, dtype=dtype, stream=stream, post=post, groups=groups, gate=gate, scale=scale, pre=pre)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # generation: the window of 64 sequences moves on by a token
        _conv("conv_step", 64, 4096, "bf16", carried=True, name="conv_token"),
        # prefill of one long prompt: half of a fused projection
        _conv("conv", 1, 2048, "bf16", T=16384, name="conv_prefill"),
        # training: sequences of unequal lengths that continue earlier ones, float32
        _conv("conv_train", 3, 1664, "f32", T=1537, carried=True, ragged=True, name="conv_train_ragged"),
        # training: a large batch
        _conv("conv_train", 8, 4096, "bf16", T=8192, name="conv_train_large"),
        # generation for one sequence: a launch and the host path
        _scan("scan_step", 1, 1024, 16, "bf16", name="scan_token_few"),
        # generation for a serving batch: the states of 64 sequences through memory once
        _scan("scan_step", 64, 4096, 16, "bf16", name="scan_token_batch"),
        # one long prompt
        _scan("scan", 1, 2048, 16, "bf16", T=32768, name="scan_long"),
        # training: unequal lengths, two groups of wide states that continue earlier ones, float32
        _scan("scan_train", 3, 1664, 32, "f32", T=1537, groups=2, carried=True, ragged=True, name="scan_train_ragged"),
        # training: an ordinary batch
        _scan("scan_train", 8, 4096, 16, "bf16", T=2048, name="scan_train"),
        # generation: what follows a block and precedes the next, 64 sequences, the residual stream in float32
        _norm("norm", 64, 1, 4096, "bf16", stream="f32", post=True, scale=True, name="norm_token"),
        # training: a gated norm for each of 13 heads, no residual, float32
        _norm("norm_train", 3, 1537, 1664, "f32", stream="none", post=True, groups=13, gate="silu", pre=False, name="norm_train_heads"),
        # training: norms on both sides of a gated block, a large batch
        _norm("norm_train", 8, 4096, 4096, "bf16", post=True, gate="silu", scale=True, name="norm_train_large"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("conv", "conv_train", "conv_step", "scan", "scan", "scan_train", "scan_train", "scan_step", "norm", "norm_train"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    B, n = _log(rng, 1, 64), 8 * _log(rng, 8, 512)
    opt = dict(carried=rng.random() < 0.4, ragged=rng.random() < 0.25)
    half = 2 if dtype == "f32" else 1
    if kind.startswith("conv"):
        opt.update(width=rng.choice((2, 3, 4, 4)), bias=rng.random() < 0.7, silu=rng.random() < 0.7)
        if kind == "conv_step":
            return _conv(kind, B, n, dtype, **dict(opt, carried=True, ragged=False))
        return _conv(kind, B, n, dtype, T=max(1, min(_log(rng, 1, 32768), 2 ** 27 // (half * B * n))), **opt)
    if kind.startswith("scan"):
        N, groups = rng.choice((8, 16, 16, 16, 32, 64)), rng.choice((1, 1, 2, 4))
        if n % (8 * groups):
            groups = 1
        opt.update(groups=groups, gate=rng.random() < 0.7)
        if kind == "scan_step":
            return _scan(kind, B, n, N, dtype, **dict(opt, carried=True, ragged=False))
        longest, most = (32768, 2 ** 30) if kind == "scan" else (8192, 2 ** 29)
        return _scan(kind, B, n, N, dtype, T=max(1, min(_log(rng, 1, longest), most // (half * B * n * N))), **opt)
    post, gate, stream = rng.random() < 0.6, rng.choice(("none", "silu", "sigmoid")), rng.choice(("none", "same", "same", "f32"))
    groups = n // rng.choice([g for g in (32, 64, 96, 128, n, n) if n % g == 0]) if post else 1
    return _norm(kind, B, max(1, min(_log(rng, 1, 16384), 2 ** 26 // (half * B * n))), n, dtype, stream=stream, post=post, groups=groups,
                 gate=gate, scale=rng.random() < 0.5, pre=stream != "none" or not post)


# ---- inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _lengths(case, gen):
    if not case["ragged"]:
        return None
    return torch.randint(0, case["T"] + 1, (case["B"],), generator=gen, device="cuda", dtype=torch.int32)


def _prepare_conv(case, gen, dtype):
    B, T, n, W = (case[k] for k in ("B", "T", "n", "width"))
    x = _randn(gen, B, T, 2 * n).to(dtype)[:, :, :n]       # the first half of a fused projection, the gate is the other one
    weight = ((2 * torch.rand((n, W), generator=gen, device="cuda") - 1) * W ** -0.5).to(dtype)
    bias = ((2 * torch.rand((n,), generator=gen, device="cuda") - 1) * W ** -0.5).to(dtype) if case["bias"] else None
    state = _randn(gen, B, W - 1, n).to(dtype) if case["carried"] else None
    s = dict(case=case, x=x, weight=weight, bias=bias, state=state, lengths=_lengths(case, gen))
    if case["kind"] == "conv_step":
        s["x"] = x[:, 0]
    if case["kind"] == "conv_train":
        s["grads"] = [_randn(gen, B, T, n).to(dtype), _randn(gen, B, W - 1, n).to(dtype)]
        s["leaves"] = {k: s[k].detach().requires_grad_() for k in ("x", "weight", "bias", "state") if s[k] is not None}
    return s


def _prepare_scan(case, gen, dtype):
    B, T, n, N, G = (case[k] for k in ("B", "T", "n", "N", "groups"))
    rank = 8 * max(1, n // 128)
    u = torch.nn.functional.silu(_randn(gen, B, T, n)).to(dtype)
    # steps: a bias that spreads them from 1e-3 to 1e-1 between the channels, and a projection's values around it
    step = torch.exp(math.log(1e-3) + torch.rand((n,), generator=gen, device="cuda") * math.log(1e2))
    delta_bias = step + torch.log(-torch.expm1(-step))
    delta = (0.7 * _randn(gen, B, T, n)).to(dtype)
    # rates 1 to N in every channel, as they are initialised, moved by training
    A = -torch.arange(1, N + 1, device="cuda") * torch.exp(0.1 * _randn(gen, n, N))
    rows = _randn(gen, B, T, rank + 2 * G * N).to(dtype)   # slices of one projection: what delta comes from, B, C
    Bm, Cm = (rows[:, :, rank + i * G * N:rank + (i + 1) * G * N].unflatten(-1, (G, N)) for i in range(2))
    D = 1 + 0.1 * _randn(gen, n)
    z = _randn(gen, B, T, 2 * n).to(dtype)[:, :, n:] if case["gate"] else None
    h = 0.1 * _randn(gen, B, n, N) if case["carried"] or case["kind"] == "scan_step" else None
    s = dict(case=case, u=u, delta=delta, A=A, B=Bm, C=Cm, D=D, z=z, delta_bias=delta_bias, h=h, lengths=_lengths(case, gen))
    if case["kind"] == "scan_step":
        s.update({k: s[k][:, 0] for k in ("u", "delta", "B", "C", "z") if s[k] is not None})
    if case["kind"] == "scan_train":
        s["grads"] = [_randn(gen, B, T, n).to(dtype), 0.1 * _randn(gen, B, n, N)]
        s["leaves"] = {k: s[k].detach().requires_grad_() for k in ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "h") if s[k] is not None}
    return s


def _prepare_norm(case, gen, dtype):
    B, T, n = (case[k] for k in ("B", "T", "n"))
    y = _randn(gen, B, T, n).to(dtype)
    x = None if case["stream"] == "none" else (3 * _randn(gen, B, T, n)).to(torch.float32 if case["stream"] == "f32" else dtype)
    gate = _randn(gen, B, T, 2 * n).to(dtype)[:, :, n:] if case["gate"] != "none" else None
    weight, post_weight = ((1 + 0.1 * _randn(gen, n)).to(dtype) if case[k] else None for k in ("pre", "post"))
    scale = (0.1 + 0.05 * _randn(gen, n)).to(dtype) if case["scale"] else None
    s = dict(case=case, x=x, y=y, gate=gate, weight=weight, post_weight=post_weight, scale=scale)
    if case["kind"] == "norm_train":
        s["grads"] = [_randn(gen, B, T, n).to(y.dtype if x is None else x.dtype)] + ([_randn(gen, B, T, n).to(dtype)] if case["pre"] else [])
        s["leaves"] = {k: s[k].detach().requires_grad_() for k in ("x", "y", "gate", "weight", "post_weight", "scale") if s[k] is not None}
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"].split("_")[0]
    return {"conv": _prepare_conv, "scan": _prepare_scan, "norm": _prepare_norm}[kind](case, gen, DTYPES[case["dtype"]])


# ---- plain forms

def _live(lengths, T):
    return torch.arange(T, device=lengths.device)[None, :, None] < lengths[:, None, None]


def _plain_conv(x, weight, bias, state, lengths, silu):
    """Windows of the sequence with the carried tokens before it, times the weights."""
    (B, T, n), W, dtype = x.shape, weight.shape[1], x.dtype
    before = torch.zeros((B, W - 1, n), device=x.device) if state is None else state.float()
    rows = torch.cat((before, x.float()), 1)
    y = (rows.unfold(1, W, 1) * weight.float()).sum(-1)
    if bias is not None:
        y = y + bias.float()
    if silu:
        y = y * torch.sigmoid(y)
    if lengths is None:
        return y.to(dtype), rows[:, T:].to(dtype)
    last = lengths.long()[:, None, None] + torch.arange(W - 1, device=x.device)[None, :, None]
    return torch.where(_live(lengths, T), y, 0.0).to(dtype), rows.take_along_dim(last.expand(B, W - 1, n), 1).to(dtype)


def _scanned(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from zero, by doubling."""
    s = 1
    while s < a.shape[1]:
        b = torch.cat((b[:, :s], b[:, s:] + a[:, s:] * b[:, :-s]), 1)
        a = torch.cat((a[:, :s], a[:, s:] * a[:, :-s]), 1)
        s *= 2
    return b


def _plain_scan(s, grads=None):
    """Chunks of 64 tokens; the state passes from chunk to chunk.  The gradients by the recurrence in reverse, chunk by chunk."""
    u, delta, A, Bm, Cm, D, z, bias, h, lengths = (s[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "h", "lengths"))
    dtype, (B, T, n), N, share = u.dtype, u.shape, A.shape[1], u.shape[2] // Bm.shape[2]
    live = None if lengths is None else _live(lengths, T)
    kept = lambda x: x if live is None else torch.where(live, x, 0.0)
    u, raw = kept(u.float()), delta.float() + bias
    dt = kept(torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20)))))
    Bm, Cm = Bm.float(), Cm.float()
    of_channels = lambda x: x.repeat_interleave(share, 2)                 # [B, tokens, G, N] -> [B, tokens, n, N]
    h = torch.zeros((B, n, N), device=u.device) if h is None else h
    y, starts = [], []
    for t in range(0, T, CHUNK):
        c = slice(t, t + CHUNK)
        a = torch.exp(dt[:, c, :, None] * A)
        b = (dt[:, c] * u[:, c]).unsqueeze(-1) * of_channels(Bm[:, c])
        b[:, 0] += a[:, 0] * h
        starts.append(h)
        b = _scanned(a, b)
        h = b[:, -1]
        y.append((b * of_channels(Cm[:, c])).sum(-1))
    inner = torch.cat(y, 1) + D * u
    out = inner
    if z is not None:
        z = z.float()
        sig = torch.sigmoid(z)
        out = inner * z * sig
    result = [kept(out).to(dtype), h]
    if grads is None:
        return tuple(result)
    dy, G = kept(grads[0].float()), grads[1]
    dz = None
    if z is not None:
        dz = kept(dy * inner * sig * (1 + z * (1 - sig)))
        dy = dy * z * sig
    dA = torch.zeros_like(A)
    du, ddt, dB, dC = [], [], [], []
    of_groups = lambda x: x.unflatten(2, (-1, share)).sum(3)
    for t in range((T - 1) // CHUNK * CHUNK, -1, -CHUNK):
        c = slice(t, t + CHUNK)
        a, Bc, Cc, start = torch.exp(dt[:, c, :, None] * A), of_channels(Bm[:, c]), of_channels(Cm[:, c]), starts.pop()
        b = (dt[:, c] * u[:, c]).unsqueeze(-1) * Bc
        b[:, 0] += a[:, 0] * start
        hs = _scanned(a, b)
        g = dy[:, c].unsqueeze(-1) * Cc
        g[:, -1] += G
        dC.append(of_groups(dy[:, c].unsqueeze(-1) * hs))
        g = _scanned(torch.cat((torch.zeros_like(a[:, :1]), a.flip(1)[:, :-1]), 1), g.flip(1)).flip(1)
        G = a[:, 0] * g[:, 0]
        decayed = a * torch.cat((start.unsqueeze(1), hs[:, :-1]), 1) * g
        inward = (g * Bc).sum(-1)
        du.append(D * dy[:, c] + dt[:, c] * inward)
        ddt.append((decayed * A).sum(-1) + u[:, c] * inward)
        dA += (decayed * dt[:, c, :, None]).sum((0, 1))
        dB.append(of_groups(g * (dt[:, c] * u[:, c]).unsqueeze(-1)))
    whole = lambda parts: torch.cat(parts[::-1], 1)
    draw = kept(whole(ddt) * torch.sigmoid(raw))
    result += [kept(whole(du)).to(dtype), draw.to(dtype), dA, whole(dB).to(dtype), whole(dC).to(dtype), (dy * u).sum((0, 1))]
    if z is not None:
        result.append(dz.to(dtype))
    result.append(draw.sum((0, 1)))
    return result + ([] if s["h"] is None else [G])


def _plain_scan_step(s):
    u, delta, A, Bm, Cm, D, z, h = (s[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "h"))
    share, raw, x = u.shape[1] // Bm.shape[1], delta.float() + s["delta_bias"], u.float()
    dt = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))
    Bm, Cm = (v.float().repeat_interleave(share, 1) for v in (Bm, Cm))
    h = torch.exp(dt.unsqueeze(-1) * A) * h + (dt * x).unsqueeze(-1) * Bm
    y = (h * Cm).sum(-1) + D * x
    if z is not None:
        y = y * z.float() * torch.sigmoid(z.float())
    return y.to(u.dtype), h


def _plain_norm(x, y, gate, weight, post_weight, scale, groups, activation):
    t = y.float()
    if post_weight is not None:
        t = t.unflatten(-1, (groups, -1))
        t = (t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS)).flatten(-2) * post_weight.float()
    if gate is not None:
        g = gate.float()
        t = t * torch.sigmoid(g) * (g if activation == "silu" else 1.0)
    if scale is not None:
        t = t * scale.float()
    s = t if x is None else x.float() + t
    out = s.to(y.dtype if x is None else x.dtype)
    if weight is None:
        return (out,)
    return out, (s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * weight.float()).to(y.dtype)


# ---- one pass

def _pass_conv(s):
    args = s["x"], s["weight"], s["bias"], s["state"]
    if own:
        import paper_2605_11196_amd as vla

        return vla.causal_conv(*args, lengths=s["lengths"], activation="silu" if s["case"]["silu"] else None)
    return _plain_conv(*args, s["lengths"], s["case"]["silu"])


def _pass_scan(s):
    if own:
        import paper_2605_11196_amd as vla

        return vla.selective_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["h"], delta_bias=s["delta_bias"],
                                  lengths=s["lengths"])
    return _plain_scan(s)


def _pass_norm(s):
    c = s["case"]
    if own:
        import paper_2605_11196_amd as vla

        out, h = vla.residual_norm(s["x"], s["y"], s["weight"], post_weight=s["post_weight"], groups=c["groups"], gate=s["gate"],
                                   activation="sigmoid" if c["gate"] == "sigmoid" else "silu", scale=s["scale"], eps=EPS)
        return (out,) if h is None else (out, h)
    return _plain_norm(s["x"], s["y"], s["gate"], s["weight"], s["post_weight"], s["scale"], c["groups"], c["gate"])


def _pass_step(s):
    conv = s["case"]["kind"] == "conv_step"
    if own:
        import paper_2605_11196_amd as vla

        if conv:
            return vla.causal_conv_step(s["x"], s["weight"], s["state"], s["bias"], activation="silu" if s["case"]["silu"] else None), s["state"]
        return vla.selective_scan_step(s["u"], s["delta"], s["A"], s["B"], s["C"], s["h"], s["D"], s["z"], delta_bias=s["delta_bias"]), s["h"]
    kept = s["state" if conv else "h"]
    if conv:
        y, state = _plain_conv(s["x"].unsqueeze(1), s["weight"], s["bias"], kept, None, s["case"]["silu"])
        y = y[:, 0]
    else:
        y, state = _plain_scan_step(s)
    kept.copy_(state)
    return y, kept


def run(state):
    kind, way = state["case"]["kind"].split("_")[0], state["case"]["kind"].split("_")[-1]
    if way == "step":
        return _pass_step(state)
    forward = {"conv": _pass_conv, "scan": _pass_scan, "norm": _pass_norm}[kind]
    if way != "train":
        return forward(state)
    if kind == "scan" and not own:
        return _plain_scan(state, state["grads"])
    out = forward({**state, **state["leaves"]})
    return [o.detach() for o in out] + list(torch.autograd.grad(out, list(state["leaves"].values()), state["grads"]))


# ---- the definitions in 64 bits

def _exact_conv(s):
    """The taps one after the other; the gradients by the chain rule."""
    c = s["case"]
    B, T, n, W = (c[k] for k in ("B", "T", "n", "width"))
    x = s["x"].double().reshape(B, T, n)
    rows = torch.zeros((B, W - 1 + T, n), dtype=torch.float64, device="cuda")
    rows[:, W - 1:] = x
    if s["state"] is not None:
        rows[:, :W - 1] = s["state"].double()
    weight = s["weight"].double()
    pre = torch.zeros_like(x) if s["bias"] is None else s["bias"].double().expand(B, T, n).clone()
    for j in range(W):
        pre += weight[:, j] * rows[:, j:j + T]
    length = torch.full((B,), T) if s["lengths"] is None else s["lengths"].cpu()
    sig = 1 / (1 + torch.exp(-pre))
    y = pre * sig if c["silu"] else pre.clone()
    for b in range(B):
        y[b, length[b]:] = 0
    out = [y, torch.stack([rows[b, length[b]:length[b] + W - 1] for b in range(B)])]
    if c["kind"] != "conv_train":
        return out
    d = s["grads"][0].double()
    if c["silu"]:
        d = d * sig * (1 + pre * (1 - sig))
    for b in range(B):
        d[b, length[b]:] = 0
    back = torch.zeros_like(rows)
    for j in range(W):
        back[:, j:j + T] += weight[:, j] * d
    for b in range(B):
        back[b, length[b]:length[b] + W - 1] += s["grads"][1][b].double()
    out += [back[:, W - 1:], torch.stack([(d * rows[:, j:j + T]).sum((0, 1)) for j in range(W)], 1)]
    if s["bias"] is not None:
        out.append(d.sum((0, 1)))
    return out + ([] if s["state"] is None else [back[:, :W - 1]])


def _exact_scan(s):
    """Token by token."""
    c = s["case"]
    B, T, n, N, share = c["B"], c["T"], c["n"], c["N"], c["n"] // c["groups"]
    f = lambda k: None if s[k] is None else s[k].double().reshape(B, T, *s[k].shape[-(2 if k in "BC" else 1):])
    u, raw, Bm, Cm, z = f("u"), f("delta") + s["delta_bias"].double(), f("B"), f("C"), f("z")
    A, D = s["A"].double(), s["D"].double()
    length = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"]
    live = (torch.arange(T, device="cuda") < length[:, None]).double().unsqueeze(-1)
    dt = torch.logaddexp(raw, torch.zeros_like(raw)) * live
    h = torch.zeros((B, n, N), dtype=torch.float64, device="cuda") if s["h"] is None else s["h"].double()
    wide = lambda x: x[:, :, None].expand(B, c["groups"], share, N).reshape(B, n, N)
    train, kept, inner = c["kind"] == "scan_train", [], torch.empty_like(u)
    for t in range(T):
        if train:
            kept.append(h)
        h = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * u[:, t])[..., None] * wide(Bm[:, t])
        inner[:, t] = (h * wide(Cm[:, t])).sum(-1)
    inner += D * u
    gated = 1.0 if z is None else z / (1 + torch.exp(-z))
    out = [inner * gated * live, h.clone()]
    if not train:
        return out
    dy, g = s["grads"][0].double() * live, s["grads"][1].double().clone()
    d_inner = dy * gated
    du, ddt, dB, dC = d_inner * D, torch.zeros_like(u), torch.zeros_like(Bm), torch.zeros_like(Cm)
    dA = torch.zeros_like(A)
    for t in range(T - 1, -1, -1):
        before = kept.pop()
        wb = wide(Bm[:, t])
        dC[:, t] = (d_inner[:, t, :, None] * h).view(B, c["groups"], share, N).sum(2)
        g += d_inner[:, t, :, None] * wide(Cm[:, t])
        decay = torch.exp(dt[:, t, :, None] * A)
        dB[:, t] = (g * (dt[:, t] * u[:, t])[..., None]).view(B, c["groups"], share, N).sum(2)
        through = (g * wb).sum(-1)
        du[:, t] += dt[:, t] * through
        moved = g * before * decay
        ddt[:, t] = (moved * A).sum(-1) + u[:, t] * through
        dA += (moved * dt[:, t, :, None]).sum(0)
        g *= decay
        h = before
    draw = ddt * live / (1 + torch.exp(-raw))
    out += [du * live, draw, dA, dB * live[..., None], dC * live[..., None], (d_inner * u).sum((0, 1))]
    if z is not None:
        sig = 1 / (1 + torch.exp(-z))
        out.append(dy * inner * sig * (1 + z * (1 - sig)))
    out.append(draw.sum((0, 1)))
    return out + ([] if s["h"] is None else [g])


def _exact_norm(s):
    """Each factor on its own; the gradients by the chain rule."""
    c = s["case"]
    n, groups = c["n"], c["groups"]
    wide = lambda r: r.repeat_interleave(n // groups, -1)
    y = s["y"].double()
    r1 = wide((y.square().unflatten(-1, (groups, -1)).sum(-1) * (groups / n) + EPS) ** -0.5) if c["post"] else torch.ones_like(y)
    w1 = s["post_weight"].double() if c["post"] else torch.ones(n, dtype=torch.float64, device="cuda")
    gate = None if s["gate"] is None else s["gate"].double()
    sig = None if gate is None else 1 / (1 + torch.exp(-gate))
    act = torch.ones_like(y) if gate is None else gate * sig if c["gate"] == "silu" else sig
    k = s["scale"].double() if c["scale"] else torch.ones(n, dtype=torch.float64, device="cuda")
    unit = y * r1
    total = unit * w1 * act * k + (0 if s["x"] is None else s["x"].double())
    out = [total]
    if c["pre"]:
        w2 = s["weight"].double()
        r2 = (total.square().mean(-1, keepdim=True) + EPS) ** -0.5
        out.append(total * r2 * w2)
    if c["kind"] != "norm_train":
        return out
    d = s["grads"][0].double()
    dw2 = None
    if c["pre"]:
        dh = s["grads"][1].double()
        dw2 = (dh * total * r2).sum((0, 1))
        d = d + r2 * (dh * w2 - total * r2 ** 2 * (dh * w2 * total).mean(-1, keepdim=True))
    through = d * k * act
    dunit = through * w1
    dy = dunit
    if c["post"]:
        dy = r1 * (dunit - unit * wide((dunit * unit).unflatten(-1, (groups, -1)).mean(-1)))
    if s["x"] is not None:
        out.append(d)
    out.append(dy)
    if gate is not None:
        slope = sig * (1 + gate * (1 - sig)) if c["gate"] == "silu" else sig * (1 - sig)
        out.append(d * k * unit * w1 * slope)
    if c["pre"]:
        out.append(dw2)
    if c["post"]:
        out.append((through * unit).sum((0, 1)))
    return out + ([(d * unit * w1 * act).sum((0, 1))] if c["scale"] else [])


def exact(case, seed):
    if case["kind"].startswith("scan"):
        steps = case["T"] * (45 if case["kind"] == "scan_train" else 15)
        if steps * (1.2e-5 + case["B"] * case["n"] * case["N"] * 1e-11) > 18:
            return None
    s = prepare(case, seed)
    kind = case["kind"].split("_")[0]
    out = {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[kind](s)
    if case["kind"].endswith("step"):
        return out[0][:, 0], out[1]
    return out if case["kind"].endswith("train") else tuple(out)


def work(case):
    es, rows, n = 2 if case["dtype"] == "bf16" else 4, case["B"] * case["T"], case["n"]
    kind, way = case["kind"].split("_")[0], case["kind"].split("_")[-1]
    if kind == "norm":
        stream = {"none": es, "same": es, "f32": 4}[case["stream"]]
        read = es + (stream if case["stream"] != "none" else 0) + (es if case["gate"] != "none" else 0)
        wrote = stream + (es if case["pre"] else 0)
        # backward: everything that was read and the outputs' gradients read, the inputs' gradients written
        return {"bytes": rows * n * ((read + wrote) + (2 * read + wrote if way == "train" else 0)), "flops": rows * n * (40 if way == "train" else 15)}
    live = rows / 2 if case["ragged"] else rows          # lengths are uniform between none and all
    if kind == "conv":
        W = case["width"]
        states = case["B"] * (W - 1) * n * es * (2 if case["carried"] else 1)
        # backward: x and dy read, dx written
        return {"bytes": live * n * es * (5 if way == "train" else 2) + states * (2 if way == "train" else 1),
                "flops": live * n * (2 * W + 5) * (3 if way == "train" else 1)}
    N, gate = case["N"], 1 if case["gate"] else 0
    states = 4 * case["B"] * n * N * (2 if case["carried"] or way == "step" else 1)
    moved = live * es * ((3 + gate) * n + 2 * case["groups"] * N)
    # an element of the state: the exponent, its exponential, the input, the update and the read-out
    flops = live * n * (7 * N + 20)
    if way == "train":
        # backward: the inputs and dy read, their gradients written; an element of the state formed again, its gradient and what that gives
        moved += live * es * ((5 + 2 * gate) * n + 4 * case["groups"] * N)
        flops += live * n * (21 * N + 40)
        states *= 2
    return {"bytes": moved + states + 4 * n * N, "flops": flops}

"""The gated delta rule and the norm of queries and keys with the position rotation, as cases to time: each operator over
whole sequences, for one token, and in training (forward and backward).

A case is a dict: kind ("delta", "delta_train", "delta_step", "norm" or "norm_train"), B, H_k, H_v (key and value heads),
T, d_k, d_v, dtype ("f32" or "bf16") and the choices of that kind.
"""
import math

import torch

own = False   # false: the plain forms below; true: this repository's kernels

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64    # tokens of a step of the plain gated delta rule
EPS = 1e-6


def _delta(kind, B, H_k, H_v, d, dtype, *, T=1, d_v=None, carried=False, ragged=False, name=None):
    c = dict(kind=kind, B=B, H_k=H_k, H_v=H_v, T=T, d_k=d, d_v=d if d_v is None else d_v, dtype=dtype, carried=carried, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _norm(kind, B, T, H_q, H_k, d, dtype, *, rot=None, interleaved=False, l2=False, name=None):
    c = dict(kind=kind, B=B, T=T, H_v=H_q, H_k=H_k, d_k=d, dtype=dtype, rot=d if rot is None else rot, interleaved=interleaved, l2=l2)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # generation: one token of 64 sequences, each at a position of its own
        _norm("norm", 64, 1, 16, 4, 128, "bf16", name="norm_token"),
        # prefill of one long prompt, keys and queries of the recurrence (unit length)
        _norm("norm", 1, 16384, 16, 16, 64, "bf16", l2=True, name="norm_prefill"),
        # training: odd length, a quarter of each head rotated, float32
        _norm("norm_train", 3, 1537, 13, 13, 96, "f32", rot=32, interleaved=True, name="norm_train_ragged"),
        # training: a large batch, shared key heads
        _norm("norm_train", 8, 8192, 32, 8, 128, "bf16", name="norm_train_large"),
        # generation for one sequence: a launch and the host path
        _delta("delta_step", 1, 16, 16, 64, "bf16", name="step_few_heads"),
        # generation for a serving batch: the states of 2048 heads through memory once
        _delta("delta_step", 64, 16, 32, 128, "bf16", name="step_large_batch"),
        # a short prompt in float32
        _delta("delta", 1, 4, 4, 64, "f32", T=256, name="short"),
        # one long prompt, few heads
        _delta("delta", 1, 16, 16, 128, "bf16", T=32768, name="context_32768"),
        # the later part of sequences of unequal lengths, unequal head sizes, float32
        _delta("delta", 3, 13, 13, 128, "f32", T=1537, d_v=64, carried=True, ragged=True, name="carried_ragged"),
        # prefill of a large batch
        _delta("delta", 16, 32, 32, 128, "bf16", T=8192, name="large_batch"),
        # training: an ordinary batch of short sequences, heads of 64
        _delta("delta_train", 16, 8, 8, 64, "bf16", T=1024, name="train_d64"),
        # training: longer sequences, key heads shared by four value heads
        _delta("delta_train", 4, 4, 16, 128, "bf16", T=4096, name="train_shared"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("delta", "delta", "delta_train", "delta_train", "delta_step", "norm", "norm_train"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    d, H_k, share, B = rng.choice((16, 32, 64, 64, 96, 128, 128)), rng.randint(1, 16), rng.choice((1, 1, 1, 2, 4)), _log(rng, 1, 64)
    if kind.startswith("norm"):
        rows = 2 ** 21 // (2 if dtype == "f32" else 1)
        T = max(1, min(_log(rng, 1, 16384), rows // (B * H_k * (share + 1))))
        rot = rng.choice((d, d, 16 if d % 32 else d // 2))
        return _norm(kind, B, T, H_k * share, H_k, d, dtype, rot=rot, interleaved=rng.random() < 0.4, l2=rng.random() < 0.4)
    d_v = d if rng.random() < 0.75 else rng.choice((16, 32, 64, 96, 128))
    opt = dict(d_v=d_v, carried=rng.random() < 0.4, ragged=rng.random() < 0.25)
    if kind == "delta_step":
        return _delta(kind, B, H_k, H_k * share, d, dtype, d_v=d_v, carried=True)
    most, longest = (2 ** 22, 32768) if kind == "delta" else (2 ** 18, 8192)
    if dtype == "f32":
        most //= 4
    T = max(1, min(_log(rng, 1, longest), most // (B * H_k * share)))
    return _delta(kind, B, H_k, H_k * share, d, dtype, T=T, **opt)


# ---- inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def _prepare_delta(case, gen, dtype):
    B, H_k, H_v, T, d_k, d_v = (case[n] for n in ("B", "H_k", "H_v", "T", "d_k", "d_v"))
    # q and k come out of the norm with heads before tokens; v is a view of a projection's rows [B, T, H d]
    q, k = (_unit(_randn(gen, B, H_k, T, d_k)).to(dtype) for _ in range(2))
    v = _randn(gen, B, T, H_v, d_v).to(dtype).transpose(1, 2)
    # decays: each head has a rate of its own, from states that last thousands of tokens to ones that last a few
    rate = torch.exp(math.log(1e-3) + torch.rand((1, H_v, 1), generator=gen, device="cuda") * math.log(1e3))
    g = -rate * torch.nn.functional.softplus(_randn(gen, B, H_v, T))
    beta = torch.sigmoid(_randn(gen, B, H_v, T))
    step = case["kind"] == "delta_step"
    S = _randn(gen, B, H_v, d_v, d_k) * d_k ** -0.5 if case["carried"] or step else None
    s = dict(case=case, q=q, k=k, v=v, g=g, beta=beta, S=S, scale=d_k ** -0.5, lengths=None)
    if case["ragged"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    if step:
        s.update(q=q[:, :, 0].contiguous(), k=k[:, :, 0].contiguous(), v=v[:, :, 0].contiguous(), g=g[:, :, 0].contiguous(),
                 beta=beta[:, :, 0].contiguous())
    if case["kind"] == "delta_train":
        s["do"] = _randn(gen, B, T, H_v, d_v).to(dtype).transpose(1, 2)
        s["dS"] = _randn(gen, B, H_v, d_v, d_k) * d_v ** -0.5
        s["leaves"] = [s[n].detach().requires_grad_() for n in ("q", "k", "v", "g", "beta")]
        if S is not None:
            s["leaves"].append(S.detach().requires_grad_())
    return s


def _prepare_norm(case, gen, dtype):
    B, T, H_q, H_k, d, rot = (case[n] for n in ("B", "T", "H_v", "H_k", "d_k", "rot"))
    # slices of one fused projection [B, T, (H_q + 2 H_k) d]: queries, keys, values
    rows = _randn(gen, B, T, (H_q + 2 * H_k) * d).to(dtype)
    q = rows[:, :, :H_q * d].view(B, T, H_q, d).transpose(1, 2)
    k = rows[:, :, H_q * d:(H_q + H_k) * d].view(B, T, H_k, d).transpose(1, 2)
    wq, wk = (1 + 0.1 * _randn(gen, d) for _ in range(2))
    wq, wk = wq.to(dtype), wk.to(dtype)
    places = 16384 if T == 1 else T
    angle = torch.arange(places, device="cuda").unsqueeze(1) * 10000.0 ** (-torch.arange(rot // 2, device="cuda") * 2.0 / rot)
    s = dict(case=case, q=q, k=k, wq=wq, wk=wk, cos=angle.cos(), sin=angle.sin(), positions=None)
    if T == 1:
        s["positions"] = torch.randint(0, places, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
    if case["kind"] == "norm_train":
        s["dy"] = [_randn(gen, B, H, T, d).to(dtype) for H in (H_q, H_k)]
        s["leaves"] = [x.detach().requires_grad_() for x in (q, k, wq, wk)]
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (_prepare_norm if case["kind"].startswith("norm") else _prepare_delta)(case, gen, DTYPES[case["dtype"]])


# ---- plain forms

def _inverse(M):
    """The inverse of I + M, M strictly lower triangular, from those of its two halves."""
    n = M.shape[-1]
    if n == 1:
        return torch.ones_like(M)
    h = n // 2
    a, d = _inverse(M[..., :h, :h]), _inverse(M[..., h:, h:])
    top = torch.cat((a, torch.zeros_like(M[..., :h, h:])), -1)
    return torch.cat((top, torch.cat((-(d @ (M[..., h:, :h] @ a)), d), -1)), -2)


def _plain_delta(q, k, v, g, beta, S, scale, lengths):
    """Chunks of 64 tokens: what one writes is solved within the chunk, the state passes from chunk to chunk."""
    dtype, (B, H_v, T, d_v), share = q.dtype, v.shape, v.shape[1] // q.shape[1]
    pad = -T % CHUNK
    if lengths is not None:
        live = torch.arange(T, device=q.device) < lengths[:, None, None]
        g, beta, q = torch.where(live, g, 0.0), torch.where(live, beta, 0.0), torch.where(live[..., None], q, 0.0)
        v = torch.where(live[..., None], v, 0.0)
    full = lambda x: torch.nn.functional.pad(x.float(), (0, 0, 0, pad)).reshape(B, x.shape[1], -1, CHUNK, x.shape[-1])
    q, k, v = full(q).repeat_interleave(share, 1), full(k).repeat_interleave(share, 1), full(v)
    g, beta = full(g.unsqueeze(-1)), full(beta.unsqueeze(-1))
    G = g.cumsum(-2)
    gamma, rest = G.exp(), (G[..., -1:, :] - G).exp()
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=q.device).tril()
    D = torch.where(lower, G - G.transpose(-1, -2), float("-inf")).exp()
    kt = k.transpose(-1, -2).contiguous()
    X = _inverse((beta * D * (k @ kt)).tril(-1))
    A = D * (q @ kt)
    first, second = X @ (beta * v), X @ (beta * gamma * k)
    qg, kr, end = (scale * gamma) * q, rest * k, gamma[..., -1:, :]
    A = scale * A
    S = torch.zeros((B, H_v, d_v, q.shape[-1]), device=q.device) if S is None else S
    o = []
    for n in range(q.shape[2]):
        St = S.transpose(-1, -2).contiguous()
        u = first[:, :, n] - second[:, :, n] @ St
        o.append(qg[:, :, n] @ St + A[:, :, n] @ u)
        S = end[:, :, n] * S + u.transpose(-1, -2).contiguous() @ kr[:, :, n]
    return torch.cat(o, 2)[:, :, :T].to(dtype), S


def _plain_step(q, k, v, g, beta, S, scale):
    share = v.shape[1] // q.shape[1]
    q, k = (x.float().repeat_interleave(share, 1).unsqueeze(-1) for x in (q, k))
    S = g.exp()[..., None, None] * S
    r = beta.unsqueeze(-1) * (v.float() - (S @ k)[..., 0])
    S = S + r.unsqueeze(-1) * k.transpose(-1, -2)
    return (scale * (S @ q)[..., 0]).to(v.dtype), S


def _plain_norm(x, w, cos, sin, positions, rot, interleaved, l2):
    dtype, x = x.dtype, x.float()
    total = (x * x).sum(-1, keepdim=True)
    x = x * torch.rsqrt((total if l2 else total / x.shape[-1]) + EPS) * w.float()
    c, s = ((t[:x.shape[2]] if positions is None else t[positions.long()].unsqueeze(1)) for t in (cos, sin))
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * c - b * s, a * s + b * c), -1)
    return torch.cat((turned, x[..., rot:]), -1).to(dtype).contiguous()


# ---- one pass

def _pass_delta(s, leaves=None):
    q, k, v, g, beta = leaves[:5] if leaves else (s["q"], s["k"], s["v"], s["g"], s["beta"])
    S = leaves[5] if leaves and len(leaves) > 5 else s["S"]
    if own:
        import paper_2605_11196_amd as vla

        return vla.gated_delta(q, k, v, g, beta, S, scale=s["scale"], lengths=s["lengths"])
    return _plain_delta(q, k, v, g, beta, S, s["scale"], s["lengths"])


def _pass_norm(s, leaves=None):
    c = s["case"]
    q, k, wq, wk = leaves or (s["q"], s["k"], s["wq"], s["wk"])
    if own:
        import paper_2605_11196_amd as vla

        return vla.qk_norm_rope(q, k, wq, wk, s["cos"], s["sin"], positions=s["positions"], eps=EPS, norm="l2" if c["l2"] else "rms",
                                interleaved=c["interleaved"])
    return tuple(_plain_norm(x, w, s["cos"], s["sin"], s["positions"], c["rot"], c["interleaved"], c["l2"]) for x, w in ((q, wq), (k, wk)))


def run(state):
    kind = state["case"]["kind"]
    if kind == "delta":
        return _pass_delta(state)
    if kind == "norm":
        return _pass_norm(state)
    if kind == "delta_step":
        s = state
        if own:
            import paper_2605_11196_amd as vla

            o = vla.gated_delta_decode_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["S"], scale=s["scale"])
        else:
            o, S = _plain_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["S"], s["scale"])
            s["S"].copy_(S)
        return o, s["S"]
    if kind == "delta_train":
        o, S = _pass_delta(state, state["leaves"])
        return [o.detach(), S.detach(), *torch.autograd.grad((o, S), state["leaves"], (state["do"], state["dS"]))]
    q, k = _pass_norm(state, state["leaves"])
    return [q.detach(), k.detach(), *torch.autograd.grad((q, k), state["leaves"], state["dy"])]


# ---- the definitions in 64 bits

def _exact_delta(s):
    """Token by token; the gradients by the recurrence in reverse, from the states kept at every 64th token."""
    c = s["case"]
    B, H_k, H_v, T, d_k, d_v, scale = (*(c[n] for n in ("B", "H_k", "H_v", "T", "d_k", "d_v")), s["scale"])
    N, share = B * H_v, H_v // H_k
    heads = lambda x: x.double().reshape(B, x.shape[1], -1, x.shape[-1])
    q, k = (heads(s[n])[:, :, None].expand(B, H_k, share, T, d_k).reshape(N, T, d_k) for n in ("q", "k"))
    v = heads(s["v"]).reshape(N, T, d_v)
    g, beta = s["g"].double().reshape(N, T, 1), s["beta"].double().reshape(N, T, 1)
    length = torch.full((B,), T, device=q.device) if s["lengths"] is None else s["lengths"]
    live = (torch.arange(T, device=q.device) < length[:, None]).repeat_interleave(H_v, 0).double().unsqueeze(-1)
    alpha, beta = torch.exp(g * live), beta * live
    S = torch.zeros((N, d_v, d_k), dtype=torch.float64, device=q.device) if s["S"] is None else s["S"].double().reshape(N, d_v, d_k)
    o, kept = torch.empty((N, T, d_v), dtype=torch.float64, device=q.device), []

    def forward(S, t):
        old = S * alpha[:, t, :, None]
        r = v[:, t] - torch.bmm(old, k[:, t, :, None])[..., 0]
        return old, r, old + (beta[:, t] * r).unsqueeze(-1) * k[:, t, None]

    train = c["kind"] == "delta_train"
    for t in range(T):
        if train and t % 64 == 0:
            kept.append(S)
        S = forward(S, t)[2]
        o[:, t] = torch.bmm(S, q[:, t, :, None])[..., 0]
    shape = lambda x: x.view(B, H_v, *x.shape[1:])
    out = [shape(o * live * scale), shape(S)]
    if not train:
        return tuple(out)
    do, dS = heads(s["do"]).reshape(N, T, d_v) * live * scale, s["dS"].double().reshape(N, d_v, d_k).clone()
    dq, dk, dv, dg, dbeta = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    for first in range((T - 1) // 64 * 64, -1, -64):
        S, steps = kept.pop(), []
        for t in range(first, min(first + 64, T)):
            steps.append((S, *forward(S, t)))
            S = steps[-1][3]
        for t in range(min(first + 64, T) - 1, first - 1, -1):
            _, old, r, new = steps[t - first]
            dq[:, t] = torch.bmm(do[:, t, None], new)[:, 0]
            dS += do[:, t, :, None] * q[:, t, None]
            de = torch.bmm(dS, k[:, t, :, None])[..., 0]
            dbeta[:, t] = (de * r).sum(-1, keepdim=True)
            dr = beta[:, t] * de
            dk[:, t] = torch.bmm((beta[:, t] * r)[:, None], dS)[:, 0] - torch.bmm(dr[:, None], old)[:, 0]
            dv[:, t] = dr
            dS -= dr.unsqueeze(-1) * k[:, t, None]
            dg[:, t] = (dS * old).sum((-1, -2)).unsqueeze(-1)
            dS *= alpha[:, t, :, None]
        del steps
    shared = lambda x: x.view(B, H_k, share, T, d_k).sum(2)
    out += [shared(dq), shared(dk * live), shape(dv), shape(dg * live)[..., 0], shape(dbeta * live)[..., 0]]
    return out + ([] if s["S"] is None else [shape(dS)])


def _exact_norm(s):
    """Pairs of columns as complex numbers; the gradients by the chain rule."""
    c = s["case"]
    d, rot = c["d_k"], c["rot"]
    col = torch.arange(rot, device="cuda")
    col = (col.view(-1, 2) if c["interleaved"] else col.view(2, -1).T).T     # first and second columns of the pairs
    place = torch.arange(c["T"], device="cuda")[None] if s["positions"] is None else s["positions"].long()
    turn = torch.complex(s["cos"].double()[place], s["sin"].double()[place])[:, None]
    n = 1 if c["l2"] else d

    def rotate(x, turn):
        y, z = x.clone(), torch.complex(x[..., col[0]], x[..., col[1]]) * turn
        y[..., col[0]], y[..., col[1]] = z.real, z.imag
        return y

    out, grads, weights = [], [], []
    for i, (name, weight) in enumerate((("q", "wq"), ("k", "wk"))):
        x, w = s[name].double(), s[weight].double()
        r = (x.square().sum(-1, keepdim=True) / n + EPS) ** -0.5
        out.append(rotate(x * r * w, turn))
        if c["kind"] == "norm_train":
            back = rotate(s["dy"][i].double(), turn.conj())
            weights.append((back * x * r).sum((0, 1, 2)))
            dn = back * w
            grads.append(r * dn - x * r ** 3 * (dn * x).sum(-1, keepdim=True) / n)
    return out + grads + weights


def exact(case, seed):
    if not case["kind"].startswith("norm"):
        steps = case["T"] * (6 if case["kind"] == "delta_train" else 1)
        cost = steps * (6e-5 + case["B"] * case["H_v"] * case["d_k"] * case["d_v"] * 2e-11)
        if cost > 18:
            return None
    s = prepare(case, seed)
    out = _exact_norm(s) if case["kind"].startswith("norm") else _exact_delta(s)
    if case["kind"] == "delta_step":
        return out[0][:, :, 0], out[1]
    return out if case["kind"].endswith("train") else tuple(out)


def work(case):
    es, B, T = 2 if case["dtype"] == "bf16" else 4, case["B"], case["T"]
    if case["kind"].startswith("norm"):
        rows = B * T * (case["H_v"] + case["H_k"])
        train = case["kind"] == "norm_train"
        tables = 4 * case["rot"] * (min(B, T) if T == 1 else T)
        # forward: x read, y written; backward: x and dy read, dx written
        return {"bytes": rows * case["d_k"] * es * (5 if train else 2) + tables, "flops": rows * case["d_k"] * (20 if train else 8)}
    H_k, H_v, d_k, d_v = (case[n] for n in ("H_k", "H_v", "d_k", "d_v"))
    rows, state = B * T * (2 * H_k * d_k + 2 * H_v * d_v) * es + 8 * B * T * H_v, 4 * B * H_v * d_k * d_v
    if case["ragged"]:
        rows = rows // 2      # lengths are uniform between none and all
    states = state * (2 if case["carried"] or case["kind"] == "delta_step" else 1)
    # the residual, the update and the read-out of a token: a product with the state each
    flops = B * T * H_v * 6 * d_k * d_v / (2 if case["ragged"] else 1)
    if case["kind"] != "delta_train":
        return {"bytes": rows + states, "flops": flops}
    # backward: q, k, v, g, beta and dO read again, their gradients written; seven products with a state
    back = (B * T * (4 * H_k * d_k + 3 * H_v * d_v) * es + 16 * B * T * H_v) / (2 if case["ragged"] else 1)
    return {"bytes": rows + back + 2 * states, "flops": flops * 20 / 6}

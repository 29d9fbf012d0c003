"""CPU-only checks of the operators around the recurrence (include/vla.h): option structures, sizes, and what is refused on the host
before anything is launched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_11196_amd as vla
from paper_2605_11196_amd import binding
from paper_2605_11196_amd.binding import VlaDeltaOpts, VlaNormOpts, VlaStrides

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000   # 16-byte aligned, non-null, never dereferenced on these paths
PLACE = {name: FAKE + i * 0x100000 for i, name in enumerate(
    ("q", "k", "v", "g", "beta", "S0", "o", "S_T", "dO", "dS_T", "dq", "dk", "dv", "dg", "dbeta", "dS0", "ws", "saved", "wq", "wk", "cos", "sin"))}


def lib():
    return vla.load_library()


def ref(x):
    return ctypes.byref(x)


@pytest.mark.parametrize("struct,mirror", [("vla_strides", VlaStrides), ("vla_delta_opts", VlaDeltaOpts), ("vla_norm_opts", VlaNormOpts)])
def test_structures_match_the_header(struct, mirror):
    text = open(os.path.join(ROOT, "include", "vla.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            names += [n.strip(" *") for n in re.sub(r"^(const )?(long long|\w+)\s*\*?\s+", "", line + " ", count=1).split(",")]
    assert [n.split()[-1] for n in names] == [f[0] for f in mirror._fields_]


def test_default_options():
    d, n = VlaDeltaOpts(scale=3.0, segments=5), VlaNormOpts(l2=1)
    lib().vla_delta_default_opts(ref(d))
    lib().vla_norm_default_opts(ref(n))
    assert bytes(d) == bytes(VlaDeltaOpts())
    assert abs(n.eps - 1e-6) < 1e-12 and n.l2 == 0 and n.rot == 0 and n.places == 0 and n.positions is None


def forward(opts=None, **kw):
    a = dict(PLACE, B=1, H_k=1, H_v=1, T=8, d_k=16, d_v=16, io=vla.VLA_F32, ws_bytes=0)
    a.update(kw)
    return lib().vla_delta_forward(*(a[n] or None for n in ("q", "k", "v", "g", "beta", "S0", "o", "S_T")), a["B"], a["H_k"], a["H_v"], a["T"],
                                   a["d_k"], a["d_v"], a["io"], None if opts is None else ref(opts), a["ws"] if a["ws_bytes"] else None,
                                   a["ws_bytes"], None)


S = VlaStrides


@pytest.mark.parametrize("kw,opts,status", [
    (dict(B=0), None, 1), (dict(H_k=0), None, 1), (dict(H_v=-1), None, 1), (dict(T=-1), None, 1), (dict(H_k=2, H_v=3), None, 1), (dict(H_k=4, H_v=2), None, 1),
    (dict(io=2), None, 1), (dict(d_k=0), None, 1), (dict(d_k=48), None, 2), (dict(d_v=256), None, 2), (dict(B=1 << 20, H_k=64, H_v=64), None, 2),
    (dict(q=0), None, 1), (dict(g=0), None, 1), (dict(beta=0), None, 1), (dict(o=0), None, 1), (dict(q=FAKE + 8), None, 1), (dict(S0=PLACE["S0"] + 4), None, 1),
    (dict(o=PLACE["q"]), None, 1), (dict(o=PLACE["v"] + 16), None, 1), (dict(S_T=PLACE["S0"] + 256), None, 1), (dict(o=PLACE["g"] - 64), None, 1),
    (dict(S_T=PLACE["o"] + 16), None, 1), (dict(ws=PLACE["o"], ws_bytes=64), None, 1),
    ({}, dict(scale=float("nan")), 1), ({}, dict(scale=float("inf")), 1), ({}, dict(segments=-1), 1),
    ({}, dict(q=S(128, 128, 18)), 1),            # rows that are not whole 16-byte pieces apart
    ({}, dict(k=S(128, 128, -16)), 1),
    ({}, dict(v=S(128, 128, 8)), 1),             # tokens that overlap
    ({}, dict(o=S(128, 0, 8)), 1),
    (dict(H_k=2, H_v=2), dict(o=S(256, 64, 16)), 1),   # heads of o in each other
    (dict(H_k=2, H_v=2), dict(q=S(0, 0, 16), o=S(0, 64, 16)), 1),
    ({}, dict(q=S(0, 0, 1 << 25)), 2),           # tokens too far apart
    ({}, dict(saved=PLACE["saved"], saved_bytes=16), 3), ({}, dict(saved=PLACE["saved"] + 4, saved_bytes=1 << 16), 1),
    ({}, dict(saved=PLACE["o"], saved_bytes=1 << 16), 1),
])
def test_forward_refuses(kw, opts, status):
    assert forward(None if opts is None else VlaDeltaOpts(**opts), **kw) == status


def test_single_token_and_backward_refuse():
    z = lambda *names: [PLACE[n] for n in names]
    step = lambda S, **kw: lib().vla_delta_decode_step(*z("q", "k", "v", "g", "beta"), S, PLACE["o"], 1, kw.get("H_k", 1), kw.get("H_v", 1), 32, 32, 1, None, None)
    assert step(None) == 1 and step(PLACE["S0"] + 4) == 1 and step(PLACE["S0"], H_k=2, H_v=3) == 1 and step(PLACE["o"]) == 1
    need = lib().vla_delta_workspace_bytes(1, 1, 1, 40, 32, 32, 1, None, 1)
    kept = lib().vla_delta_saved_bytes(1, 1, 40, 32, 32, 1)
    assert need > 0 and kept >= 4 * (32 * 32 + 40 * 32)
    order = ("q", "k", "v", "g", "beta", "dO", "dS_T", "dq", "dk", "dv", "dg", "dbeta", "dS0")

    def back(saved_bytes=kept, ws_bytes=need, opts=None, **kw):
        a = dict(PLACE, **kw)
        op = VlaDeltaOpts(saved=a["saved"] or None, saved_bytes=saved_bytes, **(opts or {}))
        return lib().vla_delta_backward(*(a[n] or None for n in order), 1, 1, 1, 40, 32, 32, 1, ref(op), a["ws"], ws_bytes, None)

    assert back(saved_bytes=kept - 1) == 3 and back(ws_bytes=need - 1) == 3
    for name in ("q", "dO", "dq", "dv", "dg", "dbeta", "saved"):
        assert back(**{name: 0}) == 1, name
    assert back(dq=PLACE["k"]) == 1 and back(dv=PLACE["dk"] + 16) == 1 and back(dS0=PLACE["dS_T"]) == 1 and back(ws=PLACE["saved"]) == 1
    assert back(opts=dict(dq=S(0, 0, 16))) == 1 and back(opts=dict(dk=S(4096, 4096, 36))) == 1


def test_sizes():
    ws = lambda *a, back=0: lib().vla_delta_workspace_bytes(*a, None, back)
    assert ws(64, 32, 32, 8192, 128, 128, 1) == 0                      # many heads: no segments
    assert ws(1, 16, 16, 32768, 128, 128, 1) == 16 * 16 * 4 * (128 * 128 + 256 * 128)
    assert ws(1, 16, 16, 32768, 128, 130, 1) == 0 and ws(0, 1, 1, 1, 16, 16, 1) == 0
    assert ws(1, 4, 8, 64, 32, 32, 1, back=1) > ws(1, 8, 8, 64, 32, 32, 1, back=1)   # heads that share a key head: parts of dq as well
    assert lib().vla_delta_saved_bytes(1, 1, 257, 16, 16, 0) == 2 * 16 * 16 * 4 + (257 * 16 * 4 + 255) // 256 * 256
    assert lib().vla_qk_norm_rope_workspace_bytes(64) > 0 and lib().vla_qk_norm_rope_workspace_bytes(65) == 0


def norm(opts=None, **kw):
    a = dict(PLACE, B=1, T=4, H_q=2, H_k=1, d=32, io=0)
    a.update(kw)
    op = VlaNormOpts(eps=1e-6, places=16)
    for key, val in (opts or {}).items():
        setattr(op, key, val)
    return lib().vla_qk_norm_rope(*(a[n] or None for n in ("q", "k", "wq", "wk", "cos", "sin", "o", "dO")), a["B"], a["T"], a["H_q"], a["H_k"],
                                  a["d"], a["io"], ref(op), None)


@pytest.mark.parametrize("kw,opts,status", [
    (dict(B=0), None, 1), (dict(T=-1), None, 1), (dict(H_q=0, H_k=0), None, 1), (dict(H_k=-1), None, 1), (dict(d=48), None, 2), (dict(io=3), None, 1),
    (dict(q=0), None, 1), (dict(o=0), None, 1), (dict(sin=0), None, 1), (dict(cos=0, sin=0), dict(rot=8), 1), (dict(q=FAKE + 4), None, 1),
    (dict(wk=PLACE["wk"] + 4), None, 1), ({}, dict(eps=0.0), 1), ({}, dict(eps=float("nan")), 1), ({}, dict(places=0), 1), ({}, dict(offset=-1), 1),
    ({}, dict(rot=12), 1), ({}, dict(rot=40), 1), ({}, dict(rot=-8), 1), ({}, dict(weight_dtype=2), 1), ({}, dict(q=S(0, 0, 30)), 1),
    ({}, dict(q_out=S(256, 16, 32)), 1), (dict(o=PLACE["q"]), None, 1), (dict(dO=PLACE["o"] + 64), None, 1), (dict(o=PLACE["cos"]), None, 1),
    ({}, dict(positions=PLACE["o"]), 1),
])
def test_norm_refuses(kw, opts, status):
    assert norm(opts, **kw) == status


def test_norm_backward_refuses():
    order = ("q", "k", "wq", "wk", "cos", "sin", "dO", "dS_T", "dq", "dk", "dg", "dbeta")

    def back(ws_bytes=1 << 20, **kw):
        a = dict(PLACE, **kw)
        return lib().vla_qk_norm_rope_backward(*(a[n] or None for n in order), 1, 4, 2, 1, 32, 0, ref(VlaNormOpts(eps=1e-6, places=16)), a["ws"] or None, ws_bytes, None)

    assert back(ws_bytes=100) == 3 and back(ws=0) == 3 and back(dO=0) == 1 and back(dq=0) == 1 and back(dq=PLACE["q"]) == 1 and back(dg=PLACE["dbeta"]) == 1


def test_tensor_front_ends_refuse():
    q = torch.zeros(1, 2, 4, 32)
    gate = torch.zeros(1, 2, 4)
    with pytest.raises(ValueError, match="GPU"):
        vla.gated_delta(q, q, q, gate, gate)
    with pytest.raises(ValueError, match="GPU"):
        vla.gated_delta_decode_step(q[:, :, 0], q[:, :, 0], q[:, :, 0], gate[:, :, 0], gate[:, :, 0], torch.zeros(1, 2, 32, 32))
    with pytest.raises(ValueError, match="GPU"):
        vla.qk_norm_rope(q, q)
    with pytest.raises(ValueError, match="GPU"):
        vla.qk_norm_rope_backward(q, q, None, None, None, None, q, q)
    assert "vla_delta_forward" in str(binding.VlaError(1, "VLA_ERR_INVALID_ARG", "vla_delta_forward"))
    with pytest.raises(ValueError, match="stream"):
        vla.qk_norm_rope(q.requires_grad_(), q, stream=1)

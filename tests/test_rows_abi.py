"""CPU-only checks of the operators on rows of channels (include/vla.h): option structures, sizes, and what is refused on the host before
anything is launched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_11196_amd as vla
from paper_2605_11196_amd.binding import VlaConvOpts, VlaResidualOpts, VlaScanOpts, VlaStrides

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
S = VlaStrides
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
NAMES = ("x", "y", "weight", "bias", "state", "state_T", "dy", "dstate_T", "dx", "dweight", "dbias", "dstate", "ws", "u", "delta", "A", "Bm", "Cm", "D", "z",
         "h0", "h_T", "dh_T", "du", "ddelta", "dA", "dBm", "dCm", "dD", "dz", "dh0", "saved", "gate", "post", "scale", "s", "h", "ds", "dh", "dgate",
         "dpost", "dscale")
# 16-byte aligned, far apart, never dereferenced on these paths
PLACE = {name: 0x100000000 + i * 0x10000000 for i, name in enumerate(NAMES)}


def lib():
    return vla.load_library()


def call(name, arguments, defaults, opts, given):
    a = dict(PLACE, io=vla.VLA_F32, ws_bytes=1 << 24, **defaults)
    a.update(given)
    values = []
    for n in arguments.split():
        if n == "opts":
            values.append(None if opts is None else ctypes.byref(opts))
        elif n == "stream":
            values.append(None)
        else:
            values.append(a[n] or None if n in PLACE else a[n])
    return getattr(lib(), name)(*values)


CONV = "x weight bias state y state_T B T n width io opts stream"
CONV_STEP = "x weight bias state y B n width io opts stream"
CONV_BACK = "x weight bias state dy dstate_T dx dweight dbias dstate B T n width io opts ws ws_bytes stream"
SCAN = "u delta A Bm Cm D z bias h0 y h_T B T n N io opts ws ws_bytes stream"
SCAN_STEP = "u delta A Bm Cm D z bias h y B n N io opts stream"
SCAN_BACK = "u delta A Bm Cm D z bias dy dh_T du ddelta dA dBm dCm dD dz dbias dh0 B T n N io opts ws ws_bytes stream"
NORM = "x y gate post scale weight s h B T n io opts stream"
NORM_BACK = "x y gate post scale weight ds dh dx dy dgate dpost dscale dweight B T n io opts ws ws_bytes stream"
SIZES = dict(B=2, T=24, n=32, width=4, N=16)


def conv_opts(**kw):
    o = VlaConvOpts()
    lib().vla_conv_default_opts(ctypes.byref(o))
    return _with(o, kw)


def scan_opts(**kw):
    o = VlaScanOpts()
    lib().vla_scan_default_opts(ctypes.byref(o))
    return _with(o, kw)


def norm_opts(**kw):
    o = VlaResidualOpts()
    lib().vla_residual_default_opts(ctypes.byref(o))
    return _with(o, kw)


def _with(o, kw):
    for k, v in kw.items():
        setattr(o, k, v)
    return o


@pytest.mark.parametrize("struct,mirror", [("vla_conv_opts", VlaConvOpts), ("vla_scan_opts", VlaScanOpts), ("vla_residual_opts", VlaResidualOpts)])
def test_structures_match_the_header(struct, mirror):
    text = open(os.path.join(ROOT, "include", "vla.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            names += [n.strip(" *") for n in re.sub(r"^(const )?\w+\s*\*?\s+", "", line + " ", count=1).split(",")]
    assert [n.split()[-1] for n in names] == [f[0] for f in mirror._fields_]


def test_default_options():
    c, s, r = VlaConvOpts(silu=7, weight_dtype=1), VlaScanOpts(segments=4), VlaResidualOpts(group=8)
    lib().vla_conv_default_opts(ctypes.byref(c))
    lib().vla_scan_default_opts(ctypes.byref(s))
    lib().vla_residual_default_opts(ctypes.byref(r))
    assert bytes(c) == bytes(VlaConvOpts(1)) and bytes(s) == bytes(VlaScanOpts(1, 1)) and bytes(r) == bytes(VlaResidualOpts(eps=1e-6))
    for f in (lib().vla_conv_default_opts, lib().vla_scan_default_opts, lib().vla_residual_default_opts):
        f(None)


# ---- short causal convolution

@pytest.mark.parametrize("given,opts,status", [
    (dict(B=0), {}, INVALID), (dict(T=-1), {}, INVALID), (dict(n=0), {}, INVALID), (dict(io=2), {}, INVALID), (dict(width=0), {}, INVALID),
    (dict(n=36), {}, UNSUPPORTED), (dict(width=1), {}, UNSUPPORTED), (dict(width=5), {}, UNSUPPORTED), (dict(T=0x7fffffff), {}, UNSUPPORTED),
    (dict(B=2 ** 31 - 1, T=17, n=8, io=1, y=2 ** 60, state=0, state_T=0), dict(x=S(0, 0, 8)), UNSUPPORTED),      # runs of tokens that an int does not count
    (dict(x=0), {}, INVALID), (dict(weight=0), {}, INVALID), (dict(y=0), {}, INVALID), (dict(x=PLACE["x"] + 8), {}, INVALID),
    (dict(weight=PLACE["weight"] + 4), {}, INVALID), (dict(state_T=PLACE["state_T"] + 4), {}, INVALID), ({}, dict(weight_dtype=3), INVALID),
    (dict(y=PLACE["x"]), {}, INVALID), (dict(y=PLACE["weight"] - 16), {}, INVALID), (dict(state_T=PLACE["state"] + 16), {}, INVALID),
    (dict(state_T=PLACE["y"] + 64), {}, INVALID), ({}, dict(lengths=PLACE["y"]), INVALID),
    ({}, dict(x=S(768, 32, 32)), INVALID), ({}, dict(x=S(768, 0, 33)), INVALID), ({}, dict(y=S(768, 0, 0)), INVALID), ({}, dict(y=S(16, 0, 32)), INVALID)])
def test_convolution_refuses(given, opts, status):
    assert call("vla_causal_conv", CONV, SIZES, conv_opts(**opts), given) == status


@pytest.mark.parametrize("given,opts,status", [
    (dict(state=0), {}, INVALID), (dict(y=0), {}, INVALID), ({}, dict(lengths=PLACE["u"]), INVALID), (dict(y=PLACE["state"]), {}, INVALID),
    (dict(y=PLACE["x"]), {}, INVALID), (dict(state=PLACE["x"]), {}, INVALID), (dict(state=PLACE["state"] + 8), {}, INVALID), (dict(width=8), {}, UNSUPPORTED)])
def test_convolution_step_refuses(given, opts, status):
    assert call("vla_causal_conv_step", CONV_STEP, SIZES, conv_opts(**opts), given) == status


@pytest.mark.parametrize("given,opts,status", [
    (dict(dy=0), {}, INVALID), (dict(dx=0), {}, INVALID), (dict(dx=PLACE["dy"]), {}, INVALID), (dict(dx=PLACE["x"]), {}, INVALID),
    (dict(dstate=PLACE["dstate_T"]), {}, INVALID), (dict(dweight=PLACE["dbias"]), {}, INVALID), (dict(ws=PLACE["dx"]), {}, INVALID),
    (dict(ws=0), {}, WORKSPACE), (dict(ws_bytes=64), {}, WORKSPACE), (dict(dbias=PLACE["dbias"] + 4), {}, INVALID), ({}, dict(dx=S(768, 0, 0)), INVALID)])
def test_convolution_backward_refuses(given, opts, status):
    assert call("vla_causal_conv_backward", CONV_BACK, SIZES, conv_opts(**opts), given) == status


def test_convolution_workspace():
    size = lib().vla_causal_conv_workspace_bytes
    assert size(2, 24, 1024, 4, 0) == 2 * 2 * 5 * 1024 * 4      # two runs of 16 tokens a sequence, four taps and the bias
    assert size(2, 24, 32, 4, 0) == 5 * 32 * 4                  # 8 lanes a run: the four runs lie in one workgroup
    assert size(3, 1537, 72, 2, 1) == 11 * 3 * 72 * 4           # 97 runs of 9 lanes a sequence
    assert size(1, 0, 32, 2, 1) == 3 * 32 * 4
    assert size(0, 24, 32, 4, 0) == 0 and size(2, 24, 30, 4, 0) == 0 and size(2, 24, 32, 5, 0) == 0 and size(2, 24, 32, 4, 7) == 0


# ---- selective scan

SCAN_CASES = [
    (dict(B=0), {}, INVALID), (dict(T=-1), {}, INVALID), (dict(n=-8), {}, INVALID), (dict(io=9), {}, INVALID), (dict(N=0), {}, INVALID),
    (dict(N=12), {}, UNSUPPORTED), (dict(N=128), {}, UNSUPPORTED), (dict(n=36), {}, UNSUPPORTED), ({}, dict(groups=0), INVALID), ({}, dict(groups=3), INVALID),
    ({}, dict(groups=8), UNSUPPORTED), ({}, dict(segments=-1), INVALID), (dict(n=1 << 25, N=64), {}, UNSUPPORTED), (dict(B=1 << 24, n=1024), {}, UNSUPPORTED),
    (dict(u=0), {}, INVALID), (dict(delta=0), {}, INVALID), (dict(A=0), {}, INVALID), (dict(Bm=0), {}, INVALID), (dict(Cm=0), {}, INVALID),
    (dict(u=PLACE["u"] + 4), {}, INVALID), (dict(A=PLACE["A"] + 8), {}, INVALID), (dict(D=PLACE["D"] + 4), {}, INVALID),
    ({}, dict(u=S(768, 0, 30)), INVALID), ({}, dict(B=S(768, 8, 17)), INVALID), ({}, dict(z=S(768, 8, 32)), INVALID),
    ({}, dict(delta=S(0, 0, 1 << 27)), UNSUPPORTED)]      # rows too far apart for the kernels' offsets


@pytest.mark.parametrize("given,opts,status", SCAN_CASES + [
    (dict(y=0), {}, INVALID), (dict(y=PLACE["u"]), {}, INVALID), (dict(h_T=PLACE["h0"] + 64), {}, INVALID), (dict(h_T=PLACE["y"]), {}, INVALID),
    (dict(y=PLACE["A"] - 16), {}, INVALID), (dict(y=PLACE["Bm"]), {}, INVALID), ({}, dict(y=S(768, 0, 16)), INVALID),
    ({}, dict(y=S(0, 0, 32)), INVALID), ({}, dict(saved=PLACE["saved"], saved_bytes=64), WORKSPACE), ({}, dict(saved=PLACE["saved"] + 4, saved_bytes=1 << 20), INVALID),
    ({}, dict(saved=PLACE["y"], saved_bytes=1 << 20), INVALID), (dict(ws=PLACE["y"]), dict(segments=3), INVALID), ({}, dict(lengths=PLACE["h_T"]), INVALID)])
def test_scan_refuses(given, opts, status):
    assert call("vla_selective_scan", SCAN, SIZES, scan_opts(**opts), given) == status


@pytest.mark.parametrize("given,opts,status", [c for c in SCAN_CASES if "T" not in c[0]] [:14] + [
    (dict(h=0), {}, INVALID), (dict(y=0), {}, INVALID), (dict(h=PLACE["h"] + 4), {}, INVALID), ({}, dict(lengths=PLACE["dx"]), INVALID),
    (dict(h=PLACE["A"]), {}, INVALID), (dict(y=PLACE["h"] + 32), {}, INVALID), (dict(y=PLACE["z"]), {}, INVALID)])
def test_scan_step_refuses(given, opts, status):
    assert call("vla_selective_scan_step", SCAN_STEP, SIZES, scan_opts(**opts), given) == status


KEPT = dict(saved=PLACE["saved"], saved_bytes=1 << 20)


@pytest.mark.parametrize("given,opts,status", SCAN_CASES + [
    (dict(dy=0), {}, INVALID), (dict(du=0), {}, INVALID), (dict(ddelta=0), {}, INVALID), (dict(dA=0), {}, INVALID), (dict(dBm=0), {}, INVALID),
    (dict(dCm=0), {}, INVALID), (dict(dz=0), {}, INVALID), ({}, dict(saved=None), INVALID), ({}, dict(saved_bytes=64), WORKSPACE), (dict(ws=0), {}, WORKSPACE),
    (dict(ws_bytes=64), {}, WORKSPACE), (dict(du=PLACE["dy"]), {}, INVALID), (dict(ddelta=PLACE["du"] + 16), {}, INVALID), (dict(dBm=PLACE["dCm"]), {}, INVALID),
    (dict(dh0=PLACE["dh_T"]), {}, INVALID), (dict(dA=PLACE["saved"]), {}, INVALID), (dict(ws=PLACE["dh0"] - 4096), {}, INVALID), ({}, dict(du=S(0, 0, 32)), INVALID),
    ({}, dict(dz=S(768, 0, 16)), INVALID), ({}, dict(ddelta=S(1 << 40, 0, 1 << 27)), UNSUPPORTED)])
def test_scan_backward_refuses(given, opts, status):
    assert call("vla_selective_scan_backward", SCAN_BACK, SIZES, scan_opts(**dict(KEPT, **opts)), given) == status


def test_scan_sizes():
    saved, ws = lib().vla_selective_scan_saved_bytes, lib().vla_selective_scan_workspace_bytes
    opts = lambda **kw: ctypes.byref(scan_opts(**kw))
    assert saved(2, 17, 32, 16, 0, opts()) == 2 * 3 * 32 * 16 * 4        # a state at every 8th token
    assert saved(2, 0, 32, 16, 0, None) == 0 and saved(2, 17, 32, 24, 0, None) == 0 and saved(0, 17, 32, 16, 0, None) == 0
    assert ws(1, 24, 32, 16, 0, opts(segments=1), 0) == 0
    # three segments of a block: a state and the sum of the steps for each
    assert ws(1, 24, 32, 16, 0, opts(segments=3), 0) == 3 * 32 * 16 * 4 + 512
    assert ws(1, 24, 32, 16, 0, opts(segments=1 << 30), 0) == 3 * 32 * 16 * 4 + 512      # no more segments than blocks
    # backward: parts of dA, dD and the bias, of dB and dC for each workgroup of channels, and the segments' states
    assert ws(1, 24, 32, 16, 0, opts(segments=3), 1) == 3 * 32 * 16 * 4 + 2 * 512 + 24 * 2 * 16 * 4 + 3 * 32 * 16 * 4 + 512
    assert ws(1, 24, 32, 15, 0, None, 1) == 0 and ws(1, 24, 32, 16, 0, opts(groups=5), 0) == 0 and ws(1, 24, 32, 16, 0, opts(segments=-3), 1) == 0


# ---- norms around a block

NORM_CASES = [
    (dict(B=0), {}, INVALID), (dict(T=-2), {}, INVALID), (dict(n=0), {}, INVALID), (dict(io=5), {}, INVALID), (dict(n=12), {}, UNSUPPORTED),
    (dict(n=8200), {}, UNSUPPORTED), ({}, dict(eps=0.0), INVALID), ({}, dict(eps=float("nan")), INVALID), ({}, dict(eps=float("inf")), INVALID),
    ({}, dict(group=-8), INVALID), ({}, dict(group=24), INVALID), ({}, dict(group=4), UNSUPPORTED), ({}, dict(activation=2), INVALID),
    ({}, dict(stream_dtype=1), UNSUPPORTED), ({}, dict(weight_dtype=2), INVALID), (dict(x=0, y=0), {}, INVALID), (dict(y=0), {}, INVALID),
    (dict(gate=PLACE["gate"] + 8), {}, INVALID), (dict(weight=PLACE["weight"] + 4), {}, INVALID), ({}, dict(x=S(768, 32, 32)), INVALID),
    ({}, dict(gate=S(768, 0, 34)), INVALID)]


@pytest.mark.parametrize("given,opts,status", NORM_CASES + [
    (dict(s=0), {}, INVALID), (dict(h=0), {}, INVALID), (dict(weight=0), {}, INVALID), (dict(s=PLACE["y"]), {}, INVALID), (dict(s=PLACE["x"] + 16), {}, INVALID),
    (dict(h=PLACE["x"]), {}, INVALID), (dict(h=PLACE["s"]), {}, INVALID), (dict(h=PLACE["gate"]), {}, INVALID), (dict(s=PLACE["x"]), dict(x=S(1536, 0, 64)), INVALID),
    ({}, dict(s=S(768, 0, 16)), INVALID), ({}, dict(h=S(0, 0, 32)), INVALID), (dict(s=PLACE["scale"] - 16), {}, INVALID)])
def test_norms_refuse(given, opts, status):
    assert call("vla_residual_norm", NORM, SIZES, norm_opts(**opts), given) == status


@pytest.mark.parametrize("given,opts,status", NORM_CASES + [
    (dict(x=0), {}, INVALID), (dict(gate=0), {}, INVALID), (dict(post=0), {}, INVALID), (dict(scale=0), {}, INVALID), (dict(weight=0), {}, INVALID),
    (dict(ws=0), {}, WORKSPACE), (dict(ws_bytes=100), {}, WORKSPACE), (dict(dx=PLACE["ds"]), {}, INVALID), (dict(dy=PLACE["dx"] + 16), {}, INVALID),
    (dict(dgate=PLACE["gate"]), {}, INVALID), (dict(dscale=PLACE["dpost"]), {}, INVALID), (dict(ws=PLACE["dgate"]), {}, INVALID),
    (dict(ds=PLACE["ds"] + 4), {}, INVALID), ({}, dict(dy=S(768, 0, 16)), INVALID)])
def test_norms_backward_refuses(given, opts, status):
    assert call("vla_residual_norm_backward", NORM_BACK, SIZES, norm_opts(**opts), given) == status


def test_norm_workspace():
    size = lib().vla_residual_norm_workspace_bytes
    assert size(32) == 512 * 3 * 32 * 4 and size(0) == 0 and size(12) == 0 and size(8200) == 0


# ---- torch front ends, with tensors that are not on the GPU or do not fit

def test_front_ends_refuse_tensors_of_the_cpu():
    x, w, h = torch.zeros(1, 4, 16), torch.zeros(16, 4), torch.zeros(1, 16, 8)
    A, Bm = torch.zeros(16, 8), torch.zeros(1, 4, 8)
    for f in (lambda: vla.causal_conv(x, w), lambda: vla.causal_conv_step(x[:, 0], w, torch.zeros(1, 3, 16)), lambda: vla.causal_conv_backward(x, w, None, None, x),
              lambda: vla.selective_scan(x, x, A, Bm, Bm), lambda: vla.selective_scan_step(x[:, 0], x[:, 0], A, Bm[:, 0], Bm[:, 0], h),
              lambda: vla.selective_scan_backward(x, x, A, Bm, Bm, None, None, torch.zeros(64, dtype=torch.uint8), x),
              lambda: vla.residual_norm(x, x, w[:, 0]), lambda: vla.residual_norm_backward(x, x, w[:, 0], x, x)):
        with pytest.raises(ValueError, match="GPU"):
            f()


def test_steps_refuse_to_lose_a_gradient():
    x, w, state = torch.zeros(1, 16, requires_grad=True), torch.zeros(16, 4), torch.zeros(1, 3, 16)
    with pytest.raises(ValueError, match="no gradient"):
        vla.causal_conv_step(x, w, state)
    with pytest.raises(ValueError, match="no gradient"):
        vla.selective_scan_step(x, x, torch.zeros(16, 8), torch.zeros(1, 8), torch.zeros(1, 8), torch.zeros(1, 16, 8))


def test_gradients_stay_on_the_current_stream():
    x = torch.zeros(1, 4, 16, requires_grad=True)
    for f in (lambda: vla.causal_conv(x, torch.zeros(16, 4), stream=1), lambda: vla.residual_norm(x, None, torch.zeros(16), stream=1),
              lambda: vla.selective_scan(x, x, torch.zeros(16, 8), torch.zeros(1, 4, 8), torch.zeros(1, 4, 8), stream=1)):
        with pytest.raises(ValueError, match="current stream"):
            f()


def test_forward_mode_is_refused():
    x, t = torch.zeros(1, 4, 16), torch.ones(1, 4, 16)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, t)
        for f in (lambda: vla.causal_conv(dual, torch.zeros(16, 4)), lambda: vla.residual_norm(dual, None, torch.zeros(16)),
                  lambda: vla.selective_scan(dual, x, torch.zeros(16, 8), torch.zeros(1, 4, 8), torch.zeros(1, 4, 8))):
            with pytest.raises(NotImplementedError):
                f()

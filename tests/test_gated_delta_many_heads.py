"""The gated delta rule with more heads than one launch holds work-items for, 2^32 (the refusals need no GPU)."""
import ctypes

import pytest
import torch

import paper_2605_11196_amd as vla
from test_layer_abi import forward


@pytest.mark.parametrize("d_v,heads", [(128, 1 << 23), (96, (1 << 32) // (96 * 4) + 1), (64, 1 << 24)])
@pytest.mark.parametrize("T", [1, 40])
def test_more_heads_than_a_launch_holds_are_refused(d_v, heads, T):
    assert forward(B=heads, d_v=d_v, T=T) == 2
    lib = vla.load_library()
    assert lib.vla_delta_workspace_bytes(heads, 1, 1, 64, 16, d_v, vla.VLA_F32, None, 1) == 0


def test_requested_segments_are_as_many_as_a_launch_holds():
    from paper_2605_11196_amd.binding import VlaDeltaOpts

    lib, heads, d = vla.load_library(), 1 << 14, 128
    ask = lambda n: lib.vla_delta_workspace_bytes(heads, 1, 1, 1 << 20, d, d, vla.VLA_BF16, ctypes.byref(VlaDeltaOpts(segments=n)), 0)
    one = heads * 4 * (d * d + 2 * d * d)       # a segment's map and state
    assert ask(256) <= 256 * one and ask(256) == ask(255)
    assert (ask(256) // one) * heads * 4 * 2 * d < 1 << 32
    assert lib.vla_delta_workspace_bytes(1 << 20, 1, 1, 4096, d, d, vla.VLA_BF16, ctypes.byref(VlaDeltaOpts(segments=2)), 0) == 0


@pytest.mark.gpu
def test_single_tokens_of_many_heads():
    """2^21 heads of 16 x 128: a workgroup of 256 for every 16 columns would take 2^32 work-items."""
    B, d_k, d_v = 2 ** 21 + 3, 16, 128
    torch.cuda.empty_cache()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    q, k, v = (rnd(4099, 1, d) for d in (d_k, d_k, d_v))
    k = k / k.norm(dim=-1, keepdim=True)
    g, beta, S = -torch.rand(4099, 1, device="cuda"), torch.rand(4099, 1, device="cuda"), rnd(4099, 1, d_v, d_k)
    every = torch.arange(B, device="cuda") % 4099
    many = [x[every] for x in (q, k, v, g, beta, S)]
    o = vla.gated_delta_decode_step(*many)
    want = vla.gated_delta_decode_step(q, k, v, g, beta, S)
    for part in (slice(0, 4099), slice(B - 5000, B)):
        scale = want.abs().amax()
        assert (o[part] - want[every[part]]).abs().max() <= 1e-5 * scale
        assert (many[5][part] - S[every[part]]).abs().max() <= 1e-5 * S.abs().max()
    del many, o
    torch.cuda.empty_cache()

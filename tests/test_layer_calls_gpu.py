"""Calls of the operators around the recurrence as programs make them: on other streams, again with tensors that start elsewhere, with the time
segments that the library chooses, without memory beyond the caller's; the gradients of the norm against differences in both types; how
often a bfloat16 result is not the nearest one (GPU)."""
import ctypes

import pytest
import torch

import paper_2605_11196_amd as vla
from paper_2605_11196_amd.binding import VlaDeltaOpts, VlaNormOpts
from test_gated_delta_backward_gpu import check
from test_gated_delta_gpu import DT, make, oracle
from test_qk_norm_gpu import make as make_norm
from test_qk_norm_gpu import oracle as norm_oracle
from test_qk_norm_gpu import tables

pytestmark = pytest.mark.gpu


# ---- the time segments that the library chooses

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_k,d_v,T", [(64, 64, 1100), (128, 128, 900), (32, 16, 700)])
def test_chosen_segments_with_gradients_and_ragged_lengths(d_k, d_v, T, dtype):
    B, H_k, H_v = 3, 1, 2
    op, io = VlaDeltaOpts(), vla.VLA_F32 if dtype == "f32" else vla.VLA_BF16
    assert vla.load_library().vla_delta_workspace_bytes(B, H_k, H_v, T, d_k, d_v, io, ctypes.byref(op), 0) > 0      # it cuts these calls
    lengths = torch.tensor([T, T // 3 + 5, 0], device="cuda", dtype=torch.int32)
    check(make(B, H_k, H_v, T, d_k, d_v, dtype, seed=T, rate=0.05), dtype, lengths=lengths)


# ---- streams

def test_gradients_on_another_stream():
    """By the argument, and by torch's current stream in the forward pass (the backward pass goes to the same one)."""
    inputs = make(2, 2, 4, 700, 64, 64, "bf16", seed=31)
    do, dS = torch.randn_like(inputs[2]), torch.randn_like(inputs[5])
    nq, nk, wq, wk, dq, dk = make_norm(2, 300, 4, 2, 64, "bf16", seed=32)

    def raw(stream=None):
        o, S, saved = vla.gated_delta_forward(*inputs, save_for_backward=True, stream=stream)
        back = vla.gated_delta_backward(*inputs[:5], saved, do, dS, stream=stream)
        return [o, S, *back, *vla.qk_norm_rope_backward(nq, nk, wq, wk, None, None, dq, dk, stream=stream)]

    def differentiated():
        leaves = [x.detach().requires_grad_() for x in inputs]
        norm_leaves = [x.detach().requires_grad_() for x in (nq, nk, wq, wk)]
        o, S = vla.gated_delta(*leaves)
        return [o.detach(), S.detach(), *torch.autograd.grad((o, S), leaves, (do, dS)),
                *torch.autograd.grad(vla.qk_norm_rope(*norm_leaves), norm_leaves, (dq, dk))]

    want = raw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = raw(side)
    with torch.cuda.stream(side):
        also = differentiated()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(torch.equal(x, y) for x, y in zip(also, want))


# ---- a call like an earlier one, its tensors elsewhere

def test_weights_and_tables_of_a_repeated_call_may_start_anywhere():
    q, k, wq, wk, dq, dk = make_norm(2, 9, 4, 2, 32, "f32", seed=33)
    cos, sin = tables(9, 16)
    want = vla.qk_norm_rope(q, k, wq, wk, cos, sin)
    grads = vla.qk_norm_rope_backward(q, k, wq, wk, cos, sin, dq, dk)

    def moved(x):
        room = torch.empty(x.numel() + 1, device="cuda", dtype=x.dtype)
        return room[1:].view(x.shape).copy_(x)

    for i in range(2, 6):
        args = [q, k, wq, wk, cos, sin]
        args[i] = moved(args[i])
        assert args[i].data_ptr() % 16
        assert all(torch.equal(x, y) for x, y in zip(vla.qk_norm_rope(*args), want))
        assert all(torch.equal(x, y) for x, y in zip(vla.qk_norm_rope_backward(*args, dq, dk), grads))


# ---- memory

def test_the_entry_points_allocate_nothing():
    """The device's free memory before and after calls with the caller's buffers alone (a first call may load code)."""
    lib, stream = vla.load_library(), torch.cuda.current_stream().cuda_stream
    B, H_k, H_v, T, d, io = 2, 1, 2, 700, 64, vla.VLA_BF16
    q, k, v, g, beta, S = make(B, H_k, H_v, T, d, d, "bf16", seed=34)
    o, dq, dk, dv, do = (torch.empty_like(x) for x in (v, q, k, v, v))
    S_T, dS0, dg, dbeta = torch.empty_like(S), torch.empty_like(S), torch.empty_like(g), torch.empty_like(g)
    w, dw = torch.ones(d, device="cuda"), torch.empty(d, device="cuda")
    p = lambda *tensors: [x.data_ptr() for x in tensors]
    kept = lib.vla_delta_saved_bytes(B, H_v, T, d, d, io)
    saved = torch.empty(kept, dtype=torch.uint8, device="cuda")
    op = VlaDeltaOpts(saved=saved.data_ptr(), saved_bytes=kept)
    sizes = [lib.vla_delta_workspace_bytes(B, H_k, H_v, T, d, d, io, ctypes.byref(op), back) for back in (0, 1)]
    sizes.append(lib.vla_qk_norm_rope_workspace_bytes(d))
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    norm = VlaNormOpts(eps=1e-6)
    nq, nk, nqo, nko = (torch.randn(B, 2, T, d, device="cuda").bfloat16() for _ in range(4))

    def calls():
        rc = lib.vla_delta_forward(*p(q, k, v, g, beta, S, o, S_T), B, H_k, H_v, T, d, d, io, ctypes.byref(op), ws.data_ptr(), sizes[0], stream)
        rc |= lib.vla_delta_backward(*p(q, k, v, g, beta, do, S_T, dq, dk, dv, dg, dbeta, dS0), B, H_k, H_v, T, d, d, io, ctypes.byref(op),
                                     ws.data_ptr(), sizes[1], stream)
        rc |= lib.vla_delta_decode_step(*p(q, k, v, g, beta, S_T, o), B, H_k, H_v, d, d, io, None, stream)
        rc |= lib.vla_qk_norm_rope(*p(nq, nk, w, w), None, None, *p(nqo, nko), B, T, 2, 2, d, io, ctypes.byref(norm), stream)
        rc |= lib.vla_qk_norm_rope_backward(*p(nq, nk, w, w), None, None, *p(nqo, nko, dv, o), dw.data_ptr(), None, B, T, 2, 2, d, io,
                                            ctypes.byref(norm), ws.data_ptr(), sizes[2], stream)
        torch.cuda.synchronize()
        return rc

    assert calls() == 0
    free = torch.cuda.mem_get_info()[0]
    for _ in range(20):
        assert calls() == 0
    assert torch.cuda.mem_get_info()[0] == free


# ---- the norm's gradients against differences

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved,l2", [(False, False), (True, True)])
def test_norm_gradients_against_differences(interleaved, l2, dtype):
    """Central differences of the float64 oracle along random directions; their own error is about 1e-9 at a step of 1e-4.  The sum along a direction u
    is off by the gradients' roundings, at most 2^-8 of |dx| |u| in bfloat16 and 1e-5 in float32, and independent of each other; the weights' gradients are
    float32 in both."""
    inputs = make_norm(2, 5, 3, 2, 32, dtype, seed=35)
    q, k, wq, wk, dq, dk = inputs
    cos, sin = tables(5, 16)
    place = torch.arange(5, device="cuda")[None].expand(2, 5)
    got = vla.qk_norm_rope_backward(q, k, wq, wk, cos, sin, dq, dk, eps=1e-6, norm="l2" if l2 else "rms", interleaved=interleaved)
    for x, w, dy, dx, dw in ((q, wq, dq, got[0], got[2]), (k, wk, dk, got[1], got[3])):
        loss = lambda x, w: (norm_oracle(x, w, cos, sin, place, eps=1e-6, l2=l2, interleaved=interleaved) * dy.double()).sum()
        assert dx.shape == x.shape and dx.dtype == x.dtype and dw.dtype == w.dtype
        h = 1e-4
        for value, grad, other, limit in ((x, dx, w, 1e-5 if dtype == "f32" else 2.0 ** -8), (w, dw, x, 1e-5)):
            for _ in range(4):
                u = torch.randn(value.shape, device="cuda", dtype=torch.float64)
                at = (lambda z: loss(z, other)) if value is x else (lambda z: loss(other, z))
                along = (at(value.double() + h * u) - at(value.double() - h * u)) / (2 * h)
                assert abs((grad.double() * u).sum() - along) <= limit * grad.double().norm() * u.norm()


# ---- bfloat16 results against the nearest ones

def test_how_often_bfloat16_results_are_not_the_nearest():
    """o and dk are formed from factors of 16 bits (two bfloat16 terms) and summed in float32 before their one rounding, dq and dv from all of a factor's bits.
    An error of e, in units of the last place, moves a result to the neighbouring number in the share 2 E|e| of the cases.  A factor cut to 16 bits is
    off by 2^-17 of itself at most (2^-18 in the mean), 2^-9 units of a result of the products' size, and a result of some products of either sign is
    a few times smaller than what their errors add up to: 2 x 4 x 2^-9 = 1.6 % at most.  All bits: float32 roundings, 2^-24 a product, 40 of them: 2 x 40 x 2^-16 =
    0.12 %.  (Factors of one bfloat16 term would give more than half.)"""
    inputs = make(2, 2, 2, 400, 64, 64, "bf16", seed=36, rate=0.05)
    q, k, v, g, beta, S0 = inputs
    do, dS = torch.randn_like(v), torch.randn_like(S0)
    o, S, saved = vla.gated_delta_forward(*inputs, save_for_backward=True)
    dq, dk, dv = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS)[:3]
    leaves = [x.double().requires_grad_() for x in inputs]
    ro, rS = oracle(*leaves)
    want = torch.autograd.grad((ro, rS), leaves[:3], (do.double(), dS.double()))
    for name, x, y, share in (("o", o, ro, 0.016), ("dk", dk, want[1], 0.016), ("dq", dq, want[0], 0.0012), ("dv", dv, want[2], 0.0012)):
        assert x.dtype == DT["bf16"]
        moved = (x != y.detach().bfloat16()).float().mean().item()
        print(f"{name}: {moved:.2e} of the values are not the nearest")
        assert moved <= share, (name, moved)

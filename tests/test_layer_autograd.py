"""What the autograd functions of the operators around the recurrence hand to the library (CPU only: calls that would launch kernels are
recorded, with their options as they are at the call).

Saved tensors may come back as other ones: hooks that offload or pack them give copies with other strides at other addresses, and a
checkpointed layer forms them again.  The library knows addresses and strides but no sizes, so the two have to be those of the tensors that the backward
pass holds."""
import contextlib
import ctypes
import importlib

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2605_11196_amd as vla
from paper_2605_11196_amd import binding
from paper_2605_11196_amd.binding import VlaDeltaOpts, VlaNormOpts, VlaStrides

gated_delta, qk_norm = (importlib.import_module("paper_2605_11196_amd." + n) for n in ("gated_delta", "qk_norm"))

LAUNCHES = {"vla_delta_forward": (VlaDeltaOpts, 15), "vla_delta_decode_step": (VlaDeltaOpts, 13), "vla_delta_backward": (VlaDeltaOpts, 20),
            "vla_qk_norm_rope": (VlaNormOpts, 14), "vla_qk_norm_rope_backward": (VlaNormOpts, 18)}   # options, their place among the arguments


class Recorder:
    """The library, with what it would launch as entries (name, arguments, options) of `calls`."""

    def __init__(self):
        self.lib, self.calls = binding.load_library(), []

    def __getattr__(self, name):
        if name not in LAUNCHES:
            return getattr(self.lib, name)
        kind, place = LAUNCHES[name]

        def launch(*args):
            self.calls.append((name, args, kind.from_buffer_copy(args[place]._obj)))
            return 0

        return launch

    def last(self, name):
        return next(c for c in reversed(self.calls) if c[0] == name)


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(binding, "load_library", lambda: r)
    monkeypatch.setattr(binding, "_on_stream", lambda torch, dev, stream: (0, contextlib.nullcontext(), None))
    for module in (gated_delta, qk_norm):
        monkeypatch.setattr(module, "_check", lambda *a: None)   # refuses tensors that are not on the GPU
        monkeypatch.setattr(module, "_plans", {})
    return r


def dense(x):
    return x.clone(memory_format=torch.contiguous_format)


def turned(x):
    """Tokens before heads, whatever the order was."""
    return x.transpose(1, 2).clone(memory_format=torch.contiguous_format).transpose(1, 2) if x.dim() >= 3 else x.clone()


def off_by_one(x):
    """Not at a 16-byte boundary."""
    room = torch.empty(x.numel() + 1, dtype=x.dtype)
    return room[1:].view(x.shape).copy_(x)


class Hooks:
    """Saved tensors come back as copies, which stay here."""

    def __init__(self, layout):
        self.layout, self.copies = layout, []

    def unpack(self, x):
        self.copies.append(self.layout(x))
        return self.copies[-1]

    def __enter__(self):
        self.context = torch.autograd.graph.saved_tensors_hooks(lambda x: x, self.unpack)
        return self.context.__enter__()

    def __exit__(self, *args):
        return self.context.__exit__(*args)


def read(address, strides, shape, dtype, contiguous):
    """The tensor that the library would read."""
    steps = (strides.b, strides.h, strides.t)[:len(shape[:3])]
    if not any(steps):
        steps = contiguous[:len(steps)]
    reach = sum(s * (n - 1) for s, n in zip(steps, shape)) + (shape[3] if len(shape) > 3 else 1)
    kind = {torch.float32: ctypes.c_float, torch.bfloat16: ctypes.c_int16, torch.int32: ctypes.c_int32}[dtype]
    flat = torch.frombuffer((kind * reach).from_address(address), dtype=dtype)
    return flat.as_strided(shape, (*steps, 1)[:len(shape)])


def holds(address, strides, copies, want):
    """Whether one of `copies` starts at the address, covers what the strides reach and reads as `want`."""
    shape, contiguous = tuple(want.shape), want.contiguous().stride()
    steps = (strides.b, strides.h, strides.t)
    steps = steps if any(steps) else contiguous[:3]
    reach = sum(s * (n - 1) for s, n in zip(steps, shape)) + (shape[3] if len(shape) > 3 else 1)
    for x in copies:
        end = x.untyped_storage().data_ptr() + x.untyped_storage().nbytes()
        if x.data_ptr() == address and address + reach * want.element_size() <= end:
            return torch.equal(read(address, strides, shape, want.dtype, contiguous), want)
    return False


def fused(B, T, H_k, H_v, d, seed=0):
    """Leaves: rows of a projection and of its gates; q, k, v, g, beta as their slices, and S0."""
    gen = torch.Generator().manual_seed(seed)
    rows = torch.randn((B, T, (2 * H_k + H_v) * d), generator=gen).requires_grad_()
    gates = torch.randn((B, T, 2 * H_v), generator=gen).requires_grad_()
    q, k, v = rows.view(B, T, -1, d).transpose(1, 2).split((H_k, H_k, H_v), 1)
    g, beta = gates.transpose(1, 2).split(H_v, 1)
    return (rows, gates), (q, k, v, g, beta), torch.randn((B, H_v, d, d), generator=gen)


@pytest.mark.parametrize("layout", [dense, turned, off_by_one])
def test_the_delta_rules_gradients_read_the_unpacked_tensors(recorder, layout):
    B, T, H_k, H_v, d = 3, 40, 2, 4, 32
    leaves, inputs, S0 = fused(B, T, H_k, H_v, d)
    lengths = torch.tensor([5, 40, 17], dtype=torch.int32)
    for _ in range(2):      # the second time as a call like an earlier one
        hooks = Hooks(layout)
        with hooks:
            o, S = vla.gated_delta(*inputs, S0.requires_grad_(), lengths=lengths)
        (o.sum() + S.sum()).backward(inputs=(*leaves, S0))
        name, args, op = recorder.calls[-1]
        copies = hooks.copies
        assert name == "vla_delta_backward" and len(copies) >= 7
        own = {x.data_ptr() for x in copies}
        for i, x in enumerate(inputs):
            name = ("q", "k", "v", "g", "beta")[i]
            if layout is off_by_one and i < 3:
                assert args[i] not in own and args[i] % 16 == 0 and not any((getattr(op, name).b, getattr(op, name).h, getattr(op, name).t)), name
            else:
                assert holds(args[i], getattr(op, name), copies, x.detach()), name
        assert holds(op.lengths, VlaStrides(), copies, lengths)
        assert op.saved in own or layout is off_by_one
        assert [args[i] for i in range(13, 19)] == [B, H_k, H_v, T, d, d]
        del o, S


def test_a_checkpointed_delta_rule_reads_the_lengths_that_are_formed_again(recorder):
    leaves, inputs, _ = fused(2, 20, 1, 2, 16)
    made = []

    def layer(q, k, v, g, beta):
        made.append(torch.tensor([7, 20], dtype=torch.int32))
        return vla.gated_delta(q, k, v, g, beta, lengths=made[-1])[0]

    o = checkpoint(layer, *inputs, use_reentrant=False)
    first = recorder.last("vla_delta_forward")[2].lengths
    o.sum().backward()
    assert len(made) == 2 and first == made[0].data_ptr()
    assert recorder.last("vla_delta_backward")[2].lengths == made[1].data_ptr()


@pytest.mark.parametrize("layout", [dense, turned, off_by_one])
@pytest.mark.parametrize("rotated", [False, True])
def test_the_norms_gradients_read_the_unpacked_tensors(recorder, layout, rotated):
    B, T, H_q, H_k, d = 3, 11, 4, 2, 32
    rows = torch.randn((B, T, (H_q + H_k) * d)).requires_grad_()
    q, k = rows.view(B, T, -1, d).transpose(1, 2).split((H_q, H_k), 1)
    weights = [torch.rand(d).requires_grad_() for _ in range(2)]
    tables = [torch.rand(20, 8) for _ in range(2)] if rotated else [None, None]
    positions = torch.randint(0, 20, (1, T), dtype=torch.int32).expand(B, T) if rotated else None
    for _ in range(2):      # the second time as a call like an earlier one
        hooks = Hooks(layout)
        with hooks:
            out = vla.qk_norm_rope(q, k, *weights, *tables, positions=positions, eps=1e-5, norm="l2", interleaved=True, offset=2)
        (out[0].sum() + out[1].sum()).backward(inputs=(rows, *weights))
        name, args, op = recorder.calls[-1]
        assert name == "vla_qk_norm_rope_backward"
        own = {x.data_ptr() for x in hooks.copies}
        for i, (x, n) in enumerate(((q, "q"), (k, "k"))):
            if layout is off_by_one:
                assert args[i] not in own and args[i] % 16 == 0
            else:
                assert holds(args[i], getattr(op, n), hooks.copies, x.detach()), n
        for i, x in enumerate((*weights, *tables)):
            assert (args[2 + i] is None) if x is None else (args[2 + i] % 16 == 0 if layout is off_by_one else args[2 + i] in own)
        if rotated:
            assert holds(op.positions, VlaStrides(), hooks.copies, positions.contiguous())
        assert (op.l2, op.interleaved, op.offset, op.rot, op.places) == (1, 1, 2, 16 if rotated else 0, 20 if rotated else 0)
        assert abs(op.eps - 1e-5) < 1e-11 and [args[i] for i in range(12, 16)] == [B, T, H_q, H_k]


def test_a_checkpointed_norm_reads_the_positions_that_are_formed_again(recorder):
    q, k, tables = torch.randn(2, 3, 5, 16).requires_grad_(), torch.randn(2, 1, 5, 16), [torch.rand(20, 8) for _ in range(2)]
    made = []

    def layer(q):
        made.append(torch.arange(10, dtype=torch.int32).view(2, 5))
        return vla.qk_norm_rope(q, k, None, None, *tables, positions=made[-1])[0]

    y = checkpoint(layer, q, use_reentrant=False)
    first = recorder.last("vla_qk_norm_rope")[2].positions
    y.sum().backward()
    assert len(made) == 2 and first == made[0].data_ptr()
    assert recorder.last("vla_qk_norm_rope_backward")[2].positions == made[1].data_ptr()


@pytest.mark.parametrize("change", [lambda x: x.float(), lambda x: x.to("meta"), lambda x: x.repeat_interleave(2)[::2], lambda x: x.view(16, -1)])
def test_what_was_saved_is_looked_at(recorder, change):
    """An address of another device or a tensor with gaps would be read all the same: the library sees an address and a size."""
    _, inputs, _ = fused(1, 20, 1, 1, 32)
    inputs = [x.detach() for x in inputs]
    saved = torch.zeros(binding.load_library().vla_delta_saved_bytes(1, 1, 20, 32, 32, 0), dtype=torch.uint8)
    with pytest.raises(ValueError, match="saved"):
        vla.gated_delta_backward(*inputs, change(saved), inputs[2])
    vla.gated_delta_backward(*inputs, saved, inputs[2])
    assert recorder.last("vla_delta_backward")[2].saved == saved.data_ptr()


def test_states_and_their_gradients_may_start_anywhere(recorder):
    """A state cut out of a larger buffer, and the gradient that torch.cat gives back: contiguous, not at a 16-byte boundary."""
    _, inputs, S0 = fused(1, 20, 1, 1, 16)
    inputs = [x.detach() for x in inputs]
    S0 = off_by_one(S0).requires_grad_()
    assert S0.data_ptr() % 16 and S0.is_contiguous()
    o, S = vla.gated_delta(*inputs, S0)
    address = recorder.last("vla_delta_forward")[1][5]
    assert address % 16 == 0 and address != S0.data_ptr()
    torch.cat((torch.ones(1), S.flatten())).sum().backward()
    address = recorder.last("vla_delta_backward")[1][6]
    assert address % 16 == 0 and address


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32 + 3, -2 ** 40])
def test_numbers_that_32_bits_do_not_hold_are_refused(recorder, number):
    """ctypes would cut them: position 3 in the place of 2^32 + 3."""
    _, inputs, _ = fused(1, 20, 1, 1, 32)
    q, k, v, g, beta = (x.detach() for x in inputs)
    tables = [torch.rand(64, 16) for _ in range(2)]
    saved = torch.zeros(binding.load_library().vla_delta_saved_bytes(1, 1, 20, 32, 32, 0), dtype=torch.uint8)
    for call in (lambda: vla.qk_norm_rope(q, k, None, None, *tables, offset=number),
                 lambda: vla.qk_norm_rope_backward(q, k, None, None, *tables, q, k, offset=number),
                 lambda: vla.gated_delta_forward(q, k, v, g, beta, segments=number),
                 lambda: vla.gated_delta_backward(q, k, v, g, beta, saved, v, segments=number)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    vla.qk_norm_rope(q, k, None, None, *tables, offset=2 ** 31 - 1)
    assert recorder.calls[-1][2].offset == 2 ** 31 - 1


def test_sizes_that_32_bits_do_not_hold_are_refused():
    """2^32 + 5 tokens would be taken for 5."""
    x = torch.empty((1, 1, 2 ** 32 + 5, 16), device="meta")
    gate = torch.empty((1, 1, 2 ** 32 + 5), device="meta")
    with pytest.raises(ValueError, match="32 bits"):
        vla.qk_norm_rope(x, x)
    with pytest.raises(ValueError, match="32 bits"):
        vla.gated_delta_forward(x, x, x, gate, gate)
    one = torch.empty((2 ** 31, 1, 16), device="meta")
    with pytest.raises(ValueError, match="32 bits"):
        vla.gated_delta_decode_step(one, one, one, one[..., 0], one[..., 0], torch.empty((2 ** 31, 1, 16, 16), device="meta"))


@pytest.mark.parametrize("wanted", [(), (0,), (1,), (0, 1)])
def test_gradients_of_frozen_weights_are_not_formed(recorder, wanted):
    q, k = torch.randn(2, 3, 5, 16).requires_grad_(), torch.randn(2, 1, 5, 16)
    weights = [torch.rand(16).requires_grad_(i in wanted) for i in range(2)]
    out = vla.qk_norm_rope(q, k, *weights)
    (out[0].sum() + out[1].sum()).backward()
    args = recorder.last("vla_qk_norm_rope_backward")[1]
    assert [i for i in range(2) if args[10 + i] is not None] == list(wanted)
    assert (args[19] is not None) == bool(wanted) and (args[20] > 0) == bool(wanted)       # the workspace of the sums
    assert [w.grad is not None for w in weights] == [i in wanted for i in range(2)]


@pytest.mark.parametrize("state", ["none", "frozen", "learned"])
def test_the_gradient_of_a_state_that_nothing_asks_for_is_not_formed(recorder, state):
    _, inputs, S0 = fused(1, 20, 1, 1, 16)
    S0 = None if state == "none" else S0.requires_grad_(state == "learned")
    o, S = vla.gated_delta(*inputs, S0)
    (o.sum() + S.sum()).backward()
    assert (recorder.last("vla_delta_backward")[1][12] is not None) == (state == "learned")
    assert S0 is None or (S0.grad is not None) == (state == "learned")


def test_a_single_token_has_no_gradient_and_says_so(recorder):
    """The state is updated in place without a graph: inputs that ask for gradients are refused, what saved the state learns of the update."""
    names = ("q", "k", "v", "g", "beta", "S")
    made = lambda: dict(zip(names, [torch.randn(2, 1, 16) for _ in range(3)] + [torch.randn(2, 1) for _ in range(2)] + [torch.randn(2, 1, 16, 16)]))
    for name in names:
        inputs = made()
        vla.gated_delta_decode_step(**inputs)
        inputs[name].requires_grad_()
        with pytest.raises(ValueError, match="no_grad"):
            vla.gated_delta_decode_step(**inputs)
        with torch.no_grad():
            vla.gated_delta_decode_step(**inputs)
    inputs = made()
    w = torch.randn(2, 1, 16, 16).requires_grad_()
    y = (w * inputs["S"]).sum()          # saves S
    with torch.no_grad():
        vla.gated_delta_decode_step(**inputs)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    with torch.inference_mode():
        vla.gated_delta_decode_step(**made())


def test_forward_mode_tangents_are_refused(recorder):
    """There are gradients in reverse alone; a tangent was dropped where no input asked for one of those."""
    import torch.autograd.forward_ad as forward_ad

    _, inputs, _ = fused(1, 4, 1, 1, 16)
    q, k, v, g, beta = (x.detach() for x in inputs)
    one = [x[:, :, 0] for x in (q, k, v, g, beta)]
    with forward_ad.dual_level():
        vla.gated_delta(q, k, v, g, beta)
        vla.qk_norm_rope(q, k)
        with torch.no_grad():
            vla.gated_delta_decode_step(*one, torch.zeros(1, 1, 16, 16))
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        for call in (lambda: vla.gated_delta(dual, k, v, g, beta), lambda: vla.qk_norm_rope(dual, k),
                     lambda: vla.gated_delta_decode_step(dual[:, :, 0], *one[1:], torch.zeros(1, 1, 16, 16))):
            with pytest.raises(NotImplementedError, match="jvp"):
                call()

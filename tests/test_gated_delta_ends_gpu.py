"""What lies past the end of a sequence, where the sequence itself holds infinities or NaN (GPU): later tokens are not part of it, their outputs
and gradients are 0."""
import pytest
import torch

import paper_2605_11196_amd as vla
from test_gated_delta_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H_k", [2, 4])
@pytest.mark.parametrize("segments", [1, 4])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_outputs_and_gradients_past_the_end_are_zero(value, segments, H_k, dtype):
    T = 300
    lengths = torch.tensor([T, 270, 33, 20, 1, 0], device="cuda", dtype=torch.int32)
    q, k, v, g, beta, S0 = make(6, H_k, 4, T, 64, 64, dtype, seed=41, rate=0.01)
    v[:, 1, 10] = value
    S0[:, 2, 3, 5] = value
    o, S, saved = vla.gated_delta_forward(q, k, v, g, beta, S0, lengths=lengths, segments=segments, save_for_backward=True)
    do, dS = torch.randn_like(v), torch.randn_like(S0)
    grads = vla.gated_delta_backward(q, k, v, g, beta, saved, do, dS, lengths=lengths, segments=segments)
    plain = vla.gated_delta_forward(q, k, v, g, beta, S0, lengths=lengths, segments=segments)[0]
    for b, n in enumerate(lengths.tolist()):
        for x in (o, plain, *grads[:5]):
            assert (x[b, :, n:] == 0).all(), (b, n)
    assert not o[0, 2].isfinite().all() and not grads[0][0].isfinite().all()

"""The norm over more tokens than one dimension of a launch holds work-items for, 2^32 (GPU)."""
import pytest
import torch

import paper_2605_11196_amd as vla

pytestmark = pytest.mark.gpu


def test_more_tokens_than_a_launch_dimension_holds():
    """2^28 + 2^15 tokens of 128 columns take 16 lanes each; a batch that repeats one sequence gives the same rows everywhere."""
    B, T, d = 2 ** 13 + 1, 2 ** 15, 128
    torch.cuda.empty_cache()
    one = torch.randn((1, 1, T, d), device="cuda").bfloat16()
    want, _ = vla.qk_norm_rope(one, one[:, :0])
    got, none = vla.qk_norm_rope(one.expand(B, 1, T, d), one[:, :0].expand(B, 0, T, d))
    assert got.shape == (B, 1, T, d) and none.numel() == 0
    for b in (0, 1, 2 ** 12, 2 ** 13 - 1, 2 ** 13):
        assert torch.equal(got[b], want[0]), b
    assert torch.equal(got[:, 0, :64].amin(0), want[0, 0, :64]) and torch.equal(got[:, 0, :64].amax(0), want[0, 0, :64])
    del got
    torch.cuda.empty_cache()

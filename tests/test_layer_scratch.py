"""Build-time check of scratch memory over every instance of the gated delta rule's kernels (CPU only: hipcc cross-compiles): none keeps more
bytes a lane there than is stated here, with the reason."""
import glob
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_11196_amd import build

# Bytes a lane of the instances that use any: types, d_k, d_v (and whether it forms maps).  All of them run at 128 registers, because four waves share
# a SIMD: two workgroups of d_v / 16 (gradients: d_k / 16) waves a compute unit, or one of the maps' 14 to 16 waves, which cannot have more.
# float32 blocks and gradients of 96 and 128 columns: operands of the FP32 matrix instruction are twice as wide as bfloat16 ones beside the same state (at
# most 18 scratch instructions in the loop over blocks, of some 2000 instructions).  bfloat16 values of 64 and 96 columns beside wider keys: four or six waves form six
# matrices between tokens, and the gradients of 64 have the next rows on registers (up to 9).  "bf16, 16, 64" and "bf16, 64, 96" set bytes aside and
# use none.  The others are addresses outside the loops.
ALLOWED = {
    "delta_chunk_kernel": {
        "f32, 128, 128, false": 48, "f32, 128, 128, true": 44, "f32, 128, 96, true": 124, "f32, 96, 128, false": 44, "f32, 96, 128, true": 36,
        "f32, 64, 96, false": 12, "bf16, 128, 64, false": 40, "bf16, 128, 96, false": 20, "bf16, 128, 96, true": 16, "bf16, 16, 64, false": 68,
        "bf16, 64, 96, false": 68, "bf16, 96, 64, false": 20},
    "delta_reverse_kernel": {
        "f32, 128, 128, false": 20, "f32, 128, 128, true": 20, "f32, 128, 96, true": 84, "f32, 96, 128, true": 12, "bf16, 128, 64, false": 20},
    "delta_grad_kernel": {
        "f32, 128, 64": 68, "bf16, 128, 128": 16, "bf16, 128, 96": 12, "bf16, 128, 64": 32, "bf16, 128, 32": 8, "bf16, 128, 16": 8, "bf16, 96, 32": 16,
        "bf16, 96, 16": 16, "bf16, 64, 32": 8},
}


@pytest.fixture(scope="module")
def scratch():
    """{kernel: {template arguments: bytes a lane}}"""
    sources = sorted(glob.glob(os.path.join(build.CSRC, "delta_*.hip")))
    with ThreadPoolExecutor(8) as pool:
        reports = list(pool.map(build.resource_usage, sources))
    out = {}
    for report in reports:
        for name, r in report.items():
            m = re.search(r"(\w+)<([^(]*)>\(", name)
            out.setdefault(m.group(1), {})[m.group(2).replace("unsigned short", "bf16").replace("float", "f32")] = r["ScratchSize"]
    return out


@pytest.mark.parametrize("kernel,instances", [("delta_chunk_kernel", 100), ("delta_reverse_kernel", 100), ("delta_grad_kernel", 50),
                                              ("delta_step_kernel", 10), ("delta_combine_kernel", 5), ("delta_shared_kernel", 2)])
def test_scratch_memory_of_every_instance(scratch, kernel, instances):
    allowed = ALLOWED.get(kernel, {})
    assert len(scratch[kernel]) == instances and set(allowed) <= set(scratch[kernel])
    over = {args: n for args, n in scratch[kernel].items() if n > allowed.get(args, 0)}
    assert not over, over

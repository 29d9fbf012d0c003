"""Build-time check of the registers and the LDS the compiler gives the kernels of the gated delta rule and of the norm (CPU only: hipcc
cross-compiles).

The block kernels keep a state of d_k x 16 numbers a wave on registers at the limit of 128, where four waves run on a SIMD: a change that
pushes the state into scratch memory inside the token loop, or the second workgroup off a compute unit, fails no numerical test."""
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_11196_amd import build

LDS = 160 * 1024   # of a compute unit


@pytest.fixture(scope="module")
def usage():
    """{(kernel, template arguments): resources}"""
    sources = ["delta_chunk_128.hip", "delta_chunk_64.hip", "delta_reverse_128.hip", "delta_grad_128.hip", "delta_step.hip", "delta_combine.hip",
               "qk_norm_rope.hip"]
    with ThreadPoolExecutor(len(sources)) as pool:
        reports = list(pool.map(lambda f: build.resource_usage(os.path.join(build.CSRC, f)), sources))
    out = {}
    for report in reports:
        for name, r in report.items():
            m = re.search(r"(\w+)<([^(]*)>\(", name)
            if m:
                out[m.group(1), m.group(2).replace("unsigned short", "bf16").replace("float", "f32")] = r
    return out


@pytest.mark.parametrize("kernel,args", [("delta_chunk_kernel", "bf16, 128, 128, false"), ("delta_chunk_kernel", "bf16, 64, 64, false"),
                                         ("delta_reverse_kernel", "bf16, 128, 128, false")])
def test_two_workgroups_of_a_compute_unit(usage, kernel, args):
    r = usage[kernel, args]
    waves = r["Threads"] // 64
    assert r["ScratchSize"] == 0 and r["Occupancy"] >= waves // 2 and 2 * r["LDSSize"] <= LDS, r


@pytest.mark.parametrize("kernel", ["delta_chunk_kernel", "delta_reverse_kernel"])
def test_the_maps_of_segments_keep_their_state_on_registers(usage, kernel):
    r = usage[kernel, "bf16, 128, 128, true"]
    assert r["Threads"] == 1024 and r["ScratchSize"] == 0 and r["Occupancy"] >= 4 and r["LDSSize"] <= LDS, r


def test_the_gradients_run_two_workgroups_of_a_compute_unit(usage):
    r = usage["delta_grad_kernel", "bf16, 128, 128"]
    assert r["Occupancy"] >= 4 and 2 * r["LDSSize"] <= LDS and r["ScratchSize"] <= 16, r      # addresses, outside the products


def test_kernels_bound_by_memory_use_no_scratch(usage):
    seen = 0
    for (kernel, args), r in usage.items():
        if kernel not in ("delta_chunk_kernel", "delta_reverse_kernel", "delta_grad_kernel"):
            assert r["ScratchSize"] == 0, (kernel, args, r)
            seen += 1
    assert seen >= 10

"""Build-time check of the registers that the compiler gives the kernels on rows of channels (CPU only: hipcc cross-compiles).

Two things fail no numerical test for certain: scratch memory inside a loop over tokens, and accumulation registers.  With more than 256 values
alive the compiler keeps some of them (addresses too) in accumulation registers, and it has written them while the lanes that leave a divergent branch were
still switched off, so that those lanes went on with garbage."""
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_11196_amd import build

SOURCES = ["causal_conv", "selective_scan", "selective_backward", "selective_step", "residual_norm"]
LDS = 160 * 1024   # of a compute unit


@pytest.fixture(scope="module")
def usage():
    """{(kernel, template arguments): resources}"""
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        reports = list(pool.map(lambda f: build.resource_usage(os.path.join(build.CSRC, f + ".hip")), SOURCES))
    out = {}
    for report in reports:
        for name, r in report.items():
            m = re.search(r"(\w+)(?:<([^(]*)>)?\(", name.replace("(anonymous namespace)::", ""))
            out[m.group(1), (m.group(2) or "").replace("unsigned short", "bf16").replace("float", "f32")] = r
    return out


def test_no_kernel_uses_accumulation_registers_or_scratch(usage):
    assert len(usage) >= 60
    for key, r in usage.items():
        assert r["AGPRs"] == 0 and r["ScratchSize"] == 0 and r["VGPRSpill"] == 0, (key, r)


@pytest.mark.parametrize("kernel,args,waves", [
    ("scan_kernel", "16, bf16, false", 2), ("backward_kernel", "16, bf16, false", 2), ("backward_kernel", "64, f32, false", 2),
    ("residual_kernel", "bf16, bf16, true", 6), ("residual_backward_kernel", "bf16, bf16, true", 4), ("residual_backward_kernel", "f32, f32, true", 4),
    ("conv_kernel", "4, bf16", 3), ("conv_step_kernel", "4, bf16", 7), ("step_kernel", "16, bf16", 8)])
def test_waves_of_a_simd(usage, kernel, args, waves):
    r = usage[kernel, args]
    assert r["Occupancy"] >= waves and r["LDSSize"] <= LDS, r

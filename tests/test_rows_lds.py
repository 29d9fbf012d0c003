"""Build-time check of the shared arrays of the kernels on rows of channels (CPU only: hipcc cross-compiles): an array that takes 16-byte pieces has to be
declared at a 16-byte boundary, since the compiler places it by its declaration and takes the pieces' addresses as multiples of 16."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_11196_amd import build

SOURCES = ["causal_conv", "selective_scan", "selective_backward", "residual_norm"]
# as in the kernels' sources; `outs` takes pairs of floats alone
PIECES = {"causal_conv": {"of_run"}, "selective_scan": {"steps", "staged"}, "selective_backward": {"steps", "staged", "sums"}, "residual_norm": {"lds"}}


def shared_arrays(source):
    """{array: smallest alignment among the kernels' instances}, as declared (before the compiler's passes)."""
    flags = [*build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes"]
    text = subprocess.run([build.HIPCC, *flags, os.path.join(build.CSRC, source + ".hip"), "-o", "-"], capture_output=True, text=True, check=True).stdout
    out = {}
    for mangled, align in re.findall(r"^@(\S+) = [^\n]*addrspace\(3\) global [^\n]*align (\d+)", text, flags=re.M):
        for name in PIECES[source] | {"outs"}:
            if re.search(r"(?<![a-z_])(\d*)%s(?![a-z_])" % name, mangled):
                out[name] = min(out.get(name, 1 << 20), int(align))
    return out


@pytest.fixture(scope="module")
def arrays():
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(shared_arrays, SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_arrays_that_take_16_byte_pieces_are_aligned(arrays, source):
    found = arrays[source]
    assert PIECES[source] <= set(found), found
    for name in PIECES[source]:
        assert found[name] >= 16, (name, found)

"""Launches of the operators on rows of channels at the largest sizes that they take (CPU only: a stand-in for the runtime's launch writes down
what it is given).  A launch holds less than 2^32 work-items; the runtime wraps a larger one without an error, and what it leaves out stays unwritten."""
import json
import os
import subprocess
import sys

import pytest

from paper_2605_11196_amd import binding

RECORDER = r"""
#include <stdint.h>
#include <stdio.h>
typedef struct { uint32_t x, y, z; } dim3;
int hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, void* stream) {
  (void)f; (void)args; (void)lds; (void)stream;
  printf("[%u, %u, %u, %u, %u, %u]\n", grid.x, grid.y, grid.z, block.x, block.y, block.z);
  fflush(stdout);
  return 0;
}
"""

# the stand-in comes before the library, whose launches then go to it; addresses are never followed on the host
CALL = r"""
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
name, args = sys.argv[3], json.loads(sys.argv[4])
value = lambda a: ctypes.c_size_t(int(a)) if isinstance(a, str) else ctypes.c_int(a)
sys.path.insert(0, sys.argv[5])
from paper_2605_11196_amd.binding import VlaScanOpts
opts = None
if "scan" in name:
    opts = ctypes.pointer(VlaScanOpts(1, 1, saved=1 << 60, saved_bytes=1 << 50))
print(getattr(lib, name)(*(opts if a == "opts" else value(a) for a in args)))
"""


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    folder = tmp_path_factory.mktemp("recorder")
    source, out = folder / "launch.c", folder / "liblaunch.so"
    source.write_text(RECORDER)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(out), str(source)], check=True)
    return str(out)


def launches(recorder, name, args):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CALL, recorder, binding.lib_path(), name, json.dumps(args), root], capture_output=True, text=True, check=True)
    *grids, status = [json.loads(line) for line in r.stdout.splitlines()]
    return grids, status


def places(count):
    """Addresses a TiB and more apart, which no two buffers of these calls share."""
    return [str((i + 1) << 41) for i in range(count)]


ROOM = str(1 << 41)


@pytest.mark.parametrize("name,args", [
    # dA of 2^22 channels with 64 states: 2^28 columns
    ("vla_selective_scan_backward", [*places(19), 1, 1, 2 ** 22, 64, 1, "opts", str(100 << 41), ROOM, "0"]),
    # and of as many as are taken
    ("vla_selective_scan_backward", [*places(19), 1, 1, 2 ** 25 - 8, 64, 0, "opts", str(100 << 41), ROOM, "0"]),
    ("vla_causal_conv_backward", [*places(10), 1, 1, 2 ** 28, 2, 1, "0", str(100 << 41), ROOM, "0"]),
    ("vla_causal_conv_backward", [*places(10), 1, 1, 2 ** 31 - 8, 4, 1, "0", str(100 << 41), ROOM, "0"]),
    ("vla_causal_conv", [*places(6), 1, 1, 2 ** 31 - 8, 4, 1, "0", "0"]),
])
def test_every_launch_holds_its_work_items(recorder, name, args):
    grids, status = launches(recorder, name, args)
    assert status == 0 and grids
    for x, y, z, threads, *rest in grids:
        assert rest == [1, 1] and x >= 1 and x * threads < 2 ** 32 and y <= 65535 and z == 1 and threads <= 1024, grids


@pytest.mark.parametrize("name,place", [("vla_causal_conv", 4), ("vla_causal_conv_step", 4), ("vla_causal_conv_backward", 6)])
@pytest.mark.parametrize("n,width", [(2 ** 29, 4), (2 ** 30, 2), (2 ** 31 - 8, 4)])
def test_outputs_inside_the_taps_of_many_channels_are_refused(recorder, name, place, n, width):
    """An output that starts in the second half of taps [n, width] whose number passes 31 bits."""
    at = places(10)
    at[place] = str(int(at[1]) + n * width // 2 * 4)      # float32
    if name.endswith("step"):
        args = [*at[:5], 1, n, width, 1, "0", "0"]
    elif place == 4:
        args = [*at[:6], 1, 1, n, width, 1, "0", "0"]
    else:
        args = [*at, 1, 1, n, width, 1, "0", str(100 << 41), ROOM, "0"]
    assert launches(recorder, name, args) == ([], 1)

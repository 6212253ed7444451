"""Which kernel converts to 8 bits and how many tiles a call may have: no launch reaches 2^32 threads (the rule of tac_quantize_plan.h, compiled into
a library of its own), and the entry point refuses what is beyond."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_13810_amd import api, build

HERE = os.path.dirname(os.path.abspath(__file__))
P = 1 << 20                                  # an address that is never read: nothing is launched


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "quantize_plan.so")
    subprocess.check_call([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++20", "-fPIC", "-shared", "-x", "hip", "-I",
                           build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "quantize_plan_shim.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    L.quantize_rows_alone.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong]
    L.quantize_most_tiles.restype = ctypes.c_longlong
    return L


@pytest.mark.parametrize("columns", [0, 1])
@pytest.mark.parametrize("tiles", [0, 1])
def test_no_launch_reaches_2_to_the_32_threads(shim, columns, tiles):
    most = shim.quantize_most_tiles()
    for count in (1, 1000, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, most - 1):
        alone = shim.quantize_rows_alone(columns, tiles, count)
        assert count * (512 if alone else 256) < 1 << 32
        assert bool(alone) == (not columns and not tiles and count < 1 << 23)


@pytest.mark.parametrize("rows,cols", [(1, 128 << 24), (128 << 12, 128 << 12), (1 << 31, 1)])
def test_more_tiles_than_a_launch_holds_are_refused(shim, rows, cols):
    assert shim.quantize_most_tiles() == 1 << 24 <= -(-rows // 128) * -(-cols // 128)
    d = api.tac_quantize_desc_t(rows, cols, cols, api.TAC_BF16, api.TAC_BLOCK_ROW)
    assert api.lib().tac_quantize(ctypes.byref(d), P, None, P, P, None, None, None) == api.TAC_ERR_BAD_SHAPE

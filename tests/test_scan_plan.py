"""The waves of a workgroup of the gated recurrence: no launch reaches 2^32 threads (the rule of tac_scan_plan.h, compiled into a library of its own)."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_13810_amd import api, build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "scan_plan.so")
    subprocess.check_call([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++20", "-fPIC", "-shared", "-x", "hip", "-I",
                           build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "scan_plan_shim.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    L.scan_waves_of.argtypes = [ctypes.c_longlong] * 2
    return L


@pytest.mark.parametrize("T", [1, 16, 17, 32, 33, 100, 113, 128, 129, 5000])
def test_a_wave_a_chunk_and_no_more_than_a_launch_holds(shim, T):
    usual = min(8, -(-T // api.TAC_SCAN_CHUNK))
    # B sequences of D channels, one or two a lane: the most groups are 65535 sequences of 32769 channels, one a lane
    for B, D, per_lane in ((1, 1, 1), (16, 2048, 2), (128, 128, 1), (65535, 8192, 1), (65535, 32769, 1), (65535, 32768, 2), (1, (1 << 31) - 1, 1), (40000, 53687, 1)):
        groups = B * -(-D // (64 * per_lane))
        waves = shim.scan_waves_of(T, groups)
        assert 1 <= waves <= usual and 64 * waves * groups < 1 << 32
        assert waves == usual or 64 * (waves + 1) * groups >= 1 << 32

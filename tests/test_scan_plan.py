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


def touched(at, st, sb, T, B, D, el):
    return {at + el * (t * st + b * sb + d) + i for t in range(T) for b in range(B) for d in range(D) for i in range(el)}


def test_sequences_that_share_memory_are_seen(shim):
    shim.rows_overlap_of.argtypes = [ctypes.c_longlong] * 10
    import random
    r, apart, slices = random.Random(3), 0, 0
    for _ in range(4000):
        T, B, D, el = r.randint(1, 4), r.randint(1, 3), r.randint(1, 5), r.choice([2, 4])
        wide = D * r.randint(1, 4)
        layout = lambda: r.choice([(B * wide, wide), (wide, T * wide), (B * D, D), (D, T * D)])
        x, y = layout(), layout()
        if r.random() < 0.5:
            y = x
        at = 1000 * el
        other = at + el * r.choice([0, D, -D, 2 * D, r.randint(-60, 60), r.randint(-300, 300)])
        share = bool(touched(at, *x, T, B, D, el) & touched(other, *y, T, B, D, el))
        seen = bool(shim.rows_overlap_of(at, *x, other, *y, T, B, D, el))
        assert seen or not share                         # never missed
        apart += not seen
        slices += not seen and x == y and 0 < abs(other - at) < (T - 1) * x[0] * el
    assert apart > 500 and slices > 100                  # and slices of the same rows are not taken for shared
    assert not shim.rows_overlap_of(0, 512, 256, 2 * 128, 512, 256, 100, 2, 128, 2)          # halves of rows, bfloat16

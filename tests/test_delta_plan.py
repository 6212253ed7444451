"""The host rules of the head norm and the gated delta rule (tac_delta_plan.h, compiled into a library of its own): what a launch holds, and that everything is taken."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_13810_amd import api, build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "delta_plan.so")
    subprocess.check_call([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++20", "-fPIC", "-shared", "-x", "hip", "-I",
                           build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "delta_plan_shim.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    L.head_slices_of.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    L.head_groups_of.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    L.head_groups_of.restype = ctypes.c_longlong
    L.delta_fits_of.argtypes = [ctypes.c_longlong] * 4
    L.delta_narrow_of.argtypes = [ctypes.c_longlong] * 3
    return L


@pytest.mark.parametrize("D", [2, 4, 6, 16, 62, 64, 66, 126, 128, 130, 250, 256, 258, 508, 510, 512])
def test_a_heads_lanes_hold_its_pairs(shim, D):
    for rotated in range(D // 2 + 1):
        lanes, apart = shim.head_lanes_of(D, rotated), shim.head_apart_of(D, rotated)
        assert lanes in (8, 16, 32, 64)
        if apart:                                    # pairs of both kinds on lanes of their own
            assert -(-rotated // 4) + -(-(D // 2 - rotated) // 4) <= lanes
        else:
            assert 4 * lanes >= D // 2
        assert apart or D > 500


def test_slices_and_groups_of_heads(shim):
    for lanes in (8, 16, 32, 64):
        for heads in (1, 2, 3, 24, 65535):
            for rows in (1, 2, 16, 1000, 16384, 1 << 20, (1 << 31) - 1):
                slices = shim.head_slices_of(rows, heads, lanes)
                assert 1 <= slices <= heads
                units = rows * slices
                for backward in (0, 1):
                    groups = shim.head_groups_of(rows, slices, lanes, backward)
                    assert 1 <= groups and groups * 256 < 1 << 32
                    # a lane's counter of units, one step behind the last one too, fits 32 bits
                    assert units + groups * (256 // lanes) < 1 << 32


def test_no_launch_of_the_delta_rule_reaches_2_to_the_32_threads(shim):
    taken = refused = 0
    for B in (1, 3, 1000, 65535, (1 << 31) - 1):
        for heads in (1, 16, 300):
            for Dv in (1, 16, 17, 128, 4096):
                for T in (1, 64, 65, 100_000, (1 << 31) - 1):
                    most = max(-(-T // 64), -(-Dv // 16)) * B * heads
                    fits = bool(shim.delta_fits_of(T, B, heads, Dv))
                    assert fits == (most * 512 < (1 << 32) - 512 or most == (1 << 23) - 1)
                    taken, refused = taken + fits, refused + (not fits)
    assert taken > 50 and refused > 50


def test_narrow_tiles_where_wide_ones_leave_compute_units_without_work(shim):
    assert shim.delta_narrow_of(1, 16, 128) and not shim.delta_narrow_of(8, 16, 128)
    assert shim.delta_narrow_of(10_000, 16, 16)

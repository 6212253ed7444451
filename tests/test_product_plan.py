"""Which tile and how many parts a product of 8-bit matrices takes: the host rules of tac_product_plan.h, compiled into a library of
their own (product_plan_shim.cpp)."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2603_13810_amd import api, build
from test_gpu_product_tiles import CASES

HERE = os.path.dirname(os.path.abspath(__file__))
STAGES = {0: (8, 2), 1: (4, 4), 2: (4, 2), 3: (4, 2), 4: (2, 2), 5: (2, 4), 6: (4, 4), 7: (4, 2), 8: (2, 8)}       # waves and stages of a tile


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "product_plan.so")
    subprocess.check_call([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++20", "-fPIC", "-shared", "-x", "hip", "-I",
                           build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "product_plan_shim.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    L.product_plan_of.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int, ctypes.c_void_p]
    return L


def plan(shim, M, N, K, bf16):
    out = (ctypes.c_int * 2)()
    shim.product_plan_of(M, N, K, bf16, ctypes.addressof(out))
    return tuple(out)


def tile(shim, t, bf16):
    out = (ctypes.c_int * 3)()
    used = shim.product_tile_of(t, bf16, out)
    return None if used < 0 else (bool(used), *out)


@pytest.mark.parametrize("bf16,t,M,N,K,parts,rounds", CASES)
def test_case_takes_the_tile_it_is_there_for(shim, bf16, t, M, N, K, parts, rounds):
    assert plan(shim, M, N, K, bf16) == (t, parts)
    used, rows, cols, shared = tile(shim, t, bf16)
    items = -(-M // rows) * -(-N // cols) * parts
    assert used and (-(-items // (256 * shared)) > 1) == rounds


def test_every_tile_of_a_type_has_a_case(shim):
    t = 0
    while tile(shim, t, 0) is not None:
        for bf16 in (0, 1):
            assert tile(shim, t, bf16)[0] == any(c[:2] == (bf16, t) for c in CASES)
        t += 1
    assert t == len(STAGES)


def test_workgroups_that_share_a_unit_fit_its_lds(shim):
    for t, (waves, stages) in STAGES.items():
        _, rows, cols, shared = tile(shim, t, 0)
        lds = shim.product_tile_lds(rows, cols, waves, stages)
        assert 160 * 1024 // lds == shared


def test_plans_of_any_size(shim):
    r = random.Random(5)
    for _ in range(3000):
        M, N, K = (int(2 ** r.uniform(0, 17)) for _ in range(3))
        bf16 = r.randint(0, 1)
        t, parts = plan(shim, M, N, K, bf16)
        assert tile(shim, t, bf16)[0] and 1 <= parts <= 32 and (parts == 1 or 2 * parts <= -(-K // 128))
        d = api.tac_product_desc_t(M, N, K, N, bf16)
        bytes_ = api.lib().tac_scaled_product_workspace_bytes(ctypes.byref(d))
        assert bytes_ == (4 * parts * M * N if parts > 1 else 0)

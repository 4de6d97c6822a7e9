"""Calls for branches of one context where they can go wrong, without a GPU."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2607_00151_amd as sa
from test_branches_cpu import CTX, NULL, OK, ROOT, SHAPE, UNSUPPORTED, i32, layout, lib, rope  # noqa: F401
from test_gpu_branch_edges import ANCHORED, PATHS, plan_of
from test_gpu_branches import SHARED, anchor


@pytest.mark.parametrize("want,eps", [(CTX, 1.2e-38), (CTX, 1e-6), (SHAPE, 1.1e-38), (SHAPE, 1e-45), (SHAPE, -1e-6)])
def test_rope_refuses_an_eps_that_the_norm_takes_for_zero(lib, want, eps):  # noqa: F811
    assert rope(lib, eps=eps) == want, lib.sa_last_error()


def test_the_gpu_tests_reach_the_paths_they_are_for():
    """Which prefixes the planner computes once in the batches of the GPU tests: a cost rule that moves shows here."""
    for heads, page, groups, once in PATHS:
        plan = plan_of(heads, page, groups)
        assert plan["once"] == [bool(x) for x in once], (heads, groups, plan)
        assert any(once) == (plan["items"] > 0)
    for (heads, page, groups), once in zip(SHARED, ANCHORED, strict=True):
        plan = plan_of(heads, page, [anchor(heads)] + groups)
        assert plan["once"] == [True] + [bool(x) for x in once], (heads, groups, plan)


def test_plan_stats_refusals(lib):  # noqa: F811
    def go(L=layout(), q=(1, 1), kv=(10, 9), groups=(0, 2), shared=(8,), cus=256, out=True):
        a, b, g, s, o = i32(q), i32(kv), i32(groups), i32(shared), np.zeros(4, np.int64)
        return lib.sa_shared_plan_stats(ctypes.byref(L), len(a), a.ctypes.data, b.ctypes.data, len(s), g.ctypes.data,
                                        s.ctypes.data, cus, o.ctypes.data if out else None, None)
    assert go() == OK
    assert go(out=False) == NULL and go(cus=0) == SHAPE and go(shared=[9]) == SHAPE and go(groups=[0, 1]) == SHAPE
    assert go(q=[11, 1]) == SHAPE and go(L=layout(head_dim=64)) == UNSUPPORTED
    with pytest.raises(ValueError, match="one entry more"):
        sa.sa_shared_plan_stats(layout(), [1], [4], [0, 1], [0, 0])


@pytest.mark.parametrize("value", [np.float32([1, 0.5, 0.25] * 8), [1.0] * 16, np.arange(32.0)[::2], np.float32(1)])
def test_rope_frequencies_may_be_set_from_any_array(value):
    rope = sa.Rope(np.ones(64))
    rope.inv_freq = value
    s, want = rope._struct(128, None), np.float64(value).reshape(-1)
    assert s.rot_dim == 2 * len(want)
    np.testing.assert_array_equal((ctypes.c_double * len(want)).from_address(s.h_inv_freq), want)


@pytest.mark.timeout(300)
def test_debug_check_of_shared_prefixes_under_asan_ubsan(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "shared_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-Wall", "-Werror",
                           "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2607_00151_amd", "csrc"),
                           os.path.join(ROOT, "tests", "host", "shared_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=240)
    print(r.stdout[-2000:], r.stderr[-4000:])
    assert r.returncode == 0 and "ALL OK" in r.stdout

"""Calls for branches of one context: host planning under sanitizers and refusals, without a GPU."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2607_00151_amd as sa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000   # aligned non-null stand-in device address; never dereferenced


@pytest.mark.timeout(300)
def test_branch_plans_under_asan_ubsan(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "branch_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-Wall", "-Werror",
                           "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2607_00151_amd", "csrc"),
                           os.path.join(ROOT, "tests", "host", "branch_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=240)
    print(r.stdout[-2000:], r.stderr[-4000:])
    assert r.returncode == 0 and "ALL OK" in r.stdout


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sa.library_path()):
        from paper_2607_00151_amd import build
        build.build()
    return sa.load_library()


def layout(**kw):
    d = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_layers=2, num_slots=64)
    d.update(kw)
    return sa.Layout(**d)


def i32(x):
    return np.asarray(x, dtype=np.int32)


OK, NULL, SHAPE, UNSUPPORTED, ALIGN, RANGE, NO_PAGES = 0, 1, 2, 3, 4, 5, 6
CTX = NULL        # every argument good: the NULL context is refused last


def rope(lib, L=None, freq=None, rot=128, eps=1e-6, w=FAKE, off=0.0, interleaved=0, layer=0, q=FAKE, qs=1024, ks=256,
         vs=256, k=FAKE, q_out=FAKE, pool=FAKE, start=(3,), new=(2,), pos=None, table=FAKE, no_struct=False):
    L = L or layout()
    freq = np.ones(64) if freq is None else np.asarray(freq, dtype=np.float64)
    r = sa._Rope(rot, interleaved, freq.ctypes.data if freq.size else None, w, w, eps, off)
    st, nl = i32(start), i32(new)
    ps = None if pos is None else i32(pos)
    return lib.sa_kv_append_rope(None, ctypes.byref(L), layer, None if no_struct else ctypes.byref(r), q, qs, k, ks,
                                 FAKE, vs, q_out, pool, FAKE, len(st), st.ctypes.data, nl.ctypes.data,
                                 None if ps is None else ps.ctypes.data, sa._Pages(table, FAKE), None)


@pytest.mark.parametrize("want,kw", [
    (CTX, {}), (CTX, dict(rot=0, freq=[])), (CTX, dict(w=None, eps=0.0)), (CTX, dict(interleaved=1)),
    (CTX, dict(pos=[2**31 - 3])), (CTX, dict(new=[0], q=None, k=None, q_out=None)), (CTX, dict(qs=1536)),
    (UNSUPPORTED, dict(L=layout(head_dim=64))), (UNSUPPORTED, dict(rot=24)), (UNSUPPORTED, dict(rot=144)),
    (UNSUPPORTED, dict(rot=-16)), (UNSUPPORTED, dict(L=layout(num_q_heads=65536, num_kv_heads=1), qs=65536 * 128)), (NULL, dict(no_struct=True)), (NULL, dict(freq=[])), (SHAPE, dict(eps=0.0)),
    (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(off=float("inf"))), (SHAPE, dict(freq=[-1.0] + [1.0] * 63)),
    (SHAPE, dict(freq=[float("nan")] * 64)), (SHAPE, dict(freq=[2000.0] * 64)), (SHAPE, dict(qs=1016)),
    (SHAPE, dict(ks=128)), (SHAPE, dict(vs=0)), (SHAPE, dict(qs=1 << 40)), (ALIGN, dict(qs=1028)), (SHAPE, dict(layer=2)),
    (SHAPE, dict(start=[-1])), (SHAPE, dict(new=[-1])), (SHAPE, dict(start=[2**31 - 1], new=[1])),
    (SHAPE, dict(pos=[-1])), (SHAPE, dict(pos=[2**31 - 2])), (NULL, dict(q=None)), (NULL, dict(q_out=None)),
    (NULL, dict(pool=None)), (NULL, dict(table=None)), (ALIGN, dict(q=FAKE + 8)), (ALIGN, dict(w=FAKE + 2)),
    (ALIGN, dict(pool=FAKE + 4)),
])
def test_rope_refusals(lib, want, kw):
    assert rope(lib, **kw) == want, lib.sa_last_error()


def test_rope_reaches_the_context_last(lib):
    assert rope(lib) == NULL and b"context" in lib.sa_last_error()


def fork(lib, L=None, src=(20,), parent=(0, 0), reserve=(4, 16), nfresh=8, cap=8, pool=FAKE, fresh=FAKE, dst=FAKE,
         used=True, table=FAKE):
    L = L or layout()
    s, p, r, u = i32(src), i32(parent), i32(reserve), np.zeros(1, np.int32)
    return lib.sa_kv_fork(None, ctypes.byref(L), pool, FAKE, len(s), s.ctypes.data, len(p), p.ctypes.data,
                          r.ctypes.data, sa._Pages(FAKE, table), fresh, nfresh, dst, FAKE, cap, None,
                          u.ctypes.data if used else None, None)


@pytest.mark.parametrize("want,kw", [
    (UNSUPPORTED, dict(L=layout(page_size=8))), (SHAPE, dict(src=[])), (SHAPE, dict(parent=[], reserve=[])),
    (SHAPE, dict(src=[-1])), (RANGE, dict(parent=[0, 1])), (RANGE, dict(parent=[-1, 0])), (SHAPE, dict(reserve=[4, -1])),
    (SHAPE, dict(nfresh=-1)), (NO_PAGES, dict(nfresh=2)), (NO_PAGES, dict(cap=4)), (NULL, dict(pool=None)),
    (NULL, dict(fresh=None)), (NULL, dict(dst=None)), (NULL, dict(used=False)), (NULL, dict(table=None)),
    (ALIGN, dict(pool=FAKE + 8)),
])
def test_fork_refusals(lib, want, kw):
    assert fork(lib, **kw) == want, lib.sa_last_error()


def test_fork_reaches_the_context_last(lib):
    assert fork(lib) == NULL and b"context" in lib.sa_last_error()


def test_count_refusals(lib):
    L, P = layout(), sa._Pages(FAKE, FAKE)
    assert lib.sa_kv_retain(None, ctypes.byref(L), 1, P, 4, FAKE, None) == NULL and b"context" in lib.sa_last_error()
    assert lib.sa_kv_retain(None, ctypes.byref(L), 0, P, 4, FAKE, None) == SHAPE
    assert lib.sa_kv_retain(None, ctypes.byref(L), 1, P, -1, FAKE, None) == SHAPE
    assert lib.sa_kv_retain(None, ctypes.byref(L), 1, P, 4, None, None) == NULL and b"d_ref" in lib.sa_last_error()
    assert lib.sa_kv_release(None, ctypes.byref(L), 1, P, 4, FAKE, FAKE, None, None) == NULL
    assert b"d_num_free" in lib.sa_last_error()
    assert lib.sa_kv_release(None, ctypes.byref(L), 1, P, 4, FAKE, None, None, None) == NULL
    assert b"context" in lib.sa_last_error()
    bad = layout(num_slots=0)
    assert lib.sa_kv_release(None, ctypes.byref(bad), 1, P, 4, FAKE, FAKE, FAKE, None) == SHAPE


def test_compact_refusals(lib):
    def go(L=layout(), limit=8, pool=FAKE, ref=FAKE, entries=4, ix=FAKE, moved=FAKE):
        return lib.sa_kv_compact(None, ctypes.byref(L), pool, FAKE, limit, ref, FAKE, ix, FAKE, entries, FAKE, moved, None)
    assert go() == NULL and b"context" in lib.sa_last_error()
    assert go(limit=-1) == RANGE and go(limit=65) == RANGE
    assert go(entries=-1) == SHAPE
    assert go(pool=None) == NULL and go(ref=None) == NULL and go(ix=None) == NULL and go(moved=None) == NULL
    assert go(entries=0, ix=None) == NULL and b"context" in lib.sa_last_error()
    assert go(pool=FAKE + 2) == ALIGN
    assert go(L=layout(head_dim=96)) == UNSUPPORTED


def test_sizes_beyond_32_bits_are_refused(lib):
    wide, deep = layout(num_q_heads=1 << 20, num_kv_heads=1 << 20, num_slots=1), layout(num_slots=2**31 - 1, num_layers=1)
    assert fork(lib, L=wide) == UNSUPPORTED and fork(lib, L=deep) == UNSUPPORTED
    assert rope(lib, L=wide) == UNSUPPORTED
    P = sa._Pages(FAKE, FAKE)
    for L in (wide, deep):
        assert lib.sa_kv_release(None, ctypes.byref(L), 1, P, 4, FAKE, FAKE, FAKE, None) == UNSUPPORTED
        assert lib.sa_kv_compact(None, ctypes.byref(L), FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE,
                                 None) == UNSUPPORTED
    # a destination table past 2^31 entries
    assert fork(lib, src=[2**31 - 1] * 20, parent=range(20), reserve=[0] * 20, nfresh=2**31 - 1, cap=2**31 - 1) == SHAPE


def test_shared_refusals(lib):
    def go(L=layout(), q_len=(1, 1), kv=(10, 9), groups=(0, 2), shared=(8,), q=FAKE, o=FAKE, lse=None, scale=0.1, layer=0):
        a, b, g, s = i32(q_len), i32(kv), i32(groups), i32(shared)
        return lib.sa_shared_prefix_attn(None, ctypes.byref(L), layer, q, FAKE, FAKE, len(a), a.ctypes.data,
                                         b.ctypes.data, sa._Pages(FAKE, FAKE), len(s), g.ctypes.data, s.ctypes.data,
                                         scale, o, lse, None)
    assert go() == NULL and b"context" in lib.sa_last_error()
    assert go(shared=[9]) == SHAPE and go(shared=[-1]) == SHAPE
    assert go(groups=[0, 1]) == SHAPE and go(groups=[1, 2]) == SHAPE and go(groups=[0, 3, 2], shared=[0, 0]) == SHAPE
    assert go(q_len=[10, 1]) == SHAPE            # the whole context is new: nothing is shared
    assert go(q_len=[11, 1]) == SHAPE and go(layer=2) == SHAPE and go(scale=0.0) == SHAPE
    assert go(o=None) == NULL and go(q=FAKE + 8) == ALIGN and go(lse=FAKE + 2) == ALIGN
    assert go(L=layout(page_size=64)) == UNSUPPORTED
    assert go(q_len=[0, 0], q=None, o=None) == NULL and b"context" in lib.sa_last_error()


def test_binding_refuses_what_the_library_would_misread():
    import torch
    L = layout()
    pool = torch.zeros((2, 64, 2, 16, 128), dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        sa.sa_kv_fork(None, L, pool, pool, [4], [0], [1], t, t, t, t, t)
    with pytest.raises(ValueError, match="differ in length"):
        sa.sa_kv_fork(None, L, pool, pool, [4], [0, 0], [1], t, t, t, t, t)
    rows = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on a GPU"):
        sa.sa_kv_append_rope(None, L, 0, sa.Rope(), rows, rows, rows, rows, pool, pool, [0], [2], t, t)
    with pytest.raises(ValueError, match="differ in length"):
        sa.sa_kv_append_rope(None, L, 0, sa.Rope(), rows, rows, rows, rows, pool, pool, [0], [2], t, t, pos=[0, 1])
    with pytest.raises(ValueError, match="one entry more"):
        sa.sa_shared_prefix_attn(None, L, 0, rows, pool, pool, [1], [4], t, t, [0, 1], [0, 0], 0.1, rows)
    with pytest.raises(ValueError, match="not on a GPU"):
        sa.sa_kv_release(None, L, t, t, t)

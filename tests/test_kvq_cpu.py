"""A cache of 4 bits and rotations on several axes: refusals, host planning and the format's definition, without a GPU."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2607_00151_amd as sa
from kvq_reference import GRID, page_bytes, page_values, quantise
from test_branches_cpu import (ALIGN, CTX, FAKE, NULL, ROOT, SHAPE, UNSUPPORTED, i32, layout, lib)  # noqa: F401


@pytest.mark.timeout(300)
def test_plans_under_asan_ubsan(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "kvq_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-Wall", "-Werror",
                           "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2607_00151_amd", "csrc"),
                           os.path.join(ROOT, "tests", "host", "kvq_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=240)
    print(r.stdout[-2000:], r.stderr[-4000:])
    assert r.returncode == 0 and "ALL OK" in r.stdout


# ------------------------------------------------------------------------- rows

def axes_struct(n=3, axis=None, pos=FAKE, stride=8, rot=128):
    a = i32([0] * (rot // 2) if axis is None else axis)
    return sa._Axes(n, a.ctypes.data if a.size else None, pos, stride), a


def rows(lib, name="sa_kvq_append", L=None, layer=0, rot=128, freq=None, w=FAKE, eps=1e-6, rope=True, axes=None, q=FAKE,  # noqa: F811
         qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, q_out=FAKE, pool=FAKE, start=(3,), new=(2,), pos=None, table=FAKE):
    L = L or layout()
    freq = np.ones(64) if freq is None else np.asarray(freq, dtype=np.float64)
    r = sa._Rope(rot, 0, freq.ctypes.data if freq.size else None, w, w, eps, 0.0)
    st, nl = i32(start), i32(new)
    ps = None if pos is None else i32(pos)
    x, kept = (None, None) if axes is None else axes_struct(**axes)
    args = [None, ctypes.byref(L), layer, ctypes.byref(r) if rope else None, None if x is None else ctypes.byref(x), q, qs,
            k, ks, v, vs, q_out, pool, FAKE, len(st), st.ctypes.data, nl.ctypes.data]
    if name == "sa_kvq_append":
        args.append(None if ps is None else ps.ctypes.data)
    return getattr(lib, name)(*args, sa._Pages(table, FAKE), None)


BARE = dict(rope=False, q=None, q_out=None, qs=0)


@pytest.mark.parametrize("want,kw", [
    (CTX, {}), (CTX, BARE), (CTX, dict(q=None, q_out=None, qs=0)), (CTX, dict(pos=[7])), (CTX, dict(axes={})),
    (CTX, dict(rot=0, freq=[], axes=dict(rot=0))), (CTX, dict(new=[0], k=None, v=None)), (CTX, dict(axes=dict(stride=2))),
    (CTX, dict(axes=dict(n=8, axis=[7] * 64))), (CTX, dict(new=[0], axes=dict(pos=None, stride=0))),
    (SHAPE, dict(BARE, q=FAKE)), (SHAPE, dict(BARE, q_out=FAKE, qs=1024)), (SHAPE, dict(BARE, pos=[1])), (SHAPE, dict(BARE, axes={})),
    (SHAPE, dict(q=None)), (SHAPE, dict(q_out=None)), (SHAPE, dict(pos=[1], axes={})),
    (SHAPE, dict(axes=dict(n=0))), (SHAPE, dict(axes=dict(n=9))), (SHAPE, dict(axes=dict(axis=[3] * 64))),
    (SHAPE, dict(axes=dict(axis=[0] * 63 + [-1]))), (SHAPE, dict(axes=dict(stride=1))), (NULL, dict(axes=dict(pos=None))),
    (NULL, dict(axes=dict(rot=0))), (ALIGN, dict(axes=dict(pos=FAKE + 2))),
    (UNSUPPORTED, dict(L=layout(head_dim=64))), (UNSUPPORTED, dict(L=layout(page_size=64))), (UNSUPPORTED, dict(rot=24)),
    (UNSUPPORTED, dict(BARE, L=layout(num_kv_heads=65536, num_q_heads=65536), ks=65536 * 128, vs=65536 * 128)),
    (NULL, dict(freq=[])), (SHAPE, dict(eps=0.0)), (SHAPE, dict(freq=[2000.0] * 64)), (SHAPE, dict(qs=1016)),
    (SHAPE, dict(ks=128)), (SHAPE, dict(vs=0)), (ALIGN, dict(ks=260)), (SHAPE, dict(layer=2)), (SHAPE, dict(start=[-1])),
    (SHAPE, dict(new=[-1])), (SHAPE, dict(start=[2**31 - 1], new=[1])), (SHAPE, dict(pos=[-1])), (NULL, dict(k=None)),
    (NULL, dict(v=None)), (NULL, dict(pool=None)), (NULL, dict(table=None)), (ALIGN, dict(k=FAKE + 8)),
    (ALIGN, dict(pool=FAKE + 4)), (ALIGN, dict(w=FAKE + 2)),
])
def test_append_refusals(lib, want, kw):  # noqa: F811
    assert rows(lib, **kw) == want, lib.sa_last_error()


@pytest.mark.parametrize("want,kw", [
    (CTX, dict(axes={})), (NULL, dict()), (NULL, dict(axes={}, rope=False)), (NULL, dict(axes={}, q=None)),
    (NULL, dict(axes={}, q_out=None)), (SHAPE, dict(axes=dict(axis=[3] * 64))), (SHAPE, dict(axes=dict(stride=1))),
    (SHAPE, dict(axes=dict(n=0))), (NULL, dict(axes=dict(pos=None))), (ALIGN, dict(axes=dict(pos=FAKE + 1))),
    (SHAPE, dict(axes={}, qs=1016)), (SHAPE, dict(axes={}, layer=-1)),
])
def test_append_rope_axes_refusals(lib, want, kw):  # noqa: F811
    assert rows(lib, "sa_kv_append_rope_axes", **kw) == want, lib.sa_last_error()


# ------------------------------------------------------------------------- pages

def convert(lib, name, L=None, k=FAKE, v=FAKE, s=FAKE, n4=8, k4=FAKE, v4=FAKE, s4=FAKE, n=3):  # noqa: F811
    L = L or layout()
    if name == "sa_kvq_pack":
        return lib.sa_kvq_pack(None, ctypes.byref(L), k, v, s, n4, k4, v4, s4, n, None)
    return lib.sa_kvq_unpack(None, ctypes.byref(L), n4, k4, v4, s4, k, v, s, n, None)


@pytest.mark.parametrize("name", ["sa_kvq_pack", "sa_kvq_unpack"])
@pytest.mark.parametrize("want,kw", [
    (CTX, {}), (CTX, dict(n=0, s=None, s4=None)), (SHAPE, dict(n=-1)), (SHAPE, dict(n4=0)), (SHAPE, dict(n4=1 << 40)),
    (SHAPE, dict(n=1 << 23)), (SHAPE, dict(L=layout(num_layers=40000), n=1)), (NULL, dict(k=None)), (NULL, dict(v4=None)),
    (NULL, dict(s=None)), (NULL, dict(s4=None)), (ALIGN, dict(v=FAKE + 8)), (ALIGN, dict(k4=FAKE + 4)),
    (UNSUPPORTED, dict(L=layout(head_dim=96))),
])
def test_convert_refusals(lib, name, want, kw):  # noqa: F811
    assert convert(lib, name, **kw) == want, lib.sa_last_error()


# ------------------------------------------------------------------------- attention

def attn(lib, L=None, layer=0, q=FAKE, k4=FAKE, v4=FAKE, q_len=(2,), kv_len=(9,), table=FAKE, indices=FAKE, causal=1,  # noqa: F811
         scale=0.1, o=FAKE, lse=FAKE):
    L = L or layout()
    a, b = i32(q_len), i32(kv_len)
    return lib.sa_kvq_attn(None, ctypes.byref(L), layer, q, k4, v4, len(a), a.ctypes.data, b.ctypes.data,
                           sa._Pages(table, indices), causal, scale, o, lse, None)


@pytest.mark.parametrize("want,kw", [
    (CTX, {}), (CTX, dict(causal=0)), (CTX, dict(lse=None)), (CTX, dict(q_len=[9], kv_len=[9])), (CTX, dict(q_len=[0], q=None, o=None)),
    (CTX, dict(causal=0, kv_len=[0], indices=None)), (CTX, dict(causal=0, q_len=[30], kv_len=[9])),
    (CTX, dict(q_len=[0, 1], kv_len=[5, 0], causal=0, indices=None)), (CTX, dict(kv_len=[2**31 - 64])),
    (SHAPE, dict(q_len=[10], kv_len=[9])), (SHAPE, dict(q_len=[-1])), (SHAPE, dict(kv_len=[-1], q_len=[0], causal=0)),
    (SHAPE, dict(kv_len=[2**31 - 63])), (SHAPE, dict(q_len=[2**30], kv_len=[2**30])), (SHAPE, dict(q_len=[], kv_len=[])),
    (SHAPE, dict(layer=2)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=float("nan"))), (SHAPE, dict(scale=float("inf"))),
    (NULL, dict(q=None)), (NULL, dict(o=None)), (NULL, dict(k4=None)), (NULL, dict(v4=None)), (NULL, dict(table=None)),
    (NULL, dict(indices=None)), (ALIGN, dict(q=FAKE + 2)), (ALIGN, dict(k4=FAKE + 8)), (ALIGN, dict(lse=FAKE + 2)),
    (UNSUPPORTED, dict(L=layout(page_size=8))), (SHAPE, dict(L=layout(num_q_heads=7))),
])
def test_attention_refusals(lib, want, kw):  # noqa: F811
    assert attn(lib, **kw) == want, lib.sa_last_error()


# ------------------------------------------------------------------------- the definition itself

def test_the_format_by_hand():
    row = np.zeros(128)
    row[0], row[1], row[2], row[3] = 1.0, -0.75, 0.1, 3.4          # amax 3.4: exponent 1 (1.7), unit 2^-1
    row[32], row[33] = 3.5, 1.0                                    # 1.75 rounds up to 2: exponent 2, unit 1
    row[64] = np.inf
    c, s = quantise(row)
    assert s.tolist() == [126, 127, 255, 1]
    assert c[:4].tolist() == [4, 8 + 3, 0, 7] and c[32:34].tolist() == [6, 2] and (c[64:] == 0).all()
    v = page_values(page_bytes(row[None, None]), 1)[0, 0]
    assert v[:4].tolist() == [1.0, -0.75, 0.0, 3.0] and v[32:34].tolist() == [4.0, 1.0] and np.isnan(v[64:96]).all()


def test_the_format_keeps_what_it_can_hold_and_errs_by_little():
    r = np.random.default_rng(1)
    x = r.standard_normal((50, 16, 128))
    v = page_values(page_bytes(x), 16)
    np.testing.assert_array_equal(page_bytes(v), page_bytes(x))
    amax = np.abs(x).reshape(50, 16, 4, 32).max(-1)
    assert (np.abs(v - x).reshape(50, 16, 4, 32).max(-1) <= amax / 3.5 + 1e-12).all()     # half of the widest step, 2 of >= 3.5 .. 7
    assert set(np.unique(np.abs(quantise(x)[0] & 7))) == set(range(len(GRID)))

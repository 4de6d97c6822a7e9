"""Calls for branches of one context where they can go wrong: values that are not finite, the edges of the slot scans,
contexts after a failed call, groups that take every path of the shared-prefix attention's planner."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa
from test_gpu_branches import (D, FILL, anchor, bits, branch_batch, check_attention, close_bf16, compact_reference, dev,
                               fork_reference, lay, pool_bits, rope_reference, run_shared, tables)

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------------- values that are not finite

NONFINITE = [
    # heads, page, groups; with the anchor: the shared-prefix kernel, else the segment attention
    ((8, 2), 16, [(900, [(5, 1), (40, 1), (7, 1)])], True),              # one token each
    ((32, 8), 16, [(3009, [(30, 13)] * 9)], True),                       # tiles of many members' rows
    ((8, 2), 16, [(900, [(5, 1), (40, 1), (7, 1)])], False),
    ((8, 1), 16, [(9000, [(5, 1), (40, 1)])], False),                    # split by key range
    ((4, 1), 16, [(256, [(200, 150), (300, 200)])], False),
]


def nonfinite_batch(i):
    heads, page, groups, anchored = NONFINITE[i]
    r = np.random.default_rng(300 + i)
    return branch_batch(r, heads, page, groups + ([anchor(heads)] if anchored else []))


def same_bits(a, b):
    return (a.contiguous().view(torch.uint8) == b.contiguous().view(torch.uint8)).all().item()


@pytest.mark.parametrize("i", range(len(NONFINITE)))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_query_that_is_not_finite_stays_in_its_row(i, value):
    w = nonfinite_batch(i)
    ctx = sa.Context(0)
    o, lse = (x.clone() for x in run_shared(ctx, w))
    t, h = w["q_len"][0] + w["q_len"][1] - 1, w["heads"][0] - 1          # the second member's last row
    clean = w["q"].clone()
    w["q"][t, h, 17] = value                                             # scores of both infinities, or NaN
    o2, lse2 = run_shared(ctx, w)
    assert o2[t, h].isnan().all() and lse2[t, h].isnan()
    o2[t, h], lse2[t, h] = o[t, h], lse[t, h]
    check_attention(dict(w, q=clean), o2, lse2, D ** -0.5)                     # the rows beside it


@pytest.mark.parametrize("i", range(len(NONFINITE)))
def test_a_key_that_is_nan_reaches_the_rows_that_see_it(i):
    """A shared key: every member's rows of its KV head; the last key of a member: that member's last token."""
    w = nonfinite_batch(i)
    Hq, Hkv = w["heads"]
    G, page = Hq // Hkv, w["L"].page_size
    ctx = sa.Context(0)
    o, lse = (x.clone() for x in run_shared(ctx, w))
    ip, ix = w["indptr"].tolist(), w["indices"].tolist()
    pool = w["kp"].view(torch.bfloat16)
    n = w["groups"][1]                                                   # members of the first group
    last = sum(w["q_len"][:2]) - 1
    cases = [(ix[ip[0] + 3 * 16 // page], 5, range(sum(w["q_len"][:n]))),
             (ix[ip[1] + (w["kv_len"][1] - 1) // page], (w["kv_len"][1] - 1) % page, [last])]
    for slot, row, tokens in cases:
        keep = pool[0, slot, Hkv - 1, row].clone()
        pool[0, slot, Hkv - 1, row, 100] = float("nan")
        o2, lse2 = run_shared(ctx, w)
        pool[0, slot, Hkv - 1, row] = keep
        hit = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
        hit[list(tokens), (Hkv - 1) * G:] = True
        assert o2[hit].isnan().all() and lse2[hit].isnan().all()
        check_attention(w, torch.where(hit[..., None], o, o2), torch.where(hit, lse, lse2), D ** -0.5)


@pytest.mark.parametrize("i", range(len(NONFINITE)))
def test_a_value_that_is_not_finite_leaves_the_other_members_alone(i):
    w = nonfinite_batch(i)
    Hq, Hkv = w["heads"]
    G, page = Hq // Hkv, w["L"].page_size
    ctx = sa.Context(0)
    o, lse = (x.clone() for x in run_shared(ctx, w))
    ip, ix = w["indptr"].tolist(), w["indices"].tolist()
    at = w["kv_len"][1] - 1
    w["vp"].view(torch.bfloat16)[0, ix[ip[1] + at // page], 0, at % page, 9] = float("inf")
    o2, lse2 = run_shared(ctx, w)
    t0, t1 = w["q_len"][0], sum(w["q_len"][:2])
    assert not o2[t1 - 1, :G, 9].isfinite().any()
    hit = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    hit[t0:t1, :G, 9] = True                                             # the member's rows may see it, no other does
    assert same_bits(o[~hit], o2[~hit]) and same_bits(lse, lse2)


VARIANT = r"""
import sys
sys.path.insert(0, {root!r}); sys.path.insert(0, {tests!r})
import numpy as np, torch
import paper_2607_00151_amd as sa
from test_gpu_branches import (D, anchor, bits, branch_batch, check_attention, compact_reference, dev, lay, pool_bits,
                               run_shared)
for heads, groups in (((8, 1), [(9000, [(5, 1), (40, 1)])]), ((4, 1), [(256, [(200, 150)])])):
    w = branch_batch(np.random.default_rng(5), heads, 16, groups)
    w["q"][0, 3, 17] = float("nan")
    print("variant {variant}", groups, flush=True)
    o, lse = run_shared(sa.Context(0), w)
    assert o[0, 3].isnan().all() and lse[0, 3].isnan()
    assert o[0, :3].isfinite().all() and lse[0, :3].isfinite().all()
print("variant ok", flush=True)
"""


@pytest.mark.timeout(200)
@pytest.mark.parametrize("variant", [1, 2])
def test_other_attention_kernels_keep_nan_rows(variant):
    code = VARIANT.format(root=ROOT, tests=os.path.join(ROOT, "tests"), variant=variant)
    r = subprocess.run([sys.executable, "-u", "-c", code], env=dict(os.environ, SA_ATTN_VARIANT=str(variant)),
                       capture_output=True, text=True, timeout=150)
    print(r.stdout[-2000:], r.stderr[-3000:])
    assert r.returncode == 0 and "variant ok" in r.stdout


# ------------------------------------------------------------------------- contexts

def test_a_call_that_failed_is_not_blamed_on_the_next():
    """An allocation beyond the card's memory is refused; torch and later calls of the context go on."""
    w = branch_batch(np.random.default_rng(9), (8, 2), 16, [(300, [(9, 1)] * 3), anchor((8, 2))])
    ctx = sa.Context(0)
    want, _ = run_shared(ctx, w)
    with pytest.raises(sa.SaError, match="SA_ERR_HIP"):
        sa.sa_reserve(ctx, 0, 1 << 45)
    ref = torch.zeros(w["L"].num_slots, dtype=torch.int32, device="cuda")
    with pytest.raises(sa.SaError, match="SA_ERR_HIP"):
        sa.sa_reserve(ctx, 0, 1 << 45)
    sa.sa_kv_retain(ctx, w["L"], w["indptr"], w["indices"], ref)
    assert int(ref.sum()) == len(w["indices"])
    got, _ = run_shared(ctx, w)
    assert torch.equal(got, want)


def test_reserved_contexts_scan_slots_without_allocating():
    """After sa_reserve the first release and the first compaction of a pool can be captured; replays follow the counts."""
    slots, r = 9000, np.random.default_rng(10)
    L = lay((1, 1), 16, slots)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    ctx = sa.Context(0)
    sa.sa_reserve(ctx, 16 * slots + 8 * (slots // 4096 + 1))
    ref, ix, ip = dev(np.zeros(slots)), dev([3, 4500]), dev([0, 2])
    ref_out, ix_out, smap, free = (torch.zeros_like(x) for x in (ref, ix, ref, ref))
    mv, nfree = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sa.sa_kv_compact(ctx, L, kp, vp, 4200, ref, ref_out, ix, ix_out, smap, mv)
        sa.sa_kv_release(ctx, L, ip, ix_out, ref_out, free, nfree)
    for i in range(3):
        count = (r.random(slots) < 0.3 + 0.1 * i).astype(np.int64)
        count[[3, 4500]] = 1
        ref.copy_(dev(count))
        before = kp.cpu()
        g.replay()
        sa.sa_sync_check(ctx)
        hole, high = np.flatnonzero(count[:4200] == 0), 4200 + np.flatnonzero(count[4200:])
        n = min(len(hole), len(high))
        assert mv.tolist() == [n, len(high) - n]
        after = count.copy()
        after[hole[:n]], after[high[:n]] = 1, 0
        to = np.arange(slots)
        to[high[:n]] = hole[:n]
        np.testing.assert_array_equal(ix_out.cpu(), to[[3, 4500]])
        after[to[[3, 4500]]] = 0
        np.testing.assert_array_equal(ref_out.cpu(), after)
        np.testing.assert_array_equal(free.cpu()[:int(nfree)], np.flatnonzero(after == 0))
        assert torch.equal(kp.cpu()[:, hole[:n]], before[:, high[:n]])


def test_a_growing_pool_leaves_few_scan_buffers_behind():
    """40 compactions of 200K to 400K slots need up to 6.5 MB of scan room each, 196 MB if each growth kept its own."""
    top = 400000
    pool = torch.zeros((1, top, 1, 16, D), dtype=torch.bfloat16, device="cuda")
    ref, out, smap = (torch.zeros(top, dtype=torch.int32, device="cuda") for _ in range(3))
    mv = torch.zeros(2, dtype=torch.int32, device="cuda")
    ctx = sa.Context(0)
    sa.sa_kv_compact(ctx, lay((1, 1), 16, 1000), pool, pool, 500, ref, out, None, None, smap, mv)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for slots in range(200000, top, 5000):
        sa.sa_kv_compact(ctx, lay((1, 1), 16, slots), pool, pool, slots // 2, ref, out, None, None, smap, mv)
    sa.sa_sync_check(ctx)
    assert free - torch.cuda.mem_get_info()[0] < 32 << 20


def test_the_check_says_what_a_kernel_met():
    L, ctx = lay((2, 2), 16, 8), sa.Context(0)
    ref = torch.zeros(8, dtype=torch.int32, device="cuda")
    page, count = "an out-of-range page id or slot", "a slot's count that does not fit the tables"
    for slots, met in (([2], count), ([8], page), ([8, 2], f"{page} and {count}")):
        sa.sa_kv_release(ctx, L, dev([0, len(slots)]), dev(slots), ref)
        with pytest.raises(sa.SaError, match=rf"SA_ERR_RANGE: a kernel met {met} \(flags"):
            sa.sa_sync_check(ctx)
        sa.sa_sync_check(ctx)
    assert not ref.any()


# ------------------------------------------------------------------------- the edges of the slot scans

@pytest.mark.parametrize("slots,entries", [(4095, 0), (4096, 1), (4097, 3), (8192, 5000), (8193, 700), (4096, 1535),
                                           (4096, 1536), (4096, 1537), (4095, 4096), (4096, 4097), (4097, 1536),
                                           (70000, 30000), (1, 2), (513, 1536)])
def test_release_at_the_edges_of_the_scans(slots, entries):
    """Counts lowered and listed in one launch or several, chunks of 4096 slots: twice, the second one to nothing."""
    r = np.random.default_rng(slots + entries)
    L, ctx = lay((1, 1), 16, slots), sa.Context(0)
    table = r.integers(0, slots, entries)
    table[:entries // 2] = np.sort(table[:entries // 2])                 # neighbours and strangers
    count = 2 * np.bincount(table, minlength=slots) + (r.random(slots) < 0.2)
    ref, free = dev(count), torch.full((slots,), -7, dtype=torch.int32, device="cuda")
    nfree = torch.zeros(1, dtype=torch.int32, device="cuda")
    ip, ix = dev([0, entries // 3, entries]), dev(table)
    for _ in range(2):
        count = count - np.bincount(table, minlength=slots)
        sa.sa_kv_release(ctx, L, ip, ix, ref, free, nfree)
        sa.sa_sync_check(ctx)
        np.testing.assert_array_equal(ref.cpu(), count)
        idle = np.flatnonzero(count == 0)
        assert int(nfree) == len(idle)
        np.testing.assert_array_equal(free.cpu(), np.concatenate([idle, np.full(slots - len(idle), -1)]))


@pytest.mark.parametrize("slots,limit", [(4095, 2000), (4096, 4095), (4097, 4096), (4097, 1), (8192, 4096), (8193, 4097),
                                         (12289, 8192)])
def test_compaction_at_the_edges_of_the_scans(slots, limit):
    r = np.random.default_rng(slots + limit)
    L, ctx = lay((1, 1), 16, slots), sa.Context(0)
    count = (r.random(slots) < 0.6) * r.integers(1, 4, slots)
    table = np.repeat(np.arange(slots), count).astype(np.int32)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    to, after, wix, wk, moved = compact_reference(count, limit, table, bits(kp))
    ref, ix = dev(count), dev(table)
    smap, mv = torch.full_like(ref, -7), torch.full((2,), -7, dtype=torch.int32, device="cuda")
    sa.sa_kv_compact(ctx, L, kp, vp, limit, ref, ref, ix, ix, smap, mv)
    sa.sa_sync_check(ctx)
    assert mv.tolist() == moved
    for got, want in ((smap, to), (ref, after), (ix, wix)):
        np.testing.assert_array_equal(got.cpu(), want)
    np.testing.assert_array_equal(bits(kp), wk)


DEBUG = r"""
import sys
sys.path.insert(0, {root!r}); sys.path.insert(0, {tests!r})
import numpy as np, torch
import paper_2607_00151_amd as sa
from test_gpu_branches import D, anchor, branch_batch, check_attention, run_shared
w = branch_batch(np.random.default_rng(1), (8, 2), 16, [(203, [(9, 1), (30, 1), (12, 0), (40, 2)]), anchor((8, 2))], layers=2, layer=1)
ctx = sa.Context(0)
for _ in range(2):                                                 # the copied partial pages are equal
    check_attention(w, *run_shared(ctx, w), D ** -0.5)

def refused(w, status, text):
    try:
        run_shared(ctx, w)
    except sa.SaError as e:
        assert e.name == status and text in str(e), e
        return
    raise AssertionError("not refused: " + text)

g = w["shared"]
refused(dict(w, shared=[204] + g[1:]), "SA_ERR_SHAPE", "sequences 0 and 1 differ on page 12")    # one token too far
run_shared(ctx, dict(w, shared=[192] + g[1:]))
at = int(w["indptr"][1]) + 12
keep, n = int(w["indices"][at]), w["L"].num_slots
w["indices"][at] = n
refused(w, "SA_ERR_RANGE", "outside [0, %d)" % n)
w["indices"][at] = keep
bits = w["vp"][1, keep, 1, 10]
bits[127] ^= 1                                                    # the last shared row of a copy, one bit of one value
refused(w, "SA_ERR_SHAPE", "sequences 0 and 1 differ on page 12")
bits[127] ^= 1
w["vp"][1, keep, 1, 11, 127] ^= 1                                   # the row behind it is the member's own
run_shared(ctx, w)
print("debug shared checks ok", flush=True)
"""


@pytest.mark.timeout(200)
def test_debug_checks_of_shared_prefixes():
    code = DEBUG.format(root=ROOT, tests=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-u", "-c", code], env=dict(os.environ, SA_DEBUG="1"), capture_output=True,
                       text=True, timeout=150)
    print(r.stdout[-2000:], r.stderr[-3000:])
    assert r.returncode == 0 and "debug shared checks ok" in r.stdout


# ------------------------------------------------------------------------- the planner's paths

PATHS = [
    # heads, page, groups, which prefixes are computed once
    ((12, 2), 16, [(16001, [(100, 30 + i) for i in range(7)])], [1]),           # members of 180 to 216 rows
    ((32, 8), 16, [(9000, [(60, 33), (60, 47), (64, 64), (70, 40), (33, 33), (90, 50)] * 2)], [1]),
    ((64, 8), 32, [(20000, [(40 + i, 1) for i in range(40)])], [1]),
    ((64, 8), 32, [(9001, [(40 + i, 1) for i in range(40)])], [1]),
    ((32, 4), 32, [(11000, [(20 + 13 * i, 1) for i in range(16)])], [1]),
    ((24, 8), 16, [(9001, [(300 + i, 7 + 5 * i) for i in range(10)])], [1]),
    ((24, 8), 16, [(9001, [(30 + i, 14) for i in range(10)]), (5000, [(40, 17)] * 8)], [1, 1]),
    ((32, 8), 16, [(5510, [(125, 9 + i) for i in range(9)]), (12000, [(125, 16 - i) for i in range(12)])], [1, 1]),
    ((16, 2), 16, [(12005, [(70, 1)] * 33), (300, [(10, 2), (9, 0), (70, 3)])], [1, 1]),
    ((32, 8), 16, [(6000, [(60, 48), (60, 0), (33, 33), (64, 40)] * 3), (500, [(9, 1), (40, 1)])], [1, 1]),
    ((16, 2), 16, [(30005, [(70, 25 + 3 * i) for i in range(9)])], [0]),
    ((32, 8), 16, [(6000, [(30, 1)] * 20), (100, [(30, 4)] * 3)], [1, 1]),
]
# (heads, page, groups) of SHARED behind the anchor: which groups' prefixes are computed once
ANCHORED = [[1], [1], [0, 1, 0], [1], [1], [1], [1], [0], [1], [0, 0, 1, 0], [0], [1, 1, 0], [1], [0, 1, 0, 0], [1, 0],
            [0], [0]]


def plan_of(heads, page, groups, num_cu=256):
    members = [m for _, ms in groups for m in ms]
    q, own = [q for _, q in members], [x for x, _ in members]
    s = [s for s, ms in groups for _ in ms]
    gp = np.concatenate([[0], np.cumsum([len(ms) for _, ms in groups])])
    return sa.sa_shared_plan_stats(lay(heads, page, 1 << 20), q, np.add(s, own), gp, [s for s, _ in groups], num_cu)


@pytest.mark.parametrize("i", range(len(PATHS)))
def test_shared_prefix_attention_on_every_path(i):
    """Members of several row tiles, tiles of many members, one to two prefix parts per CU and fewer, against float64;
    and beside the segment attention over the same tables: each result is within its tolerance of the float64 one."""
    heads, page, groups, once = PATHS[i]
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert plan_of(heads, page, groups, cus)["once"] == [bool(x) for x in once]
    w = branch_batch(np.random.default_rng(400 + i), heads, page, groups)
    ctx = sa.Context(0)
    o, lse = run_shared(ctx, w)
    check_attention(w, o, lse, D ** -0.5)
    o2, lse2 = run_shared(ctx, w)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    sa.sa_segment_prefill_attn(ctx, w["L"], 0, w["q"].cuda(), w["kp"], w["vp"], w["q_len"], w["kv_len"], w["indptr"],
                               w["indices"], D ** -0.5, o2, lse2)
    sa.sa_sync_check(ctx)
    check_attention(w, o2, lse2, D ** -0.5)
    assert torch.equal(o, o2) == (not any(once))         # not any: the segment attention's own launch


@pytest.mark.parametrize("heads,q,anchored", [((4, 1), 150, False), ((32, 8), 64, True), ((8, 2), 150, True)])
def test_a_masked_value_that_is_not_finite_stays_in_its_work_item(heads, q, anchored):
    """The last token's value: the rows of the work items before its own are the same bits."""
    G, page = heads[0] // heads[1], 16
    groups = [(320, [(q + 7, q), (q, q)])] + ([anchor(heads)] if anchored else [])
    w = branch_batch(np.random.default_rng(q), heads, page, groups)
    ctx = sa.Context(0)
    o, lse = (x.clone() for x in run_shared(ctx, w))
    at = w["kv_len"][1] - 1
    slot = int(w["indices"][int(w["indptr"][1]) + at // page])
    w["vp"].view(torch.bfloat16)[0, slot, :, at % page, 64] = float("nan")
    o2, lse2 = run_shared(ctx, w)
    first = (q * G - 1) // 128 * 128                                     # packed row of the last work item
    whole = q + first // G                                               # tokens of the call that are before it
    assert first > 0 and o2[2 * q - 1, :, 64].isnan().all()
    assert same_bits(o[:whole], o2[:whole]) and same_bits(o[2 * q:], o2[2 * q:]) and same_bits(lse, lse2)


# ------------------------------------------------------------------------- large batches, odd heads, two streams

@pytest.mark.parametrize("heads,page,groups,once", [
    ((8, 2), 16, [(2005, [(1 + i % 40, 1) for i in range(700)])], [1]),            # a plan of 200 KB
    ((192, 1), 32, [(9000, [(5 + i, 1) for i in range(8)])], [1]),                 # a token in two row tiles
    ((130, 2), 16, [(9000, [(i + 1, 1) for i in range(20)])], [1]),                # 65 query heads to a key head
    ((1, 1), 16, [(30000, [(i + 3, 3) for i in range(40)])], [1]),
])
def test_shared_prefix_attention_of_many_members_and_odd_heads(heads, page, groups, once):
    assert plan_of(heads, page, groups)["once"] == [bool(x) for x in once]
    w = branch_batch(np.random.default_rng(len(groups[0][1])), heads, page, groups)
    check_attention(w, *run_shared(sa.Context(0), w), D ** -0.5)


def test_append_rope_of_thousands_of_sequences():
    """5000 sequences of none to two tokens: the token search takes three rounds."""
    r = np.random.default_rng(61)
    new, start = r.integers(0, 3, 5000), r.integers(0, 40, 5000)
    pages = -(-(start + new) // 16)
    T = int(new.sum())
    L = lay((2, 1), 16, int(pages.sum()) + 1)
    indptr, indices, _ = tables(r, pages, L.num_slots)
    both = (torch.randn((T, 4, D), device="cuda") * 0.5).to(torch.bfloat16)
    q, k, v = both.split([2, 1, 1], dim=1)
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    out, inv = torch.empty((T, 2, D), dtype=torch.bfloat16, device="cuda"), 10000.0 ** (-np.arange(64) / 64)
    ctx = sa.Context(0)
    sa.sa_kv_append_rope(ctx, L, 0, sa.Rope(inv), q, k, v, out, kp, vp, start, new, dev(indptr), dev(indices))
    sa.sa_sync_check(ctx)
    seq = np.repeat(np.arange(5000), new)
    at = np.repeat(start, new) + np.arange(T) - np.repeat(np.cumsum(new) - new, new)
    slot, row = indices[indptr[seq] + at // 16], at % 16
    want = torch.full_like(vp, np.uint16(FILL).view(np.int16))
    want[0, slot, 0, row] = v[:, 0].contiguous().view(torch.int16)
    assert torch.equal(vp, want)
    close_bf16(out, *rope_reference(q.cpu(), None, at, inv, 0, False, 0.0))
    close_bf16(kp.view(torch.bfloat16)[0, slot, 0, row][:, None], *rope_reference(k.cpu(), None, at, inv, 0, False, 0.0))


def test_fork_of_thousands_of_children():
    r = np.random.default_rng(62)
    src_len, page = [37, 16, 0, 5], 16
    parent, reserve = r.integers(0, 4, 4500), r.integers(0, 20, 4500)
    pages = [-(-n // page) for n in src_len]
    need = sum(-(-(src_len[b] + x) // page) - src_len[b] // page for b, x in zip(parent, reserve))
    L = lay((1, 1), page, sum(pages) + need)
    indptr, indices, fresh = tables(r, pages, L.num_slots)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    wip, wix, used, wk = fork_reference(bits(kp), indptr, indices, src_len, parent, reserve, fresh, page)
    ref, dip, dix = dev(np.zeros(L.num_slots)), dev(np.zeros(4501)), dev(np.zeros(len(wix)))
    ctx = sa.Context(0)
    sa.sa_kv_retain(ctx, L, dev(indptr), dev(indices), ref)
    assert sa.sa_kv_fork(ctx, L, kp, vp, src_len, parent, reserve, dev(indptr), dev(indices), dev(fresh), dip, dix,
                         ref=ref) == used == need
    sa.sa_sync_check(ctx)
    np.testing.assert_array_equal(dip.cpu(), wip)
    np.testing.assert_array_equal(dix.cpu(), wix)
    np.testing.assert_array_equal(bits(kp), wk)
    np.testing.assert_array_equal(ref.cpu(), np.bincount(np.concatenate([indices, wix]), minlength=L.num_slots))


def test_two_contexts_at_once_on_two_streams():
    """Attention and counts of two contexts overlap in time; each gives what it gives alone."""
    works = [branch_batch(np.random.default_rng(70 + i), (8, 2), 16, [(700 + i, [(9, 1)] * 6), anchor((8, 2))])
             for i in range(2)]
    ctxs, streams = [sa.Context(0) for _ in works], [torch.cuda.Stream() for _ in works]
    alone = [run_shared(sa.Context(0), w) for w in works]
    qs = [w["q"].cuda() for w in works]
    outs = [[torch.empty_like(alone[i][0]) for _ in range(8)] for i in range(2)]
    L, n = lay((1, 1), 16, 9000), 9000
    refs = [dev(np.arange(n) % 3) for _ in works]
    free, nfree = [dev(np.zeros(n)) for _ in works], [dev([0]) for _ in works]
    ip, ix = dev([0, 3000]), dev(np.arange(3000) * 3 + 1)                # every count of one
    torch.cuda.synchronize()
    for k in range(8):
        for i, w in enumerate(works):
            sa.sa_shared_prefix_attn(ctxs[i], w["L"], 0, qs[i], w["kp"], w["vp"], w["q_len"], w["kv_len"], w["indptr"],
                                     w["indices"], w["groups"], w["shared"], D ** -0.5, outs[i][k], stream=streams[i])
            sa.sa_kv_release(ctxs[i], L, ip, ix, refs[i], free[i], nfree[i], stream=streams[i])
            sa.sa_kv_retain(ctxs[i], L, ip, ix, refs[i], stream=streams[i])
    for i in range(2):
        sa.sa_sync_check(ctxs[i], streams[i])
        assert all(torch.equal(o, alone[i][0]) for o in outs[i])
        assert int(nfree[i]) == 6000 and torch.equal(refs[i], dev(np.arange(n) % 3))
        np.testing.assert_array_equal(free[i].cpu()[:6000], np.flatnonzero(np.arange(n) % 3 < 2))

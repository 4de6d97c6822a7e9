"""Calls for branches of one context on the GPU, against plain definitions in float64 and in numpy.

Tolerances.  A bf16 rounding is off by at most 2^-8 of the value.
* Attention: probabilities are rounded to bf16 once (2^-8 of sum p|v| / sum p = A), the same rounding of a row's
  largest keys goes into the denominator (2^-8 |o|) and the output is rounded (2^-8 |o|).  The fp32 sums over n keys
  and 128 dims add n 2^-23 A, and a score's error e moves its weight by 2 e at most: e = 128 2^-24 max_k sum|q k| scale.
* Rotation: one rounding of each output, 2^-8; fp32 norm and rotation are below 2^-16 of the pair's size.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
D = 128
FILL = 0x7FC1          # a bf16 NaN pattern: any stray read or write shows up


def lay(heads, page, slots, layers=1):
    return sa.Layout(num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=D, page_size=page, num_layers=layers,
                     num_slots=slots)


def rows(r, shape, std=0.5):
    return torch.from_numpy((r.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)


def pool_bits(r, L, fill=None):
    shape = (L.num_layers, L.num_slots, L.num_kv_heads, L.page_size, D)
    if fill is not None:
        return torch.full(shape, np.int16(np.uint16(fill).view(np.int16)), dtype=torch.int16, device="cuda")
    return torch.from_numpy(r.integers(0, 2**15, shape, dtype=np.int64).astype(np.int16)).cuda()


def dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def tables(r, pages, slots):
    """A table of so many pages per sequence on distinct shuffled slots, and the slots that are left."""
    perm = r.permutation(slots).astype(np.int32)
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    return indptr, perm[:indptr[-1]].copy(), perm[indptr[-1]:].copy()


def bits(t):
    return t.cpu().view(torch.int16).numpy()


# ------------------------------------------------------------------------- sa_kv_append_rope

def rope_reference(x, w, pos, inv_freq, eps, interleaved, offset):
    """float64 [T][heads][128] and the size of what each output was made from."""
    y = x.double().numpy()
    if w is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + np.float32(eps)) * (w.double().numpy() + offset)
    n = len(inv_freq)
    ang = np.asarray(pos, dtype=np.longdouble)[:, None] * np.asarray(inv_freq, dtype=np.longdouble)
    c, s = (f(ang).astype(np.float64)[:, None, :] for f in (np.cos, np.sin))
    i = np.arange(n) * 2 if interleaved else np.arange(n)
    j = i + 1 if interleaved else i + n
    out, size = y.copy(), np.abs(y)
    out[..., i] = y[..., i] * c - y[..., j] * s
    out[..., j] = y[..., j] * c + y[..., i] * s
    size[..., i] = size[..., j] = np.abs(y[..., i]) + np.abs(y[..., j])
    return out, size


def close_bf16(got, ref, size):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * size + 1e-30
    worst = np.max(np.abs(got - ref) / tol)
    assert worst <= 1.0, worst


ROPE = [
    # heads, page, start, new, rot, interleaved, norms, fused, far, offset
    ((32, 8), 16, [0], [1], 128, False, "qk", True, 0, 0.0),
    ((32, 8), 16, [15, 16, 0, 40, 7], [1, 17, 0, 33, 2], 128, False, "qk", True, 0, 0.0),
    ((8, 2), 16, [3], [65], 128, True, "", False, 0, 0.0),
    ((8, 2), 32, [31, 64], [2, 1], 64, False, "q", False, 5000, 1.0),
    ((24, 8), 16, [5, 0, 9], [0, 9, 0], 96, False, "k", True, 1 << 21, 0.0),
    ((7, 7), 32, [1], [40], 32, True, "qk", True, 2**31 - 100, -0.5),
    ((64, 8), 32, [100], [3], 16, False, "qk", False, 0, 0.0),
    ((1, 1), 16, [0, 1], [5, 6], 0, False, "qk", True, 0, 0.0),
    ((1, 1), 16, [2], [6], 0, True, "", False, 0, 0.0),
    ((16, 1), 16, list(range(70)), [1] * 70, 128, False, "qk", True, 0, 0.0),
    ((4, 2), 16, list(range(300)), [i % 3 for i in range(300)], 128, True, "qk", True, 77, 0.0),
]


@pytest.mark.parametrize("heads,page,start,new,rot,inter,norms,fused,far,offset", ROPE)
def test_append_rope(heads, page, start, new, rot, inter, norms, fused, far, offset):
    r = np.random.default_rng(len(start) * 1000 + rot)
    Hq, Hkv = heads
    T = sum(new)
    pages = [-(-(a + n) // page) for a, n in zip(start, new)]
    L = lay(heads, page, sum(pages) + 5, layers=2)
    indptr, indices, _ = tables(r, pages, L.num_slots)
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    both = rows(r, (T, Hq + 2 * Hkv, D))
    both[:, :, 3] *= 20                                   # an outlier dim, as projections have
    x = list(both.split([Hq, Hkv, Hkv], dim=1))
    on_gpu = list(both.cuda().split([Hq, Hkv, Hkv], dim=1))
    if not fused:
        on_gpu = [t.contiguous() for t in on_gpu]
    qw, kw = (1 + 0.3 * rows(r, (D,)).float()).to(torch.bfloat16), rows(r, (D,), 1.0)
    qw, kw = qw if "q" in norms else None, kw if "k" in norms else None
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    pos0 = [far + i for i in range(len(start))] if far else start
    ctx = sa.Context(0)
    rope = sa.Rope(inv, None if qw is None else qw.cuda(), None if kw is None else kw.cuda(), 1e-5, inter, offset)
    q_out = torch.full((T + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):                                    # the second call finds its plan on the device
        sa.sa_kv_append_rope(ctx, L, 1, rope, *on_gpu, q_out, kp, vp, start, new, dev(indptr), dev(indices),
                             pos=pos0 if far else None)
    sa.sa_sync_check(ctx)
    pos = np.concatenate([[p + t for t in range(n)] for p, n in zip(pos0, new)] or [[]])
    assert (q_out[T:] == 7).all()
    if T == 0:
        return
    close_bf16(q_out[:T], *rope_reference(x[0], qw, pos, inv, 1e-5, inter, offset))
    slot, row = [], []
    for b, (a, n) in enumerate(zip(start, new)):
        for t in range(a, a + n):
            slot.append(int(indices[indptr[b] + t // page]))
            row.append(t % page)
    got = kp.view(torch.bfloat16)[1].permute(0, 2, 1, 3)[slot, row]
    close_bf16(got, *rope_reference(x[1], kw, pos, inv, 1e-5, inter, offset))
    want = np.full(kp.shape, np.uint16(FILL).view(np.int16))
    want[1].transpose(0, 2, 1, 3)[slot, row] = bits(x[2].contiguous())
    np.testing.assert_array_equal(bits(vp), want)         # value rows bit for bit, the rest untouched
    keys = bits(kp).copy()
    keys[1].transpose(0, 2, 1, 3)[slot, row] = np.uint16(FILL).view(np.int16)
    assert (keys == np.uint16(FILL).view(np.int16)).all()


def test_append_rope_in_place_and_on_another_stream():
    r = np.random.default_rng(5)
    L = lay((8, 2), 16, 8)
    q, k, v = rows(r, (40, 8, D)).cuda(), rows(r, (40, 2, D)).cuda(), rows(r, (40, 2, D)).cuda()
    ip, ix = dev([0, 3]), dev([4, 0, 7])
    rope = sa.Rope(10000.0 ** (-np.arange(64) / 64), rows(r, (D,)).cuda(), None)
    ctx, outs = sa.Context(0), []
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    q_out = torch.empty_like(q)
    sa.sa_kv_append_rope(ctx, L, 0, rope, q, k, v, q_out, kp, vp, [2], [40], ip, ix)
    outs.append((bits(q_out).copy(), bits(kp).copy(), bits(vp).copy()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    kp2, vp2 = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    side.wait_stream(torch.cuda.current_stream())
    sa.sa_kv_append_rope(ctx, L, 0, rope, q, k, v, q, kp2, vp2, [2], [40], ip, ix, stream=side)
    side.synchronize()
    for a, b in zip(outs[0], (q, kp2, vp2)):
        np.testing.assert_array_equal(a, bits(b))


def test_append_rope_tells_batches_of_equal_words_apart():
    """One sequence and 64 frequencies, then 17 sequences and 40, whose arrays are the same words one after another."""
    r = np.random.default_rng(7)
    L, ctx = lay((4, 2), 16, 8), sa.Context(0)
    q, k = rows(r, (5, 4, D)).cuda(), rows(r, (5, 2, D)).cuda()
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    out = torch.empty_like(q)
    sa.sa_kv_append_rope(ctx, L, 0, sa.Rope(np.zeros(64)), q, k, k, out, kp, vp, [0], [5], dev([0, 1]), dev([3]))
    sa.sa_sync_check(ctx)
    before = bits(kp).copy()
    sa.sa_kv_append_rope(ctx, L, 0, sa.Rope(np.zeros(40)), None, None, None, None, kp, vp, [0, 5] + [0] * 15, [0] * 17,
                         dev([0] * 18), dev([3]))
    sa.sa_sync_check(ctx)
    np.testing.assert_array_equal(bits(kp), before)


@pytest.mark.parametrize("rot,inter", [(128, False), (64, False), (128, True)])
def test_append_rope_of_many_tokens(rot, inter):
    """More bytes than the Infinity Cache: checked against the same rows in pieces, and some rows in float64."""
    heads, page, T = (32, 8), 16, 14001
    L = lay(heads, page, -(-T // page) + 1)
    g = torch.Generator(device="cuda").manual_seed(3)
    both = (torch.randn((T, 48, D), generator=g, device="cuda") * 0.5).to(torch.bfloat16)
    q, k, v = both.split([32, 8, 8], dim=1)
    ip, ix = dev([0, L.num_slots]), dev(np.random.default_rng(3).permutation(L.num_slots))
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    w = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    rope, ctx = sa.Rope(inv, w, w, 1e-6, inter), sa.Context(0)
    pools = [pool_bits(None, L, FILL) for _ in range(4)]
    q_out, q2 = (torch.empty((T, 32, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sa.sa_kv_append_rope(ctx, L, 0, rope, q, k, v, q_out, pools[0], pools[1], [0], [T], ip, ix)
    for a in range(0, T, 3500):
        n = min(3500, T - a)
        sa.sa_kv_append_rope(ctx, L, 0, rope, q[a:], k[a:], v[a:], q2[a:], pools[2], pools[3], [a], [n], ip, ix)
    sa.sa_sync_check(ctx)
    assert torch.equal(q_out, q2) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    pick = [0, 1, 6999, T - 1]
    close_bf16(q_out[pick], *rope_reference(q[pick].cpu(), w.cpu(), pick, inv, 1e-6, inter, 0.0))


def test_append_rope_reports_bad_pages_and_writes_the_rest():
    r = np.random.default_rng(6)
    L = lay((4, 2), 16, 8)
    T = 3
    q, k, v = rows(r, (T, 4, D)).cuda(), rows(r, (T, 2, D)).cuda(), rows(r, (T, 2, D)).cuda()
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    q_out = torch.zeros_like(q)
    ctx = sa.Context(0)
    # sequence 0's page is beyond the pool, 1's is missing, 2's is slot 5
    sa.sa_kv_append_rope(ctx, L, 0, sa.Rope(), q, k, v, q_out, kp, vp, [0, 16, 1], [1, 1, 1], dev([0, 1, 2, 3]),
                         dev([8, 3, 5]))
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    assert torch.equal(q_out, q)
    want = np.full(vp.shape, np.uint16(FILL).view(np.int16))
    want[0, 5, :, 1] = bits(v)[2]
    np.testing.assert_array_equal(bits(vp), want)


# ------------------------------------------------------------------------- pages

def fork_reference(k, indptr, indices, src_len, parent, reserve, fresh, P):
    """(dst indptr, dst indices, fresh slots taken, pool after the copies)."""
    k, out, ip, used = k.copy(), [], [0], 0
    for b, res in zip(parent, reserve):
        n = src_len[b]
        pages = -(-(n + res) // P)
        mine = list(indices[indptr[b]:indptr[b] + n // P])
        take = list(fresh[used:used + pages - n // P])
        used += len(take)
        if n % P:
            k[:, take[0], :, :n % P] = k[:, indices[indptr[b] + n // P], :, :n % P]
        out += mine + take
        ip.append(len(out))
    return np.array(ip, np.int32), np.array(out, np.int32), used, k


FORK = [
    # heads, page, layers, src_len, parent, reserve
    ((8, 2), 16, 1, [1], [0], [0]),
    ((8, 2), 16, 3, [33], [0, 0, 0, 0], [1, 0, 15, 40]),
    ((8, 2), 32, 2, [64, 0, 95, 31], [2, 0, 1, 2, 0, 3, 1], [0, 0, 0, 33, 5, 1, 70]),
    ((32, 8), 16, 1, [500, 3, 77], [0, 1, 2] * 6, [9] * 18),
    ((3, 3), 32, 1, [4096], [0] * 40, list(range(40))),
    ((1, 1), 16, 1, [0], [0], [0]),
]


@pytest.mark.parametrize("heads,page,layers,src_len,parent,reserve", FORK)
def test_fork_and_release(heads, page, layers, src_len, parent, reserve):
    r = np.random.default_rng(len(parent))
    pages = [-(-n // page) for n in src_len]
    need = sum(-(-(src_len[b] + x) // page) - src_len[b] // page for b, x in zip(parent, reserve))
    L = lay(heads, page, sum(pages) + need + 3, layers)
    indptr, indices, fresh = tables(r, pages, L.num_slots)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    k0, v0 = bits(kp).copy(), bits(vp).copy()
    wip, wix, used, wk = fork_reference(k0, indptr, indices, src_len, parent, reserve, fresh, page)
    wv = fork_reference(v0, indptr, indices, src_len, parent, reserve, fresh, page)[3]
    ref = torch.zeros(L.num_slots, dtype=torch.int32, device="cuda")
    dip = torch.full((len(parent) + 1,), -7, dtype=torch.int32, device="cuda")
    dix = torch.full((len(wix) + 2,), -7, dtype=torch.int32, device="cuda")
    free = torch.full((L.num_slots,), -7, dtype=torch.int32, device="cuda")
    nfree = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    ctx = sa.Context(0)
    sip, six = dev(indptr), dev(indices)
    sa.sa_kv_retain(ctx, L, sip, six, ref)
    for _ in range(2):
        assert sa.sa_kv_fork(ctx, L, kp, vp, src_len, parent, reserve, sip, six, dev(fresh), dip, dix, ref=ref) == used
        sa.sa_sync_check(ctx)
        np.testing.assert_array_equal(dip.cpu(), wip)
        np.testing.assert_array_equal(dix.cpu(), np.concatenate([wix, [-7, -7]]))
        np.testing.assert_array_equal(bits(kp), wk)
        np.testing.assert_array_equal(bits(vp), wv)
        count = np.bincount(np.concatenate([indices, wix]), minlength=L.num_slots)
        np.testing.assert_array_equal(ref.cpu(), count)
        sa.sa_kv_release(ctx, L, dip, dix, ref, free, nfree)
        sa.sa_sync_check(ctx)
        np.testing.assert_array_equal(ref.cpu(), np.bincount(indices, minlength=L.num_slots))
        idle = np.flatnonzero(np.bincount(indices, minlength=L.num_slots) == 0)
        assert int(nfree) == len(idle)
        np.testing.assert_array_equal(free.cpu(), np.concatenate([idle, np.full(L.num_slots - len(idle), -1)]))


def test_fork_without_counts_and_with_bad_slots():
    r = np.random.default_rng(3)
    L = lay((2, 2), 16, 8)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    ctx = sa.Context(0)
    dip, dix = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    assert sa.sa_kv_fork(ctx, L, kp, vp, [17], [0], [20], dev([0, 2]), dev([1, 6]), dev([4, 5, 7]), dip, dix) == 2
    sa.sa_sync_check(ctx)
    np.testing.assert_array_equal(dix.cpu(), [1, 4, 5])
    before = bits(kp).copy()
    # a page beyond the pool, and a table that lacks the partial page
    sa.sa_kv_fork(ctx, L, kp, vp, [17], [0], [0], dev([0, 2]), dev([8, 9]), dev([4]), dip, dix)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    sa.sa_kv_fork(ctx, L, kp, vp, [17], [0], [0], dev([0, 1]), dev([1]), dev([4]), dip, dix)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    np.testing.assert_array_equal(bits(kp), before)
    # counts that do not fit: a fresh slot in use, a shared page without a count
    ref = dev([0, 1, 0, 0, 1, 0, 0, 0])
    sa.sa_kv_fork(ctx, L, kp, vp, [16], [0], [1], dev([0, 1]), dev([1]), dev([4]), dip, dix, ref=ref)
    with pytest.raises(sa.SaError, match="0x8"):
        sa.sa_sync_check(ctx)
    ref = dev([0] * 8)
    sa.sa_kv_fork(ctx, L, kp, vp, [16], [0], [0], dev([0, 1]), dev([1]), dev([4]), dip, dix, ref=ref)
    with pytest.raises(sa.SaError, match="0x8"):
        sa.sa_sync_check(ctx)


def test_release_twice_is_reported_and_leaves_no_negative_count():
    L = lay((2, 2), 16, 300)
    ctx = sa.Context(0)
    ref = torch.ones(300, dtype=torch.int32, device="cuda")
    free, nfree = torch.zeros(300, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ip, ix = dev([0, 3, 5]), dev([7, 7, 8, 299, 8])       # 7 and 8 twice
    sa.sa_kv_release(ctx, L, ip, ix, ref, free, nfree)
    with pytest.raises(sa.SaError, match="0x8"):
        sa.sa_sync_check(ctx)
    want = np.ones(300)
    want[[7, 8, 299]] = 0
    np.testing.assert_array_equal(ref.cpu(), want)
    assert int(nfree) == 3 and free[:4].tolist() == [7, 8, 299, -1]
    # tables that run past their entries, or name slots outside the pool
    sa.sa_kv_release(ctx, L, dev([0, 6]), ix, ref)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    sa.sa_kv_retain(ctx, L, dev([0, 2]), dev([-1, 300]), ref)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    np.testing.assert_array_equal(ref.cpu(), want)
    sa.sa_kv_retain(ctx, L, dev([1, 3]), ix, ref)         # entries 1 and 2
    sa.sa_sync_check(ctx)
    want[[7, 8]] = 1
    np.testing.assert_array_equal(ref.cpu(), want)


@pytest.mark.parametrize("slots", [1, 7, 2047, 2048, 2049, 30000, 300001])
def test_free_list_of_any_pool_size(slots):
    r = np.random.default_rng(slots)
    L = lay((1, 1), 16, slots)
    ctx = sa.Context(0)
    count = r.integers(0, 3, slots)
    ref, free = dev(count), torch.zeros(slots, dtype=torch.int32, device="cuda")
    nfree = torch.zeros(1, dtype=torch.int32, device="cuda")
    sa.sa_kv_release(ctx, L, dev([0, 0]), torch.zeros(0, dtype=torch.int32, device="cuda"), ref, free, nfree)
    sa.sa_sync_check(ctx)
    idle = np.flatnonzero(count == 0)
    assert int(nfree) == len(idle)
    np.testing.assert_array_equal(free.cpu(), np.concatenate([idle, np.full(slots - len(idle), -1)]))


def compact_reference(count, limit, table, k):
    hole = [s for s in range(limit) if count[s] == 0]
    high = [s for s in range(limit, len(count)) if count[s] > 0]
    n = min(len(hole), len(high))
    to = np.where(count > 0, np.arange(len(count)), -1)
    to[high[:n]] = hole[:n]
    after = count.copy()
    after[hole[:n]], after[high[:n]] = count[high[:n]], 0
    k = k.copy()
    k[:, hole[:n]] = k[:, high[:n]]
    return to, after, to[table], k, [n, len(high) - n]


@pytest.mark.parametrize("heads,page,layers,slots,limit,used,in_place", [
    ((2, 2), 16, 1, 10, 5, 0.5, False), ((8, 2), 32, 3, 301, 150, 0.4, True), ((8, 8), 16, 2, 301, 150, 0.9, False),
    ((4, 1), 16, 2, 2500, 2048, 0.3, True), ((4, 1), 16, 1, 5000, 700, 0.6, False), ((2, 1), 16, 1, 64, 0, 0.5, False),
    ((2, 1), 16, 1, 64, 64, 0.5, True), ((2, 1), 16, 1, 64, 32, 0.0, False), ((2, 1), 16, 1, 64, 32, 1.0, False),
    ((3, 3), 32, 1, 1, 0, 1.0, True),
])
def test_compact(heads, page, layers, slots, limit, used, in_place):
    r = np.random.default_rng(slots + limit)
    L = lay(heads, page, slots, layers)
    count = (r.random(slots) < used) * r.integers(1, 4, slots)
    table = np.repeat(np.arange(slots), count).astype(np.int32)
    r.shuffle(table)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    to, after, wix, wk, moved = compact_reference(count, limit, table, bits(kp))
    wv = compact_reference(count, limit, table, bits(vp))[3]
    ref, ix = dev(count), dev(table)
    ref_out = ref if in_place else torch.full_like(ref, -7)
    ix_out = ix if in_place else torch.full_like(ix, -7)
    smap, mv = torch.full_like(ref, -7), torch.full((2,), -7, dtype=torch.int32, device="cuda")
    ctx = sa.Context(0)
    sa.sa_kv_compact(ctx, L, kp, vp, limit, ref, ref_out, ix, ix_out, smap, mv)
    sa.sa_sync_check(ctx)
    assert mv.tolist() == moved
    np.testing.assert_array_equal(smap.cpu(), to)
    np.testing.assert_array_equal(ref_out.cpu(), after)
    np.testing.assert_array_equal(ix_out.cpu(), wix)
    np.testing.assert_array_equal(bits(kp), wk)
    np.testing.assert_array_equal(bits(vp), wv)


def test_compact_reports_tables_that_do_not_fit():
    L = lay((2, 2), 16, 8)
    r = np.random.default_rng(1)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    ref, smap = dev([1, 0, 0, 0, 0, 0, 1, 0]), torch.zeros(8, dtype=torch.int32, device="cuda")
    mv, out = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ctx = sa.Context(0)
    sa.sa_kv_compact(ctx, L, kp, vp, 4, ref, torch.zeros_like(ref), dev([0, 6, -1, 8]), out, smap, mv)
    with pytest.raises(sa.SaError, match="0x4"):
        sa.sa_sync_check(ctx)
    assert out.tolist() == [0, 1, -1, 8]
    sa.sa_kv_compact(ctx, L, kp, vp, 4, ref, torch.zeros_like(ref), dev([0, 6, 3, 7]), out, smap, mv)
    with pytest.raises(sa.SaError, match="0x8"):
        sa.sa_sync_check(ctx)
    assert out.tolist() == [0, 1, -1, -1]


def test_counts_and_compaction_replay_from_a_graph():
    r = np.random.default_rng(9)
    L = lay((4, 2), 16, 3000)
    count = (r.random(3000) < 0.4).astype(np.int64)
    table = np.flatnonzero(count).astype(np.int32)
    kp, vp = pool_bits(r, L), pool_bits(r, L)
    ref, ix, ip = dev(count), dev(table), dev([0, len(table)])
    ref_out, ix_out, smap = torch.zeros_like(ref), torch.zeros_like(ix), torch.zeros_like(ref)
    mv, free = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros_like(ref)
    nfree = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = sa.Context(0)

    def step():
        sa.sa_kv_compact(ctx, L, kp, vp, 2000, ref, ref_out, ix, ix_out, smap, mv)
        sa.sa_kv_retain(ctx, L, ip, ix_out, ref_out)
        sa.sa_kv_release(ctx, L, ip, ix_out, ref_out, free, nfree)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        count = (r.random(3000) < 0.2 + 0.1 * i).astype(np.int64)
        count[table] = 1
        ref.copy_(dev(count))
        kp.copy_(pool_bits(r, L))
        to, after, wix, wk, moved = compact_reference(count, 2000, table, bits(kp))
        g.replay()
        sa.sa_sync_check(ctx)
        assert mv.tolist() == moved
        np.testing.assert_array_equal(smap.cpu(), to)
        np.testing.assert_array_equal(ix_out.cpu(), wix)
        np.testing.assert_array_equal(ref_out.cpu(), after)
        np.testing.assert_array_equal(bits(kp), wk)
        idle = np.flatnonzero(after == 0)
        np.testing.assert_array_equal(free.cpu()[:int(nfree)], idle)


# ------------------------------------------------------------------------- sa_shared_prefix_attn

def anchor(heads):
    """A group whose prefix is worth reading once: with it in the batch the call shares every group's prefix it can,
    however small, instead of passing the batch on to the segment attention."""
    return (28000 // heads[1], [(3, 1)] * 32)


def branch_batch(r, heads, page, groups, layers=1, layer=0, spare=2):
    """Caches of groups [(shared, [(own, q), ...])], pages shared as a fork leaves them: the partial one copied.
    K, V: each sequence's rows as (shared part, own part)."""
    Hq, Hkv = heads
    lists, at, q_len, kv_len, gp, need = [], 0, [], [], [0], 0
    for s, members in groups:
        need += s // page + sum(-(-(s + m) // page) - s // page for m, _ in members)
    L = lay(heads, page, need + spare, layers)
    perm = r.permutation(L.num_slots).astype(np.int32)
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    K, V = [], []
    g = torch.Generator(device="cuda").manual_seed(int(r.integers(1 << 30)))

    def gpu_rows(n):
        return (torch.randn((n, Hkv, D), generator=g, device="cuda") * 0.5).to(torch.bfloat16)

    def put(pool, pages, first, x):
        pos = first + torch.arange(len(x), device="cuda")
        slot = torch.from_numpy(np.array(pages, dtype=np.int64)).cuda()[pos // page]
        pool[layer].permute(0, 2, 1, 3)[slot, pos % page] = x.view(torch.int16)

    for s, members in groups:
        common = list(perm[at:at + s // page])
        at += s // page
        ks, vs = gpu_rows(s), gpu_rows(s)
        cut = s // page * page
        if cut:
            put(kp, common, 0, ks[:cut])
            put(vp, common, 0, vs[:cut])
        for own, q in members:
            n = -(-(s + own) // page) - s // page
            pages = common + list(perm[at:at + n])
            at += n
            lists.append(pages)
            k, v = gpu_rows(own), gpu_rows(own)
            put(kp, pages, cut, torch.cat([ks[cut:], k]))
            put(vp, pages, cut, torch.cat([vs[cut:], v]))
            K.append((ks, k))
            V.append((vs, v))
            q_len.append(q)
            kv_len.append(s + own)
        gp.append(len(lists))
    indptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
    indices = np.concatenate([np.array(x, np.int32) for x in lists])
    q = rows(r, (sum(q_len), Hq, D))
    return dict(L=L, kp=kp, vp=vp, indptr=dev(indptr), indices=dev(indices), q=q, K=K, V=V, q_len=q_len, kv_len=kv_len,
                groups=gp, shared=[s for s, _ in groups], heads=heads, layer=layer)


def check_attention(w, o, lse, scale):
    """Every row against float64 (each sequence by itself), within the tolerance at the top."""
    Hq, Hkv = w["heads"]
    G, t0 = Hq // Hkv, 0
    for b, (n, kv) in enumerate(zip(w["q_len"], w["kv_len"])):
        if n == 0:
            continue
        q = w["q"][t0:t0 + n].cuda().double().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
        k, v = (torch.cat([y.cuda() for y in x[b]]).double().permute(1, 0, 2).contiguous() for x in (w["K"], w["V"]))
        kt = k.transpose(1, 2).contiguous()
        s = torch.matmul(q, kt) * scale
        hide = torch.arange(kv, device="cuda")[None, :] > (kv - n + torch.arange(n, device="cuda").repeat_interleave(G))[:, None]
        s.masked_fill_(hide, -float("inf"))
        e = 128 * 2.0 ** -24 * scale * torch.matmul(q.abs(), kt.abs()).masked_fill(hide, 0).amax(-1, keepdim=True)
        ref_lse = torch.logsumexp(s, -1, keepdim=True)
        p = torch.exp(s - ref_lse)
        ref, A = torch.matmul(p, v), torch.matmul(p, v.abs())
        tol = 2.0 ** -8 * (A + 2 * ref.abs()) + (2 * e + (kv + 130) * 2.0 ** -23) * A

        def back(x):
            return x.reshape(Hkv, n, G, -1).permute(1, 0, 2, 3).reshape(n, Hq, -1)
        got = o[t0:t0 + n].double()
        assert torch.isfinite(got).all(), b
        worst = ((got - back(ref)).abs() / back(tol)).max().item()
        assert worst <= 1.0, (b, worst)
        if lse is not None:
            d = (lse[t0:t0 + n].double()[..., None] - back(ref_lse)).abs()
            lim = back(e) + (kv + 130) * 2.0 ** -23 + 2.0 ** -22 * back(ref_lse).abs()
            assert (d <= lim).all(), (b, (d / lim).max().item())
        t0 += n


def run_shared(ctx, w, with_lse=True, scale=D ** -0.5, stream=None):
    T, Hq = sum(w["q_len"]), w["heads"][0]
    o = torch.full((T + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, Hq), 7.0, dtype=torch.float32, device="cuda") if with_lse else None
    sa.sa_shared_prefix_attn(ctx, w["L"], w["layer"], w["q"].cuda(), w["kp"], w["vp"], w["q_len"], w["kv_len"],
                             w["indptr"], w["indices"], w["groups"], w["shared"], scale, o, lse, stream=stream)
    sa.sa_sync_check(ctx)
    assert (o[T:] == 7).all()
    return o[:T], lse


SHARED = [
    # heads, page, groups of (shared, [(own tokens, of them new), ...]); an anchor group comes with each
    ((32, 8), 16, [(200, [(1, 1), (20, 1), (64, 1), (7, 1)])]),
    ((8, 2), 16, [(64, [(1, 1), (1, 1)])]),
    ((8, 2), 16, [(63, [(1, 1), (3, 1)]), (65, [(1, 1), (2, 1), (90, 1)]), (0, [(5, 1), (6, 2)])]),
    ((8, 8), 16, [(1000, [(i + 1, 1) for i in range(40)])]),
    ((16, 1), 32, [(700, [(40 + i, 1) for i in range(9)])]),
    ((24, 8), 16, [(333, [(3 * i + 1, 1) for i in range(50)])]),
    ((10, 2), 32, [(640, [(30, i % 3) for i in range(30)])]),
    ((32, 8), 16, [(500, [(33, 33), (17, 16), (64, 5), (1, 1), (40, 40), (9, 0)])]),
    ((64, 8), 32, [(1500, [(70, 1) for _ in range(20)])]),
    ((4, 2), 16, [(128, []), (300, [(10, 1)]), (300, [(10, 0), (20, 1), (30, 1)]), (40, [(2, 0)])]),
    ((4, 1), 16, [(256, [(200, 150), (300, 200)])]),           # long segments: member by member
    ((4, 1), 16, [(3000, [(1, 1)] * 3), (100, [(2000, 1), (1, 1), (700, 3)]), (0, [(1, 1)])]),
    ((8, 2), 32, [(5000, [(129, 2)] * 17)]),
    ((16, 2), 32, [(2000, [(30, 1)]), (1500, [(900, 1)] * 2), (0, [(4000, 1)]), (70, [(5000, 300)])]),
    ((32, 8), 16, [(3009, [(30, 13)] * 9), (70, [(9, 9)] * 3)]),  # several tokens each: tiles of many members
    ((10, 2), 32, [(2650, [(20 + 7 * i, 9 + i) for i in range(14)])]),
    ((12, 2), 16, [(6001, [(100, 30 + i) for i in range(7)])]),
]


@pytest.mark.parametrize("i", range(len(SHARED)))
def test_shared_prefix_attention(i):
    heads, page, groups = SHARED[i]
    r = np.random.default_rng(100 + i)
    at = i % (len(groups) + 1)
    w = branch_batch(r, heads, page, groups[:at] + [anchor(heads)] + groups[at:], layers=1 + i % 2, layer=i % 2)
    ctx = sa.Context(0)
    o, lse = run_shared(ctx, w)
    check_attention(w, o, lse, D ** -0.5)
    # again, with the plan at hand and no lse: the same bits
    o2, _ = run_shared(ctx, w, with_lse=False)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("i", range(len(SHARED)))
def test_shared_prefix_attention_of_small_batches(i):
    """The same groups by themselves: most are passed on to the segment attention."""
    heads, page, groups = SHARED[i]
    w = branch_batch(np.random.default_rng(200 + i), heads, page, groups)
    ctx = sa.Context(0)
    sa.sa_set_exact_scale(ctx, False)                        # the call's own scale is exact all the same
    for _ in range(2):
        o, lse = run_shared(ctx, w)
        check_attention(w, o, lse, D ** -0.5)


def test_shared_prefix_attention_with_large_scores():
    r = np.random.default_rng(7)
    w = branch_batch(r, (32, 8), 16, [(900, [(50, 1)] * 12), anchor((32, 8)), (300, [(10, 1)] * 5)])
    w["kp"].view(torch.bfloat16).mul_(8)                     # exact: a power of two (and NaN stays NaN)
    w["K"] = [(a * 8, b * 8) for a, b in w["K"]]
    ctx = sa.Context(0)
    o, lse = run_shared(ctx, w, scale=1.0)
    check_attention(w, o, lse, 1.0)


def test_shared_prefix_attention_agrees_with_the_segment_attention():
    r = np.random.default_rng(8)
    w = branch_batch(r, (32, 8), 16, [(6000, [(30, 1)] * 20), (100, [(30, 4)] * 3)])
    ctx = sa.Context(0)
    o, lse = run_shared(ctx, w)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    sa.sa_segment_prefill_attn(ctx, w["L"], 0, w["q"].cuda(), w["kp"], w["vp"], w["q_len"], w["kv_len"], w["indptr"],
                               w["indices"], D ** -0.5, o2, lse2)
    sa.sa_sync_check(ctx)
    check_attention(w, o2, lse2, D ** -0.5)


def test_shared_prefix_attention_plans_follow_the_lengths():
    ctx = sa.Context(0)
    side = torch.cuda.Stream()
    for i, n in enumerate([1, 5, 12, 5, 1, 12]):             # shared, but the fifth
        groups = [(400 + 64 * i, [(9, 1)] * n)] + ([anchor((8, 2))] if i != 4 else [])
        w = branch_batch(np.random.default_rng(40 + i), (8, 2), 16, groups)
        torch.cuda.synchronize()
        o, lse = run_shared(ctx, w, stream=side if i == 2 else None)
        torch.cuda.synchronize()
        check_attention(w, o, lse, D ** -0.5)


def test_shared_prefix_attention_reports_bad_pages():
    w = branch_batch(np.random.default_rng(12), (8, 2), 16, [(256, [(9, 1)] * 6), anchor((8, 2))])
    ctx = sa.Context(0)
    w["indices"][3] = w["L"].num_slots                       # a shared page of the first member
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        run_shared(ctx, w)
    w["indices"][3] = -1
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        run_shared(ctx, w)


def test_planned_calls_refuse_capture():
    w = branch_batch(np.random.default_rng(13), (8, 2), 16, [(64, [(9, 1)] * 2)])
    ctx = sa.Context(0)
    run_shared(ctx, w)
    T = 2
    o, q = torch.empty((T, 8, D), dtype=torch.bfloat16, device="cuda"), w["q"].cuda()
    k = torch.zeros((T, 2, D), dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(8, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(sa.SaError, match="SA_ERR_UNSUPPORTED"):
            sa.sa_shared_prefix_attn(ctx, w["L"], 0, q, w["kp"], w["vp"], w["q_len"], w["kv_len"], w["indptr"],
                                     w["indices"], w["groups"], w["shared"], 0.1, o)
        with pytest.raises(sa.SaError, match="SA_ERR_UNSUPPORTED"):
            sa.sa_kv_append_rope(ctx, w["L"], 0, sa.Rope(), q, k, k, o, w["kp"], w["vp"], [64, 64], [1, 1], w["indptr"],
                                 w["indices"])
        with pytest.raises(sa.SaError, match="SA_ERR_UNSUPPORTED"):
            sa.sa_kv_fork(ctx, w["L"], w["kp"], w["vp"], [16], [0], [0], w["indptr"], w["indices"], t, t, t)


def test_counts_refuse_to_allocate_in_a_capture():
    L = lay((2, 2), 16, 10000)
    ctx = sa.Context(0)
    ref, free = torch.zeros(10000, dtype=torch.int32, device="cuda"), torch.zeros(10000, dtype=torch.int32, device="cuda")
    n, ip, ix = torch.zeros(1, dtype=torch.int32, device="cuda"), dev([0, 1]), dev([3])
    sa.sa_kv_retain(ctx, L, ip, ix, ref)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(sa.SaError, match="SA_ERR_UNSUPPORTED"):
            sa.sa_kv_release(ctx, L, ip, ix, ref, free, n)
    sa.sa_kv_release(ctx, L, ip, ix, ref, free, n)
    sa.sa_sync_check(ctx)
    assert int(n) == 10000 and torch.equal(free.cpu(), torch.arange(10000, dtype=torch.int32))


def test_binding_refuses_other_types_and_layouts():
    L = lay((4, 2), 16, 8)
    ctx = sa.Context(0)
    q, k = (torch.zeros((2, h, D), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    pool = torch.zeros((1, 8, 2, 16, D), dtype=torch.bfloat16, device="cuda")
    ip, ix = dev([0, 1]), dev([3])

    def rope(q=q, k=k, out=q, pool=pool, r=sa.Rope(), ip=ip):
        sa.sa_kv_append_rope(ctx, L, 0, r, q, k, k, out, pool, pool.clone(), [0], [2], ip, ix)

    rope()
    for bad in (dict(q=q.half()), dict(out=q.half()), dict(q=q.float()), dict(k=k.transpose(0, 1)), dict(q=q[:, :3]),
                dict(q=q.flatten(1)), dict(q=q[:1]), dict(out=q[:1]), dict(pool=pool.half()), dict(pool=pool[:, :7]),
                dict(r=sa.Rope(q_weight=q[0, 0].half())), dict(r=sa.Rope(q_weight=q[0, 0, :64])), dict(ip=ip.long()),
                dict(q=torch.zeros((2, 4, 2 * D), dtype=torch.bfloat16, device="cuda")[:, :, ::2]), dict(q=None)):
        with pytest.raises(ValueError):
            rope(**bad)
    for stride_ok in (torch.zeros((2, 9, D), dtype=torch.bfloat16, device="cuda")[:, 1:5],):
        rope(q=stride_ok)
    with pytest.raises(sa.SaError, match="SA_ERR_SHAPE"):
        rope(q=q[:1].expand(2, 4, D))
    with pytest.raises(ValueError):
        sa.sa_kv_release(ctx, L, ip, ix, torch.zeros(7, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        sa.sa_kv_compact(ctx, L, pool, pool, 4, ix, ix, ix, ix, ix, ix)
    sa.sa_sync_check(ctx)


def test_pools_beyond_4_gib_of_a_layer():
    """Slots whose rows lie past 2^32 bytes of their pool: every call reaches them."""
    r = np.random.default_rng(31)
    heads, page, far = (32, 8), 16, 139000
    w = branch_batch(r, heads, page, [(1500, [(90, 1)] * 20), anchor(heads)])
    small, big = w["L"], lay(heads, page, far + w["L"].num_slots)
    pools = []
    for name in ("kp", "vp"):
        p = torch.empty((1, big.num_slots, 8, page, D), dtype=torch.int16, device="cuda")
        p[:, far:] = w[name]
        pools.append(p)
    w.update(L=big, kp=pools[0], vp=pools[1], indices=w["indices"] + far)
    ctx = sa.Context(0)
    o, lse = run_shared(ctx, w)
    check_attention(w, o, lse, D ** -0.5)
    # new rows onto the first member's last page, through a fork of it
    ref = torch.zeros(big.num_slots, dtype=torch.int32, device="cuda")
    one_ip, one_ix = w["indptr"][:2].contiguous(), w["indices"][:int(w["indptr"][1])].contiguous()
    sa.sa_kv_retain(ctx, big, one_ip, one_ix, ref)
    fresh = dev([far + small.num_slots - 1])
    dip, dix = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(100, dtype=torch.int32, device="cuda")
    assert sa.sa_kv_fork(ctx, big, *pools, [1590], [0], [1], one_ip, one_ix, fresh, dip, dix, ref=ref) == 1
    q, k, v = rows(r, (1, 32, D)).cuda(), rows(r, (1, 8, D)).cuda(), rows(r, (1, 8, D)).cuda()
    out = torch.empty_like(q)
    sa.sa_kv_append_rope(ctx, big, 0, sa.Rope(), q, k, v, out, *pools, [1590], [1], dip, dix)
    sa.sa_sync_check(ctx)
    last = pools[0][0, int(fresh[0])]
    assert torch.equal(last[:, :6], pools[0][0, int(one_ix[-1])][:, :6])
    assert torch.equal(last[:, 6], k[0].view(torch.int16)) and torch.equal(out, q)
    # and down into the first slots
    smap, mv = torch.zeros_like(ref), torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = dix[:100].contiguous()
    before = pools[1][0, kept.long()].clone()
    sa.sa_kv_compact(ctx, big, *pools, far, ref, ref, kept, kept, smap, mv)
    sa.sa_sync_check(ctx)
    assert mv.tolist() == [101, 0] and int(kept.max()) <= 100
    assert torch.equal(pools[1][0, kept.long()], before)


DEBUG = r"""
import sys
sys.path.insert(0, {root!r}); sys.path.insert(0, {tests!r})
import numpy as np, torch
import paper_2607_00151_amd as sa
from test_gpu_branches import D, bits, dev, lay, pool_bits, rows
r = np.random.default_rng(1)
L, ctx = lay((4, 2), 16, 16), sa.Context(0)
kp, vp = pool_bits(r, L), pool_bits(r, L)
before = bits(kp).copy(), bits(vp).copy()
dip, dix = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")

def name(f):
    try:
        f()
    except sa.SaError as e:
        torch.cuda.synchronize()
        assert np.array_equal(bits(kp), before[0]) and np.array_equal(bits(vp), before[1])
        return e.name
    sa.sa_sync_check(ctx)

def fork(table=(3, 4), fresh=(7, 8, 9)):
    sa.sa_kv_fork(ctx, L, kp, vp, [20], [0, 0], [4, 16], dev([0, len(table)]), dev(table), dev(fresh), dip, dix)

def rope(table):
    T = 2
    q, k = rows(r, (T, 4, D)).cuda(), rows(r, (T, 2, D)).cuda()
    sa.sa_kv_append_rope(ctx, L, 0, sa.Rope(), q, k, k, q, kp, vp, [5, 5], [1, 1], dev([0, 1, 2]), dev(table))

assert name(lambda: fork(fresh=(7, 8, 7))) == "SA_ERR_OVERLAP"
assert name(lambda: fork(fresh=(7, 4, 9))) == "SA_ERR_OVERLAP"
assert name(lambda: fork(fresh=(7, 16, 9))) == "SA_ERR_RANGE"
assert name(lambda: fork(table=(3, 16))) == "SA_ERR_RANGE"
assert name(lambda: fork(table=(3,))) == "SA_ERR_RANGE"
assert name(lambda: rope((6, 6))) == "SA_ERR_OVERLAP"
assert name(lambda: rope((6, -1))) == "SA_ERR_RANGE"
assert name(fork) is None and dix[:5].tolist() == [3, 7, 3, 8, 9]
assert name(lambda: rope((6, 11))) is None
print("debug branch checks ok", flush=True)
"""


@pytest.mark.timeout(300)
def test_debug_checks():
    code = DEBUG.format(root=ROOT, tests=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-u", "-c", code], env=dict(os.environ, SA_DEBUG="1"), capture_output=True,
                       text=True, timeout=240)
    print(r.stdout[-2000:], r.stderr[-3000:])
    assert r.returncode == 0 and "debug branch checks ok" in r.stdout


def test_reserved_contexts_give_the_same_bits():
    w = branch_batch(np.random.default_rng(51), (8, 2), 16, [(700, [(9, 1)] * 6), anchor((8, 2))])
    o, lse = run_shared(sa.Context(0), w)
    ctx = sa.Context(0)
    sa.sa_reserve(ctx, 1 << 20, 64 << 20)
    for _ in range(2):
        o2, lse2 = run_shared(ctx, w)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        sa.sa_reserve(ctx, 4 << 20, 128 << 20)              # the plan on the device goes: made again


def test_timing_events_bind_to_the_branch_kernels():
    w = branch_batch(np.random.default_rng(52), (8, 2), 16, [anchor((8, 2))])
    ctx = sa.Context(0)
    run_shared(ctx, w)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    for e in ev:
        e.record()
    sa.sa_set_kernel_events(ctx, sa.TIMED_ATTN, ev[0].cuda_event, ev[1].cuda_event)
    sa.sa_set_kernel_events(ctx, sa.TIMED_PAGES, ev[2].cuda_event, ev[3].cuda_event)
    run_shared(ctx, w)
    ref = torch.zeros(w["L"].num_slots, dtype=torch.int32, device="cuda")
    sa.sa_kv_retain(ctx, w["L"], w["indptr"], w["indices"], ref)
    sa.sa_set_kernel_events(ctx, sa.TIMED_ATTN)
    sa.sa_set_kernel_events(ctx, sa.TIMED_PAGES)
    torch.cuda.synchronize()
    assert 0 < ev[0].elapsed_time(ev[1]) < 10 and 0 < ev[2].elapsed_time(ev[3]) < 10


# ------------------------------------------------------------------------- together

def test_branches_from_fork_to_compaction():
    """A context is forked, its branches grow by rotated rows and attend (the prefix computed once); all but two end,
    the pool is compacted, and the two go on: every step's attention against float64 over the rows in the cache."""
    r = np.random.default_rng(21)
    heads, page, layers, n0, n = (8, 2), 16, 2, 14003, 24
    Hq, Hkv = heads
    first = -(-n0 // page)
    L = lay(heads, page, first + 5 * n, layers)
    rope = sa.Rope(10000.0 ** (-np.arange(64) / 64), rows(r, (D,), 1.0).cuda(), rows(r, (D,), 1.0).cuda(), 1e-6)
    ctx = sa.Context(0)
    kp, vp = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    ref = torch.zeros(L.num_slots, dtype=torch.int32, device="cuda")
    fresh = r.permutation(L.num_slots).astype(np.int32)
    sip, six = dev([0, first]), dev(fresh[:first])
    sa.sa_kv_retain(ctx, L, sip, six, ref)

    def append(start, new, ip, ix):
        q, k, v = (rows(r, (sum(new), h, D)).cuda() for h in (Hq, Hkv, Hkv))
        out = torch.empty_like(q)
        for layer in range(layers):
            sa.sa_kv_append_rope(ctx, L, layer, rope, q, k, v, out, kp, vp, start, new, ip, ix)
        return out

    def cached(ip, ix, lens, layer=1):
        ipn = ip.tolist()
        return [[(pool.view(torch.bfloat16)[layer][ix[ipn[b]:ipn[b + 1]].long()].permute(0, 2, 1, 3)
                  .reshape(-1, Hkv, D)[:m].clone(),) for b, m in enumerate(lens)] for pool in (kp, vp)]

    def attend(new, lens, ip, ix, q):
        K, V = cached(ip, ix, lens)
        w = dict(L=L, kp=kp, vp=vp, indptr=ip, indices=ix, q=q.cpu(), K=K, V=V, q_len=new, kv_len=lens,
                 groups=[0, len(new)], shared=[n0], heads=heads, layer=1)
        check_attention(w, *run_shared(ctx, w), D ** -0.5)
        return K, V

    append([0], [n0], sip, six)
    base = cached(sip, six, [n0])
    dip = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    dix = torch.zeros(n * (first + 4), dtype=torch.int32, device="cuda")
    used = sa.sa_kv_fork(ctx, L, kp, vp, [n0], [0] * n, [40] * n, sip, six, dev(fresh[first:]), dip, dix, ref=ref)
    assert used == n * (-(-(n0 + 40) // page) - n0 // page)
    lens = [n0] * n
    for new in ([5, 1, 9, 2] * 6, [1] * n, [20, 3, 1, 0] * 6):
        q = append(lens, new, dip, dix)
        lens = [a + m for a, m in zip(lens, new)]
        K, V = attend(new, lens, dip, dix, q)
        for b in range(n):
            assert torch.equal(K[b][0][:n0], base[0][0][0]) and torch.equal(V[b][0][:n0], base[1][0][0])
    # all branches but 0 and 1 and the context's own table end; the two that go on move together
    free, nfree = torch.zeros_like(ref), torch.zeros(1, dtype=torch.int32, device="cuda")
    sa.sa_kv_release(ctx, L, dip[2:].contiguous(), dix, ref)
    sa.sa_kv_release(ctx, L, sip, six, ref, free, nfree)
    live = sorted(set(dix[:int(dip[2])].tolist()))
    assert free[:int(nfree)].tolist() == sorted(set(range(L.num_slots)) - set(live))
    kept, ip2 = dix[:int(dip[2])].contiguous(), dip[:3].contiguous()
    smap, mv = torch.zeros_like(ref), torch.zeros(2, dtype=torch.int32, device="cuda")
    sa.sa_kv_compact(ctx, L, kp, vp, len(live), ref, ref, kept, kept, smap, mv)
    sa.sa_sync_check(ctx)
    assert mv[1] == 0 and sorted(set(kept.tolist())) == list(range(len(live)))
    K2, V2 = cached(ip2, kept, lens[:2])
    assert all(torch.equal(a[0], b[0]) for a, b in zip(K[:2] + V[:2], K2 + V2))
    q = append(lens[:2], [1, 2], ip2, kept)
    attend([1, 2], [lens[0] + 1, lens[1] + 2], ip2, kept, q)

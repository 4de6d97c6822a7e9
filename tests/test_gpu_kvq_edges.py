"""Attention over a 4-bit cache where it can go wrong: queries with outlier dims, values that are infinities
or large, very many keys; and caches so long that a few lost keys hardly show.

References and bounds: kvq_bounds.py."""
import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa
from kvq_bounds import attention, coded_values, coded_worst, worst
from kvq_reference import D, page_bytes, rows_of
from test_gpu_branches import dev, lay, rows, tables

pytestmark = pytest.mark.gpu


class Case:
    """A cache, queries and page tables of one call; edit(x) changes the float64 rows k and v before they are quantised,
    patch(case) their bytes."""

    def __init__(self, seed, heads, page, q_len, kv_len, causal=True, scale=D ** -0.5, edit=None, q=None, patch=None, copies=1):
        r = np.random.default_rng(seed)
        pages = [-(-n // page) for n in kv_len]
        self.L = lay(heads, page, sum(pages) + 3)
        self.heads, self.page, self.q_len, self.kv_len, self.causal, self.scale = heads, page, q_len, kv_len, causal, scale
        self.indptr, self.indices, _ = tables(r, pages, self.L.num_slots)
        if copies > 1:                                       # that many sequences over the same pages
            self.indptr, self.indices = np.arange(copies + 1) * pages[0], np.tile(self.indices, copies)
            self.q_len, self.kv_len = q_len * copies, kv_len * copies
        self.x = {n: r.standard_normal((1, self.L.num_slots, heads[1], page, D)) * 0.5 for n in "kv"}
        if edit:
            edit(self.x)
        self.k, self.v = (page_bytes(self.x[n]) for n in "kv")
        self.q = rows(r, (sum(self.q_len), heads[0], D), 0.5)
        if q is not None:
            q(self.q)
        if patch:
            patch(self)
        self.on_gpu()

    def on_gpu(self):
        self.k4, self.v4, self.qd = torch.from_numpy(self.k).cuda(), torch.from_numpy(self.v).cuda(), self.q.cuda()
        self.ip, self.ix = dev(self.indptr), dev(self.indices)

    def run(self, ctx, stream=None):
        o = torch.full((len(self.q), self.heads[0], D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((len(self.q), self.heads[0]), 7.0, device="cuda")
        sa.sa_kvq_attn(ctx, self.L, 0, self.qd, self.k4, self.v4, self.q_len, self.kv_len, self.ip, self.ix, self.scale, o, lse,
                       causal=self.causal, stream=stream)
        return o, lse

    def check(self, o, lse, only=None, inexact=False):
        t = 0
        for b, (n, kv) in enumerate(zip(self.q_len, self.kv_len)):
            if n and (only is None or b in only):
                k, v = (rows_of(p[0], self.indptr, self.indices, b, kv, self.page) for p in (self.k, self.v))
                off = worst(o[t:t + n], lse[t:t + n], attention(self.q[t:t + n], k, v, self.scale, self.causal, inexact))
                assert max(off) <= 1.0, (b, off)
            t += n


def checked(*args, **kw):
    c = Case(*args, **kw)
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    c.check(o, lse)
    return c, o, lse


# few rows, whose waves split the keys; 40 and more, whose waves split the rows, in one sequence or beside others
SIZES = [((8, 2), 16, [1, 6], [300, 1500], True), ((8, 2), 32, [20, 3], [700, 400], True), ((32, 8), 16, [40], [900], False),
         ((4, 4), 16, [100], [3000], True)]


@pytest.mark.parametrize("power", [8, 12, 16])
@pytest.mark.parametrize("size", SIZES)
def test_dims_beside_an_outlier_count_where_its_keys_are_zero(size, power):
    """One dim of a block 2^8 to 2^16 times the others: what it hides in the query's scale is all of the score."""
    heads, page, q_len, kv_len, causal = size

    def edit(x):
        x["k"][..., [5, 40, 127]] = 0

    def q(x):
        x[..., [5, 40, 127]] *= 2.0 ** power
    checked(power, heads, page, q_len, kv_len, causal, edit=edit, q=q)


@pytest.mark.parametrize("size", SIZES)
def test_a_few_small_dims_beside_an_outlier_and_zeros(size):
    heads, page, q_len, kv_len, causal = size

    def edit(x):
        x["k"][..., 8] = 0

    def q(x):
        x[..., 32:] = 0
        x[..., 3:8], x[..., 9:32] = 0, 0
        x[..., 8] *= 5000
    checked(7, heads, page, q_len, kv_len, causal, edit=edit, q=q)


@pytest.mark.parametrize("spread", ["2", "4", "8", "32", "exponential", "lognormal"])
@pytest.mark.parametrize("heads,page,q,kv", [((32, 8), 16, [40], [60]), ((1, 1), 32, [100, 34], [100, 2000]), ((8, 1), 16, [5] * 9, [5] * 9)])
def test_what_rows_of_spread_queries_may_lose(heads, page, q, kv, spread):
    """Rows on both sides of what pieces hold well enough, over few keys and with large scores."""
    def change(x):
        r = np.random.default_rng(17)
        if spread == "lognormal":
            f = np.exp(1.5 * r.standard_normal(x.shape))
        elif spread == "exponential":
            f = np.sqrt(r.exponential(size=x.shape))
        else:
            f = np.where(np.arange(D) % 32 == 9, float(spread), 1.0)
        x.copy_((x.double() * torch.from_numpy(np.broadcast_to(f, x.shape).copy())).to(torch.bfloat16))
    c = Case(11, heads, page, q, kv, True, scale=0.3, q=change, edit=lambda x: x["k"].__setitem__((..., np.arange(D) % 32 == 9), 0))
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    c.check(o, lse, inexact=True)


def test_one_row_with_an_outlier_among_ordinary_ones():
    """Its work item's products are exact; the others' items are as they were."""
    def edit(x):
        x["k"][..., 5] = 0

    def q(x):
        x[77, 3, 5] = 20000.0
    checked(9, (32, 8), 16, [100, 60], [2000, 700], True, edit=edit, q=q)


# Codes that stand for more than a bf16 holds, by scale byte: 4 and 6 under 253, 2 and more under 254.
BEYOND = {253: {6: 1, 7: 1, 14: -1, 15: -1}, 254: {4: 1, 5: 1, 6: 1, 7: 1, 12: -1, 13: -1, 14: -1, 15: -1}}


@pytest.mark.parametrize("heads,page,q,kv,at,causal", [
    ((8, 2), 16, 1, 300, 299, True), ((8, 2), 16, 6, 300, 297, True), ((8, 2), 16, 3, 3, 1, True), ((32, 8), 32, 40, 200, 170, True),
    ((8, 2), 16, 70, 70, 3, True), ((4, 2), 16, 9, 130, 64, False), ((2, 1), 16, 100, 5000, 4950, True), ((4, 4), 16, 9, 40, 35, True),
    ((1, 1), 32, 130, 1000, 900, True), ((4, 1), 16, 32, 700, 680, True)])
@pytest.mark.parametrize("scale", [253, 254])
@pytest.mark.parametrize("outlier", [False, True])
def test_an_infinite_value_reaches_the_rows_that_see_it(heads, page, q, kv, at, causal, scale, outlier):
    """A block under a scale byte that quantising never gives, as another tool may have written it: infinities in some of
    its dims, finite values or zeros in the others."""
    signs = np.zeros(32)
    codes = np.zeros(32, np.uint8)
    for i, (c, sign) in enumerate(BEYOND[scale].items()):
        codes[3 * i + 1], signs[3 * i + 1] = c, sign
    codes[[2, 31]] = 1, 9                                   # half a unit: finite

    def bytes_of(case):
        p = case.v[0, case.indices[at // page], 0]
        return p[:64 * page].reshape(page, 64)[at % page, 32:48], p[64 * page:].reshape(page, 4)[at % page]

    def patch(case):
        b, s = bytes_of(case)
        b[:], s[2] = codes[0::2] | codes[1::2] << 4, scale

    def big(x):
        if outlier:
            x[..., 5] = 5000.0
    c = Case(31, heads, page, [q], [kv], causal, patch=patch, q=big, edit=lambda x: x["k"].__setitem__((..., 5), 0))
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    G = heads[0] // heads[1]
    sees = np.array([not causal or kv - q + i >= at for i in range(q)])
    got = o.double().cpu().numpy()
    want = np.zeros_like(got)
    want[np.ix_(sees, np.arange(G), np.arange(64, 96))] = np.where(signs == 0, 0, np.inf * np.where(signs == 0, 1, signs))
    np.testing.assert_array_equal(np.where(np.isinf(got) | np.isnan(got), got, 0), want)
    # everything else is as with zeros in those dims
    b, s = bytes_of(c)
    codes[signs != 0] = 0
    b[:] = codes[0::2] | codes[1::2] << 4
    k, v = (rows_of(p[0], c.indptr, c.indices, 0, kv, page) for p in (c.k, c.v))
    ref = attention(c.q, k, v, c.scale, causal)
    off = ((o.double().cpu() - ref[0]).abs() / ref[2]).numpy()
    assert (off[want == 0] <= 1).all()
    assert ((lse.double().cpu() - ref[1]).abs() <= ref[3]).all()


@pytest.mark.parametrize("heads,page,q,kv,at", [((8, 2), 16, 6, 300, 297), ((32, 8), 32, 40, 200, 170), ((4, 4), 16, 9, 40, 35)])
def test_an_infinite_key_stays_out_of_the_rows_that_do_not_see_it(heads, page, q, kv, at):
    def bytes_of(case):
        p = case.k[0, case.indices[at // page], 0]
        return p[:64 * page].reshape(page, 64)[at % page, 32:48], p[64 * page:].reshape(page, 4)[at % page]

    def patch(case):
        b, s = bytes_of(case)
        b[:], s[2] = 0x7E, 254
    c = Case(32, heads, page, [q], [kv], True, patch=patch)
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    bytes_of(c)[0][:] = 0
    k, v = (rows_of(p[0], c.indptr, c.indices, 0, kv, page) for p in (c.k, c.v))
    n = at - (kv - q)                                       # rows before the one at that position
    part = attention(c.q, k, v, c.scale, True)
    off = worst(o[:n], lse[:n], [x[:n] for x in part])
    assert n > 0 and max(off) <= 1.0, off


# 512 sequences over the same pages: as many items as there are places, whose keys are not cut into many parts
@pytest.mark.parametrize("q,rise", [([1], 7.5), ([20], 7.5), ([40], 10.5), ([100], 10.5)])
def test_sums_of_large_values_are_finite(q, rise):
    """Values just below 2^110, and weights that outgrow a row's first ones by nearly as much as its offset lets them."""
    kv = 20000

    def edit(x):
        x["k"][:], x["v"][:] = 0, np.abs(x["v"]) % 0.35 * 2.0 ** 110 + 2.0 ** 109

    def patch(case):                                        # every other 64 keys: ones
        ones = page_bytes(np.ones((1, 16, D)))
        for i in range(kv // 16):
            if i // 4 % 2:
                case.k[0, case.indices[i]] = ones

    def q_half(x):
        x[:] = 0.5
    c = Case(41, (1, 1), 16, q, [kv], False, scale=rise * np.log(2) / 64, edit=edit, patch=patch, q=q_half, copies=512)
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    c.check(o, lse, only=(0, 511))
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("q", [[1], [6], [20], [40], [100]])
def test_more_keys_of_one_weight_than_an_offset_keeps(q):
    """Keys of zeros: the LSE is that of their number, of which one is 6.7e-6; the output their values' mean."""
    kv = 150001

    def edit(x):
        x["k"][:] = 0
    c = Case(42, (1, 1), 16, q, [kv], False, edit=edit, copies=512)
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    v = rows_of(c.v[0], c.indptr, c.indices, 0, kv, 16)
    mean, size = (torch.from_numpy(f(v).mean(1)) for f in (np.asarray, np.abs))
    # log2 of the sum: fp32 additions of whole numbers are exact, v_log's result and the sum's power of two
    # are off by half a unit of 2^-19 each, the product with ln 2 by half a unit of 2^-20
    assert (lse.double().cpu() - np.log(kv)).abs().max() <= (2.0 ** -19 * np.log(2) + 2.0 ** -21)
    # weights are powers of two, so only the output is rounded, and fp32 sums of a sixteenth of the keys at most
    off = (o.double().cpu() - mean[None]).abs() - 2.0 ** -8 * mean[None].abs() - (kv / 16 + 64) * 2.0 ** -24 * size[None]
    assert off.max() <= 0


# ---- long caches

LONG = [((8, 2), 16, [1, 1], [40000, 31001], True), ((32, 8), 16, [1], [9000], False), ((2, 1), 32, [40], [20011], True),
        ((16, 1), 16, [6], [30000], True), ((16, 1), 16, [1, 1], [60000, 1], True), ((4, 4), 32, [1] * 3, [65000, 64, 9000], False),
        ((16, 4), 32, [2, 30, 1, 7, 14], [9000, 6000, 20000, 77, 12345], True), ((2, 1), 16, [100], [8000], True),
        ((32, 8), 16, [1, 40, 1, 1], [5000, 3000, 12000, 65], True), ((4, 1), 32, [200], [30000], False)]


@pytest.mark.parametrize("case", LONG)
def test_long_caches(case):
    checked(51, *case)


@pytest.mark.parametrize("case", LONG)
def test_every_key_of_a_long_cache_counts_once(case):
    heads, page, q_len, kv_len, causal = case

    def patch(c):
        for b, kv in enumerate(kv_len):
            slots = c.indices[c.indptr[b]:c.indptr[b + 1]]
            v = coded_values(len(slots) * page).numpy().reshape(len(slots), 1, page, D)
            c.v[0, slots] = page_bytes(v)

    def edit(x):
        x["k"][:] = 0
    c = Case(52, heads, page, q_len, kv_len, causal, edit=edit, patch=patch)
    ctx = sa.Context(0)
    o, lse = c.run(ctx)
    sa.sa_sync_check(ctx)
    t = 0
    for n, kv in zip(q_len, kv_len):
        off = coded_worst(o[t:t + n], lse[t:t + n], kv, causal)
        assert max(off) <= 1.0, (n, kv, off)
        t += n


def test_a_page_list_is_needed_only_where_queries_have_keys():
    L, ctx = lay((4, 2), 16, 4), sa.Context(0)
    pool = torch.zeros(sa.kvq_pool_shape(L), dtype=torch.uint8, device="cuda")
    q = torch.ones((2, 4, D), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full((2, 4), 7.0, device="cuda")
    sa.sa_kvq_attn(ctx, L, 0, q, pool, pool, [0, 2, 0], [50, 0, 3], dev([0, 0, 0, 0]), None, 1.0, o, lse, causal=False)
    sa.sa_sync_check(ctx)
    assert (o == 0).all() and (lse == -np.inf).all()
    sa.sa_kvq_attn(ctx, L, 0, None, pool, pool, [0], [50], dev([0, 0]), None, 1.0, None)
    with pytest.raises(ValueError):
        sa.sa_kvq_attn(ctx, L, 0, q, pool, pool, [0, 2], [50, 3], dev([0, 0, 0]), None, 1.0, o, lse)
    sa.sa_sync_check(ctx)


def test_rows_without_keys_beside_rows_with_some():
    checked(81, (32, 8), 16, [40, 1, 100, 6, 20], [0, 0, 500, 0, 77], False)

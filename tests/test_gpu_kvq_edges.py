"""Attention over a 4-bit cache where it can go wrong: queries with outlier dims.

References and bounds: kvq_bounds.py."""
import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa
from kvq_bounds import attention, worst
from kvq_reference import D, page_bytes, rows_of
from test_gpu_branches import dev, lay, rows, tables

pytestmark = pytest.mark.gpu


class Case:
    """A cache, queries and page tables of one call; edit(x) changes the float64 rows k and v before they are quantised."""

    def __init__(self, seed, heads, page, q_len, kv_len, causal=True, scale=D ** -0.5, edit=None, q=None):
        r = np.random.default_rng(seed)
        pages = [-(-n // page) for n in kv_len]
        self.L = lay(heads, page, sum(pages) + 3)
        self.heads, self.page, self.q_len, self.kv_len, self.causal, self.scale = heads, page, q_len, kv_len, causal, scale
        self.indptr, self.indices, _ = tables(r, pages, self.L.num_slots)
        self.x = {n: r.standard_normal((1, self.L.num_slots, heads[1], page, D)) * 0.5 for n in "kv"}
        if edit:
            edit(self.x)
        self.k, self.v = (page_bytes(self.x[n]) for n in "kv")
        self.q = rows(r, (sum(q_len), heads[0], D), 0.5)
        if q is not None:
            q(self.q)
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

    def check(self, o, lse):
        t = 0
        for b, (n, kv) in enumerate(zip(self.q_len, self.kv_len)):
            if n:
                k, v = (rows_of(p[0], self.indptr, self.indices, b, kv, self.page) for p in (self.k, self.v))
                off = worst(o[t:t + n], lse[t:t + n], attention(self.q[t:t + n], k, v, self.scale, self.causal))
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


def test_one_row_with_an_outlier_among_ordinary_ones():
    """Its work item's products are exact; the others' items are as they were."""
    def edit(x):
        x["k"][..., 5] = 0

    def q(x):
        x[77, 3, 5] = 20000.0
    checked(9, (32, 8), 16, [100, 60], [2000, 700], True, edit=edit, q=q)

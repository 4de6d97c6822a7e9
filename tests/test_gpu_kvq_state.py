"""What a context keeps from call to call: plans by their keys, the partials' buffer, the counters at which launches join
their parts.  Calls of every kind after one another on one context give the bits that each gives on a fresh one."""
import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa
from test_gpu_branches import FILL, dev, lay, pool_bits, rows, tables
from test_gpu_kvq import pool4
from test_gpu_kvq_edges import D, Case

pytestmark = pytest.mark.gpu


class Bf16:
    """A segment attention over a bf16 cache, split by key range."""

    def __init__(self):
        r = np.random.default_rng(3)
        self.L = lay((32, 8), 16, 600)
        self.indptr, self.indices, _ = tables(r, [563, 5], 600)
        shape = (1, 600, 8, 16, D)
        self.args = [rows(r, (3, 32, D)).cuda(), rows(r, shape).cuda(), rows(r, shape).cuda(), [1, 2], [9000, 70],
                     dev(self.indptr), dev(self.indices), D ** -0.5]

    def run(self, ctx):
        o, lse = torch.empty((3, 32, D), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 32), device="cuda")
        sa.sa_segment_prefill_attn(ctx, self.L, 0, *self.args, o, lse)
        return o, lse


def test_attentions_after_one_another_on_one_context():
    calls = [
        Case(61, (32, 8), 16, [1] * 4, [3000, 1000, 4096, 70]),              # a few rows, joined in the launch
        Case(62, (32, 8), 16, [40], [5000]),                                 # row tiles, joined by a second launch
        Case(62, (32, 8), 16, [40], [5000], causal=False),                   # another mask, the same lengths
        Case(62, (16, 8), 16, [40], [5000]),                                 # other heads, the same lengths
        Case(62, (32, 4), 16, [40], [5000]),
        Case(62, (32, 8), 32, [40], [5000]),                                 # another page size, the same lengths
        Case(63, (32, 8), 32, [6], [60000]),                                 # rows of two blocks, a second launch
        Bf16(),
        Case(64, (32, 8), 16, [1, 100, 7], [9000, 30000, 500]),              # row tiles, joined in the launch
        Case(65, (32, 8), 16, [300, 30], [20000, 60000]),                    # both, and twice the partials of those before
        Case(66, (8, 1), 16, [1] * 6, [30000, 7000, 12000, 25000, 4500, 9000]),
        Case(67, (32, 8), 16, [1, 0, 3], [70, 9, 64]),                       # no parts
    ]
    want = []
    for c in calls:
        fresh = sa.Context(0)
        want.append(c.run(fresh))
        sa.sa_sync_check(fresh)
    ctx = sa.Context(0)
    order = list(range(len(calls)))
    for i in order + order[::-1] + [0, 6, 0, 8, 0, 7, 1, 7, 9, 7, 10, 7, 2, 1, 3, 1, 5, 1]:
        o, lse = calls[i].run(ctx)
        assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1]), i
    sa.sa_sync_check(ctx)


def test_appends_after_one_another_on_one_context():
    """Only one thing differs from call to call."""
    r = np.random.default_rng(71)
    heads, page, start, new = (8, 2), 16, [3, 17, 40], [5, 30, 1]
    T = sum(new)
    L = lay(heads, page, 12)
    indptr, indices, _ = tables(r, [1, 3, 3], 12)
    ip, ix = dev(indptr), dev(indices)
    q, k, v = rows(r, (T, 8, D)).cuda(), rows(r, (T, 2, D)).cuda(), rows(r, (T, 2, D)).cuda()
    w = rows(r, (D,), 1.0).cuda()
    inv = 10000.0 ** (-np.arange(64) / 64)
    first, second = np.arange(64) % 3, np.arange(64) * 3 // 64
    pos = dev(r.integers(0, 3000, (3, T)))
    other = dev(r.integers(0, 3000, (3, T)))
    ropes = [sa.Rope(inv, w, w), sa.Rope(inv * 0.5, w, w), sa.Rope(inv, w, w, weight_offset=1.0), sa.Rope(inv, None, None),
             sa.Rope(inv, w, w, interleaved=True)]

    def kvq(rope=None, **more):
        def go(ctx):
            k4, v4, out = pool4(L), pool4(L), torch.empty_like(q)
            if rope is not None:
                more.update(rope=rope, q=q, q_out=out)
            sa.sa_kvq_append(ctx, L, 0, k, v, k4, v4, start, new, ip, ix, **more)
            return [k4, v4] + [out] * (rope is not None)
        return go

    def bf16(rope, axis=None, p=None):
        def go(ctx):
            out, kp, vp = torch.empty_like(q), pool_bits(None, L, FILL), pool_bits(None, L, FILL)
            if axis is None:
                sa.sa_kv_append_rope(ctx, L, 0, rope, q, k, v, out, kp, vp, start, new, ip, ix, pos=p)
            else:
                sa.sa_kv_append_rope_axes(ctx, L, 0, rope, axis, q, k, v, out, kp, vp, start, new, ip, ix, p)
            return [out, kp, vp]
        return go

    calls = [kvq(), kvq(ropes[0]), kvq(ropes[0], pos=[9, 0, 4000]), kvq(ropes[0], axis=first, axis_pos=pos),
             kvq(ropes[0], axis=second, axis_pos=pos), kvq(ropes[0], axis=second, axis_pos=other),
             kvq(ropes[1], axis=second, axis_pos=pos), kvq(ropes[2], axis=second, axis_pos=pos), kvq(ropes[3]), kvq(ropes[4]),
             bf16(ropes[0]), bf16(ropes[0], first, pos), bf16(ropes[0], second, pos), bf16(ropes[0], second, other),
             bf16(ropes[1], second, pos), bf16(ropes[0], None, [9, 0, 4000]), bf16(ropes[4], first, pos)]
    want = []
    for c in calls:
        fresh = sa.Context(0)
        want.append(c(fresh))
        sa.sa_sync_check(fresh)
    for i in range(len(calls)):                              # the calls do differ
        for j in range(i):
            if len(want[i]) == len(want[j]):
                assert not all(a.shape == b.shape and torch.equal(a, b) for a, b in zip(want[i], want[j])), (i, j)
    ctx = sa.Context(0)
    order = list(range(len(calls)))
    for i in order + order[::-1] + [3, 11, 4, 12, 3, 11, 0, 10, 0]:
        for a, b in zip(calls[i](ctx), want[i]):
            assert torch.equal(a, b), i
    sa.sa_sync_check(ctx)

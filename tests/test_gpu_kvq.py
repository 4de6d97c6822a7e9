"""A cache of 4 bits on the GPU: quantising pages and rows, reading them back, attention over them; rotations on several axes.

References and tolerances: kvq_reference.py.  Whatever is quantised from bf16 rows is compared byte for byte.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2607_00151_amd as sa
from kvq_reference import D, GRID, ROW, attention, page_bytes, page_values, quantise, rows_of, scale_byte
from test_gpu_branches import FILL, bits, close_bf16, dev, lay, pool_bits, rope_reference, rows, tables

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
CANARY = 0xA5            # of untouched bytes


def pool4(L, fill=CANARY):
    return torch.full(sa.kvq_pool_shape(L), fill, dtype=torch.uint8, device="cuda")


def random_pool4(r, L, std=0.5):
    """A pool of quantised rows, and its bytes."""
    x = r.standard_normal((L.num_layers, L.num_slots, L.num_kv_heads, L.page_size, D)) * std
    b = page_bytes(x)
    return torch.from_numpy(b).cuda(), b


# ------------------------------------------------------------------------- pages

def odd_rows(r, shape):
    """bf16 rows of every kind: ordinary, halves between elements, tiny, huge, zeros, infinities, NaN."""
    x = rows(r, shape).view(-1, 32)
    n = len(x)
    x[1::9] = torch.from_numpy(r.choice(np.concatenate([GRID, -GRID, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5, -2.5]]),
                                        (len(x[1::9]), 32)).astype(np.float32)).to(torch.bfloat16)
    for i, scale in enumerate((2.0 ** -140, 2.0 ** -126, 2.0 ** -120, 2.0 ** 120, 0.0, 2.0 ** -130)):
        x[2 + i::41] = (x[2 + i::41].double() * scale).to(torch.bfloat16)
    x[10::97, 5] = float("inf")
    x[11::97, 31] = float("nan")
    x[12::97, 0] = -float("inf")
    x[13::97] = 3.3895313892515355e38          # the largest bf16
    x[14::97, 3] = 7.96875
    assert n > 97
    return x.view(shape)


@pytest.mark.parametrize("heads,page,layers,slots,slots4", [
    ((8, 2), 16, 1, 7, 5), ((32, 8), 16, 2, 20, 33), ((3, 3), 32, 3, 9, 9), ((1, 1), 16, 2, 40, 3), ((5, 1), 32, 1, 6, 11)])
def test_pages_to_4_bits_and_back(heads, page, layers, slots, slots4):
    r = np.random.default_rng(slots)
    L = lay(heads, page, slots, layers)
    shape = (layers, slots, heads[1], page, D)
    k, v = odd_rows(r, shape), odd_rows(r, shape)
    n = min(slots, slots4) - 1
    src, dst = r.permutation(slots)[:n], r.permutation(slots4)[:n]
    k4 = torch.full((layers, slots4, heads[1], page * ROW), CANARY, dtype=torch.uint8, device="cuda")
    v4 = k4.clone()
    ctx = sa.Context(0)
    sa.sa_kvq_pack(ctx, L, k.cuda(), v.cuda(), dev(src), k4, v4, dev(dst))
    sa.sa_sync_check(ctx)
    want = []
    for x, got in ((k, k4), (v, v4)):
        w = np.full(k4.shape, CANARY, np.uint8)
        w[:, dst] = page_bytes(x.double().numpy()[:, src])
        np.testing.assert_array_equal(got.cpu().numpy(), w)
        want.append(w)
    back_k, back_v = pool_bits(r, L, FILL), pool_bits(r, L, FILL)
    to = r.permutation(slots)[:n]
    sa.sa_kvq_unpack(ctx, L, k4, v4, dev(dst), back_k, back_v, dev(to))
    sa.sa_sync_check(ctx)
    for w, got in zip(want, (back_k, back_v)):
        x = page_values(w[:, dst], page)
        g = got.view(torch.bfloat16).cpu().double().numpy()
        np.testing.assert_array_equal(g[:, to], x)
        rest = np.setdiff1d(np.arange(slots), to)
        assert (bits(got)[:, rest] == np.uint16(FILL).view(np.int16)).all()


def test_every_code_under_every_scale_reads_back():
    L = lay((1, 1), 16, 16)
    p = np.zeros((1, 16, 1, 16 * ROW), np.uint8)
    p[..., :1024] = np.arange(1024, dtype=np.int64) % 256              # all pairs of codes in every block
    p[0, :, 0, 1024:] = np.arange(1024, dtype=np.int64).reshape(16, 64) % 256
    k4 = torch.from_numpy(p).cuda()
    k, v = pool_bits(None, L, FILL), pool_bits(None, L, FILL)
    ctx = sa.Context(0)
    s = dev(np.arange(16))
    sa.sa_kvq_unpack(ctx, L, k4, k4, s, k, v, s)
    sa.sa_sync_check(ctx)
    want = page_values(p, 16)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    np.testing.assert_array_equal(k.view(torch.bfloat16).cpu().double().numpy(), want)
    assert torch.equal(k, v)


def test_convert_reports_slots_outside_their_pools_and_does_the_rest():
    r = np.random.default_rng(3)
    L = lay((4, 2), 16, 6)
    x = rows(r, (1, 6, 2, 16, D)).cuda()
    k4, v4 = pool4(lay((4, 2), 16, 4)), pool4(lay((4, 2), 16, 4))
    ctx = sa.Context(0)
    for s, s4 in (([6, 1], [0, 1]), ([-1, 1], [0, 1]), ([0, 1], [4, 1]), ([0, 1], [-1, 1])):
        k4.fill_(CANARY)
        sa.sa_kvq_pack(ctx, L, x, x, dev(s), k4, v4, dev(s4))
        with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
            sa.sa_sync_check(ctx)
        assert (k4[0, 0] == CANARY).all() and (k4[0, 2:] == CANARY).all()
        np.testing.assert_array_equal(k4[0, 1].cpu().numpy(), page_bytes(x[0, 1].double().cpu().numpy()))
    sa.sa_kvq_pack(ctx, L, x, x, None, k4, v4, None)                     # no pages
    sa.sa_sync_check(ctx)


def test_convert_replays_from_a_graph():
    r = np.random.default_rng(4)
    L = lay((8, 2), 16, 12, 2)
    x = [rows(r, (2, 12, 2, 16, D)).cuda() for _ in range(2)]
    k4, v4 = pool4(L), pool4(L)
    back = [torch.zeros_like(x[0]) for _ in range(2)]
    s, s4 = dev(np.arange(12)), dev(np.arange(12)[::-1])
    ctx = sa.Context(0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sa.sa_kvq_pack(ctx, L, *x, s, k4, v4, s4)
        sa.sa_kvq_unpack(ctx, L, k4, v4, s4, *back, s)
    for i in range(3):
        for t in x:
            t.copy_(rows(r, tuple(t.shape)).cuda())
        s4.copy_(dev(r.permutation(12)))
        g.replay()
        torch.cuda.synchronize()
        sa.sa_sync_check(ctx)
        for a, b in zip(x, back):
            np.testing.assert_array_equal(b.double().cpu().numpy(), page_values(page_bytes(a.double().cpu().numpy()), 16))


# ------------------------------------------------------------------------- rows

def places(start, new, indptr, indices, P):
    slot, row = [], []
    for b, (a, n) in enumerate(zip(start, new)):
        for t in range(a, a + n):
            slot.append(int(indices[indptr[b] + t // P]))
            row.append(t % P)
    return slot, row


def row_bytes(pool, slot, row, P):
    """(code bytes [T][Hkv][64], scale bytes [T][Hkv][4]) of one layer's pool at these places."""
    codes = pool[..., :64 * P].reshape(*pool.shape[:-1], P, 64)
    scales = pool[..., 64 * P:].reshape(*pool.shape[:-1], P, 4)
    return codes[slot, :, row], scales[slot, :, row]


def check_rest(pool, layer, slot, row, P):
    """Nothing but the rows of these places was written."""
    b = pool.cpu().numpy().copy()
    b[layer, ..., :64 * P].reshape(*b.shape[1:3], P, 64).transpose(0, 2, 1, 3)[slot, row] = CANARY
    b[layer, ..., 64 * P:].reshape(*b.shape[1:3], P, 4).transpose(0, 2, 1, 3)[slot, row] = CANARY
    assert (b == CANARY).all()


PLAIN = [
    ((32, 8), 16, [0], [1]), ((8, 2), 16, [15, 16, 0, 40, 7], [1, 17, 0, 33, 2]), ((3, 3), 32, [31, 64], [2, 70]),
    ((1, 1), 16, list(range(70)), [1] * 70), ((40, 8), 32, [5, 0, 9], [0, 300, 0]), ((2, 2), 16, [3], [0]),
]


@pytest.mark.parametrize("heads,page,start,new", PLAIN)
def test_append_of_rows_as_they_are(heads, page, start, new):
    r = np.random.default_rng(len(start))
    T, Hkv = sum(new), heads[1]
    pages = [-(-(a + n) // page) for a, n in zip(start, new)]
    L = lay(heads, page, sum(pages) + 3, 2)
    indptr, indices, _ = tables(r, pages, L.num_slots)
    both = odd_rows(r, (max(T, 150), 2 * Hkv, D))[:T]
    k, v = both.cuda().split([Hkv, Hkv], dim=1)
    k4, v4 = pool4(L), pool4(L)
    ctx = sa.Context(0)
    for _ in range(2):
        sa.sa_kvq_append(ctx, L, 1, k, v, k4, v4, start, new, dev(indptr), dev(indices))
    sa.sa_sync_check(ctx)
    slot, row = places(start, new, indptr, indices, page)
    for x, pool in ((both[:, :Hkv], k4), (both[:, Hkv:], v4)):
        if T:
            c, s = quantise(x.double().numpy())
            got_c, got_s = row_bytes(pool.cpu().numpy()[1], slot, row, page)
            np.testing.assert_array_equal(got_c, c[..., 0::2] | (c[..., 1::2] << 4))
            np.testing.assert_array_equal(got_s, s)
        check_rest(pool, 1, slot, row, page)


def close_quantised(codes, scales, ref, size):
    """Quantised rows of fp32 results that are within 2^-16 of `size` of ref: each block's scale is that of a largest
    magnitude within it, each value the nearest element of its scale to a value within it."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], D).astype(np.int64)
    s = scales.astype(np.int64)
    eps = 2.0 ** -16 * size
    mag = np.abs(ref).reshape(*ref.shape[:-1], 4, 32)
    e = eps.reshape(mag.shape)
    low, high = scale_byte(np.maximum(mag - e, 0).max(-1)), scale_byte((mag + e).max(-1))
    assert ((low <= s) & (s <= high)).all()
    unit = 2.0 ** np.repeat(s - 127, 32, axis=-1)
    got = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7] * unit
    y = np.clip(np.abs(ref) / unit, 0, 6)
    nearest = np.abs(GRID[:, None] - y.reshape(1, -1)).min(0).reshape(y.shape) * unit + np.maximum(np.abs(ref) - 6 * unit, 0)
    worst = np.max(np.abs(got - ref) - nearest - 2 * eps - 1e-30)
    assert worst <= 0, worst


AXES = [
    # heads, page, start, new, rot, interleaved, norms, fused, axes, mixed, far, offset
    ((32, 8), 16, [0], [1], 128, False, "qk", True, 3, False, 0, 0.0),
    ((8, 2), 16, [15, 16, 0, 40, 7], [1, 17, 0, 33, 2], 128, False, "qk", True, 3, True, 0, 0.0),
    ((8, 2), 32, [3], [65], 128, True, "", False, 2, False, 5000, 0.0),
    ((40, 8), 16, [31, 64], [2, 1], 96, False, "k", True, 3, True, 1 << 21, 1.0),
    ((7, 7), 32, [1], [40], 32, False, "q", True, 8, True, 2**31 - 100, -0.5),
    ((64, 8), 32, [100], [3], 64, True, "qk", False, 1, False, -100000, 0.0),
    ((1, 1), 16, [0, 1], [5, 6], 0, False, "qk", True, 2, False, 0, 0.0),
    ((16, 1), 16, list(range(70)), [1] * 70, 16, False, "qk", True, 4, True, -2**31, 0.0),
]


def axes_case(heads, page, start, new, rot, inter, norms, fused, axes, mixed, far, offset):
    r = np.random.default_rng(len(start) * 1000 + rot + axes)
    Hq, Hkv = heads
    T = sum(new)
    pages = [-(-(a + n) // page) for a, n in zip(start, new)]
    L = lay(heads, page, sum(pages) + 5, layers=2)
    indptr, indices, _ = tables(r, pages, L.num_slots)
    both = rows(r, (T, Hq + 2 * Hkv, D))
    both[:, :, 3] *= 20
    on_gpu = list(both.cuda().split([Hq, Hkv, Hkv], dim=1))
    if not fused:
        on_gpu = [t.contiguous() for t in on_gpu]
    qw, kw = (1 + 0.3 * rows(r, (D,)).float()).to(torch.bfloat16), rows(r, (D,), 1.0)
    qw, kw = qw if "q" in norms else None, kw if "k" in norms else None
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    axis = np.arange(rot // 2) % axes if mixed else np.arange(rot // 2) * axes // max(rot // 2, 1)
    pos = np.clip(r.integers(-50, 50, (axes, T + 3)) + far, -2**31, 2**31 - 1).astype(np.int64)
    rope = sa.Rope(inv, None if qw is None else qw.cuda(), None if kw is None else kw.cuda(), 1e-5, inter, offset)
    slot, row = places(start, new, indptr, indices, page)
    x = list(both.split([Hq, Hkv, Hkv], dim=1))

    def reference(t, w):
        """rope_reference, whose angle is pos * inv_freq: with one token's positions as part of its frequencies."""
        out = [rope_reference(t[i:i + 1], w, [1], inv * pos[axis, i], 1e-5, inter, offset) for i in range(T)]
        return [np.concatenate(z) for z in zip(*out)]

    return L, indptr, indices, x, on_gpu, qw, kw, rope, axis, pos, slot, row, reference


@pytest.mark.parametrize("case", AXES)
def test_append_rope_axes(case):
    L, indptr, indices, x, on_gpu, qw, kw, rope, axis, pos, slot, row, reference = axes_case(*case)
    start, new, T = case[2], case[3], sum(case[3])
    ctx = sa.Context(0)
    kp, vp = pool_bits(None, L, FILL), pool_bits(None, L, FILL)
    q_out = torch.full((T + 1, case[0][0], D), 7.0, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        sa.sa_kv_append_rope_axes(ctx, L, 1, rope, axis, *on_gpu, q_out, kp, vp, start, new, dev(indptr), dev(indices),
                                  dev(pos))
    sa.sa_sync_check(ctx)
    assert (q_out[T:] == 7).all()
    close_bf16(q_out[:T], *reference(x[0], qw))
    close_bf16(kp.view(torch.bfloat16)[1].permute(0, 2, 1, 3)[slot, row], *reference(x[1], kw))
    want = np.full(kp.shape, np.uint16(FILL).view(np.int16))
    want[1].transpose(0, 2, 1, 3)[slot, row] = bits(x[2].contiguous())
    np.testing.assert_array_equal(bits(vp), want)
    keys = bits(kp).copy()
    keys[1].transpose(0, 2, 1, 3)[slot, row] = np.uint16(FILL).view(np.int16)
    assert (keys == np.uint16(FILL).view(np.int16)).all()


@pytest.mark.parametrize("case", AXES)
def test_append_of_rotated_rows(case):
    L, indptr, indices, x, on_gpu, qw, kw, rope, axis, pos, slot, row, reference = axes_case(*case)
    page, start, new, T = case[1], case[2], case[3], sum(case[3])
    ctx = sa.Context(0)
    k4, v4 = pool4(L), pool4(L)
    q_out = torch.full((T + 1, case[0][0], D), 7.0, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        sa.sa_kvq_append(ctx, L, 1, on_gpu[1], on_gpu[2], k4, v4, start, new, dev(indptr), dev(indices), rope=rope,
                         q=on_gpu[0], q_out=q_out, axis=axis, axis_pos=dev(pos))
    sa.sa_sync_check(ctx)
    assert (q_out[T:] == 7).all()
    close_bf16(q_out[:T], *reference(x[0], qw))
    close_quantised(*row_bytes(k4.cpu().numpy()[1], slot, row, page), *reference(x[1], kw))
    c, s = quantise(x[2].double().numpy())
    got_c, got_s = row_bytes(v4.cpu().numpy()[1], slot, row, page)
    np.testing.assert_array_equal(got_c, c[..., 0::2] | (c[..., 1::2] << 4))
    np.testing.assert_array_equal(got_s, s)
    check_rest(k4, 1, slot, row, page)
    check_rest(v4, 1, slot, row, page)
    # keys and values alone give the same bytes
    again = pool4(L), pool4(L)
    sa.sa_kvq_append(ctx, L, 1, on_gpu[1], on_gpu[2], *again, start, new, dev(indptr), dev(indices), rope=rope,
                     axis=axis, axis_pos=dev(pos))
    sa.sa_sync_check(ctx)
    assert torch.equal(again[0], k4) and torch.equal(again[1], v4)


@pytest.mark.parametrize("inter,rot,norm", [(False, 128, True), (True, 64, False)])
def test_rotated_keys_are_the_elements_of_the_64_bit_results(inter, rot, norm):
    """Millions of values, none on the other side of a tie: the reference and the kernel are off by some 2^-40, and
    of 4 million values about one is as near as 2^-22 to a tie."""
    r = np.random.default_rng(23)
    L = lay((8, 8), 16, 256)
    T = 16 * L.num_slots
    k = rows(r, (T, 8, D))
    w = (1 + 0.2 * rows(r, (D,)).float()).to(torch.bfloat16) if norm else None
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    indices = r.permutation(L.num_slots)
    k4, v4 = pool4(L), pool4(L)
    ctx = sa.Context(0)
    rope = sa.Rope(inv, None, None if w is None else w.cuda(), 1e-5, inter)
    sa.sa_kvq_append(ctx, L, 0, k.cuda(), k.cuda(), k4, v4, [0], [T], dev([0, L.num_slots]), dev(indices), rope=rope, pos=[777])
    sa.sa_sync_check(ctx)
    ref, _ = rope_reference(k, w, np.arange(777, 777 + T), inv, 1e-5, inter, 0.0)
    c, s = quantise(ref)
    t = np.arange(T)
    codes, scales = row_bytes(k4.cpu().numpy()[0], indices[t // 16], t % 16, 16)
    np.testing.assert_array_equal(scales, s)
    np.testing.assert_array_equal(codes, c[..., 0::2] | (c[..., 1::2] << 4))


def test_axes_that_agree_give_the_bits_of_one_position():
    r = np.random.default_rng(8)
    L = lay((8, 2), 16, 12)
    T, start, new = 50, [3, 17], [30, 20]
    q, k, v = rows(r, (T, 8, D)).cuda(), rows(r, (T, 2, D)).cuda(), rows(r, (T, 2, D)).cuda()
    ip, ix = dev([0, 3, 6]), dev([4, 0, 7, 9, 1, 2])
    w = rows(r, (D,)).cuda()
    ctx = sa.Context(0)
    pos0 = [1000, 70000]
    pos = np.concatenate([p + np.arange(n) for p, n in zip(pos0, new)])
    for rot, inter in ((128, False), (64, False), (128, True)):
        rope = sa.Rope(10000.0 ** (-np.arange(rot // 2) * 2 / rot), w, w, interleaved=inter)
        one = [torch.empty_like(q), pool_bits(r, L, FILL), pool_bits(r, L, FILL)]
        several = [torch.empty_like(q), pool_bits(r, L, FILL), pool_bits(r, L, FILL)]
        sa.sa_kv_append_rope(ctx, L, 0, rope, q, k, v, *one, start, new, ip, ix, pos=pos0)
        sa.sa_kv_append_rope_axes(ctx, L, 0, rope, np.arange(rot // 2) % 3, q, k, v, *several, start, new, ip, ix,
                                  dev(np.stack([pos] * 3)))
        sa.sa_sync_check(ctx)
        for a, b in zip(one, several):
            assert torch.equal(a, b)
        k4, v4, k5, v5, o4, o5 = pool4(L), pool4(L), pool4(L), pool4(L), torch.empty_like(q), torch.empty_like(q)
        sa.sa_kvq_append(ctx, L, 0, k, v, k4, v4, start, new, ip, ix, rope=rope, q=q, q_out=o4, pos=pos0)
        sa.sa_kvq_append(ctx, L, 0, k, v, k5, v5, start, new, ip, ix, rope=rope, q=q, q_out=o5,
                         axis=np.arange(rot // 2) % 3, axis_pos=dev(np.stack([pos] * 3)))
        sa.sa_sync_check(ctx)
        assert torch.equal(k4, k5) and torch.equal(v4, v5) and torch.equal(o4, o5)


@pytest.mark.parametrize("axes", [0, 3])
def test_appends_of_many_tokens(axes):
    """More bytes than the Infinity Cache, against the same rows in pieces."""
    heads, T = (32, 8), 14001
    L = lay(heads, 16, -(-T // 16) + 1)
    g = torch.Generator(device="cuda").manual_seed(3)
    both = (torch.randn((T, 48, D), generator=g, device="cuda") * 0.5).to(torch.bfloat16)
    q, k, v = both.split([32, 8, 8], dim=1)
    ip, ix = dev([0, L.num_slots]), dev(np.random.default_rng(3).permutation(L.num_slots))
    w = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    rope, ctx = sa.Rope(10000.0 ** (-np.arange(64) / 64), w, w), sa.Context(0)
    axis = np.arange(64) % 3
    pos = torch.stack([torch.arange(T) // 64, torch.arange(T) // 8 % 8, torch.arange(T) % 8]).to(torch.int32).cuda()
    pools = [pool4(L) for _ in range(4)]
    q_out, q2 = (torch.empty((T, 32, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def go(out, pk, pv, a, n):
        more = dict(axis=axis, axis_pos=pos[:, a:a + n].contiguous()) if axes else {}
        sa.sa_kvq_append(ctx, L, 0, k[a:], v[a:], pk, pv, [a], [n], ip, ix, rope=rope, q=q[a:], q_out=out[a:], **more)

    go(q_out, pools[0], pools[1], 0, T)
    for a in range(0, T, 3500):
        go(q2, pools[2], pools[3], a, min(3500, T - a))
    sa.sa_sync_check(ctx)
    assert torch.equal(q_out, q2) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def test_append_reports_bad_pages_and_writes_the_rest():
    r = np.random.default_rng(6)
    L = lay((4, 2), 16, 8)
    q, k, v = rows(r, (3, 4, D)).cuda(), rows(r, (3, 2, D)).cuda(), rows(r, (3, 2, D)).cuda()
    k4, v4, out = pool4(L), pool4(L), torch.zeros_like(q)
    ctx = sa.Context(0)
    sa.sa_kvq_append(ctx, L, 0, k, v, k4, v4, [0, 16, 1], [1, 1, 1], dev([0, 1, 2, 3]), dev([8, 3, 5]), rope=sa.Rope(),
                     q=q, q_out=out)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    assert torch.equal(out, q)
    for x, pool in ((k, k4), (v, v4)):
        c, s = row_bytes(pool.cpu().numpy()[0], [5], [1], 16)
        want = quantise(x[2:].double().cpu().numpy())
        np.testing.assert_array_equal(c, want[0][..., 0::2] | (want[0][..., 1::2] << 4))
        np.testing.assert_array_equal(s, want[1])
        check_rest(pool, 0, [5], [1], 16)


# ------------------------------------------------------------------------- attention

def attn_case(seed, heads, page, q_len, kv_len, causal, scale=D ** -0.5, std=0.5, layers=1, spare=3, change=None, q_change=None):
    """Inputs, outputs and references of one call; change(k, v bytes of the pools, tables) edits the cache first."""
    r = np.random.default_rng(seed)
    pages = [-(-n // page) for n in kv_len]
    L = lay(heads, page, sum(pages) + spare, layers)
    indptr, indices, _ = tables(r, pages, L.num_slots)
    _, k = random_pool4(r, L, std)
    _, v = random_pool4(r, L, std)
    # rows behind the last one of each sequence: bytes of anything, NaN scales among them
    for b, n in enumerate(kv_len):
        if n % page:
            last = indices[indptr[b + 1] - 1]
            for p in (k, v):
                codes = p[..., :64 * page].reshape(*p.shape[:-1], page, 64)
                scales = p[..., 64 * page:].reshape(*p.shape[:-1], page, 4)
                codes[:, last, :, n % page:] = 0xFF
                scales[:, last, :, n % page:] = 0xFF
    if change:
        change(k, v, indptr, indices)
    T = sum(q_len)
    q = rows(r, (T, heads[0], D), std)
    if q_change:
        q_change(q)
    k4, v4 = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    o = torch.full((T + 1, heads[0], D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 1, heads[0]), 7.0, device="cuda")
    ctx = sa.Context(0)
    for _ in range(2):
        sa.sa_kvq_attn(ctx, L, layers - 1, q.cuda(), k4, v4, q_len, kv_len, dev(indptr), dev(indices), scale, o, lse,
                       causal=causal)
    sa.sa_sync_check(ctx)
    assert (o[T:] == 7).all() and (lse[T:] == 7).all()
    return L, indptr, indices, k, v, q, o[:T], lse[:T]


def check_attn(case, heads, page, q_len, kv_len, causal, scale=D ** -0.5):
    L, indptr, indices, k, v, q, o, lse = case
    t0 = 0
    for b, (n, kv) in enumerate(zip(q_len, kv_len)):
        if n == 0:
            continue
        ref = attention(q[t0:t0 + n], rows_of(k[-1], indptr, indices, b, kv, page),
                        rows_of(v[-1], indptr, indices, b, kv, page), scale, causal)
        got, got_l = o[t0:t0 + n].double().cpu(), lse[t0:t0 + n].double().cpu()
        if kv == 0:
            assert (got == 0).all() and (got_l == -np.inf).all()
        else:
            worst = ((got - ref[0]).abs() / ref[2]).max().item()
            assert worst <= 1.0, (b, worst)
            worst = ((got_l - ref[1]).abs() / ref[3]).max().item()
            assert worst <= 1.0, (b, worst)
        t0 += n


ATTN = [
    # heads, page, q_len, kv_len, causal
    ((32, 8), 16, [1], [1], True),
    ((32, 8), 16, [1, 1, 1, 0, 1], [1000, 17, 64, 5, 4096], True),
    ((8, 2), 16, [1, 1], [63, 65], True),
    ((8, 2), 32, [3, 1, 2], [3, 129, 700], True),
    ((4, 4), 16, [1, 7, 40], [200, 300, 41], True),
    ((7, 7), 32, [16, 17, 33], [16, 18, 1000], True),
    ((64, 8), 32, [2, 5], [2000, 300], True),
    ((40, 8), 16, [3, 4, 13], [99, 1500, 13], True),
    ((16, 1), 16, [1, 2, 4, 5], [500, 501, 502, 503], True),
    ((65, 1), 16, [1, 2], [300, 77], True),
    ((32, 8), 16, [70], [2100], True),
    ((32, 8), 16, [128, 1, 5], [128, 3000, 64], True),
    ((2, 1), 32, [200, 129], [200, 1337], True),
    ((8, 2), 16, [1, 1, 3, 4], [0, 1, 0, 500], False),
    ((32, 8), 16, [1] * 6, [0, 640, 1, 0, 33, 2000], False),
    ((4, 2), 32, [90, 3, 0], [10, 1700, 20], False),
    ((64, 8), 32, [33, 1], [257, 0], False),
    ((1, 1), 16, [300], [1], False),
    ((8, 2), 16, [1] * 80, [1 + 13 * i for i in range(80)], True),
]


@pytest.mark.parametrize("i", range(len(ATTN)))
def test_attention(i):
    heads, page, q_len, kv_len, causal = ATTN[i]
    check_attn(attn_case(i, *ATTN[i], layers=1 + i % 2), heads, page, q_len, kv_len, causal)


@pytest.mark.parametrize("heads,page,q,kv,causal", [((8, 2), 16, [1, 1], [40000, 31001], True), ((32, 8), 16, [1], [9000], False),
                                                    ((2, 1), 32, [40], [20011], True), ((16, 1), 16, [6], [30000], True),
                                                    ((16, 1), 16, [1, 1], [60000, 1], True), ((4, 4), 32, [1] * 3, [70000, 64, 9000], False),
                                                    ((16, 4), 32, [2, 30, 1, 7, 14], [9000, 6000, 20000, 77, 12345], True)])
def test_attention_over_long_caches(heads, page, q, kv, causal):
    check_attn(attn_case(90, heads, page, q, kv, causal), heads, page, q, kv, causal)


@pytest.mark.parametrize("scale,std", [(1.0, 1.0), (1e-3, 0.5), (D ** -0.5, 4.0), (2.0, 0.5)])
def test_attention_with_other_scores(scale, std):
    args = ((8, 2), 16, [1, 20], [700, 1111], True)
    check_attn(attn_case(91, *args, scale=scale, std=std), *args, scale=scale)


def test_a_key_that_outweighs_many():
    """One key far above thousands of small ones: they keep their weight, all of it in one tile or not."""
    kv = 6000

    def change(k, v, indptr, indices):
        x = np.zeros((1, 2, 16, D))
        x[:, :, 5] = 1.0
        k[:] = 0
        k[0, indices[100]] = page_bytes(x)[0]

    def q_change(q):
        q[:] = 0.5
    args = ((4, 2), 16, [1, 3], [kv, 77], True)
    case = attn_case(92, *args, scale=8.0 / 64, change=change, q_change=q_change)
    check_attn(case, *args, scale=8.0 / 64)


def test_queries_of_all_sizes():
    """Dims of very different size in one block, and blocks of very different size, as outlier dims make them."""
    def q_change(q):
        f = torch.ones(D)
        f[3], f[40:44], f[64:96], f[100] = 300.0, 1e-3, 1e-6, 1e4
        q.copy_((q.float() * f).to(torch.bfloat16))
    args = ((8, 2), 16, [2, 30], [300, 900], True)
    check_attn(attn_case(93, *args, q_change=q_change, scale=1e-4), *args, scale=1e-4)


@pytest.mark.parametrize("heads,page,q,kv", [((8, 2), 16, [1, 6], [900, 1500]), ((8, 2), 16, [20, 12], [1100, 640]),
                                             ((32, 4), 32, [30, 7], [3000, 1290])])
@pytest.mark.parametrize("slope", [0.5, 8.0, -8.0])
def test_scores_that_rise_or_fall_along_the_keys(heads, page, q, kv, slope):
    """Offsets that every few tiles outgrow, every one, or none behind the first."""
    def change(k, v, indptr, indices):
        for b, n in enumerate(kv):
            slots = indices[indptr[b]:indptr[b + 1]]
            x = np.zeros((len(slots), heads[1], page, D))
            x += (slope * np.arange(len(slots) * page) / 64).reshape(-1, 1, page, 1)
            k[-1, slots] = page_bytes(x * (1 + 0.25 * np.arange(D) / D))

    def q_change(x):
        x.copy_((x.float() + 0.5).to(torch.bfloat16))
    args = (heads, page, q, kv, True)
    check_attn(attn_case(95, *args, change=change, q_change=q_change, std=0.25), *args)


@pytest.mark.parametrize("power", [100, -100])
@pytest.mark.parametrize("heads,page,q,kv", [((8, 2), 16, [1, 3, 9], [300, 65, 900]), ((8, 2), 32, [12, 40], [500, 700])])
def test_scales_far_from_one(heads, page, q, kv, power):
    """Keys and values times 2^100 or 2^-100, queries by the other: scores are what they were."""
    def change(k, v, indptr, indices):
        for pool in (k, v):
            scales = pool[..., 64 * page:]
            scales[scales != 255] += np.uint8(power % 256)

    def q_change(x):
        x.copy_((x.float() * 2.0 ** -power).to(torch.bfloat16))
    args = (heads, page, q, kv, True)
    check_attn(attn_case(94, *args, change=change, q_change=q_change), *args)


# ---- values that are not finite

def scale_at(pool, layer, slot, head, row, block, P):
    return pool[layer, slot, head, 64 * P:].reshape(P, 4)[row, block:block + 1]


@pytest.mark.parametrize("heads,page,q,kv,at,causal", [
    ((8, 2), 16, 1, 300, 299, True), ((8, 2), 16, 6, 300, 297, True), ((32, 8), 32, 40, 200, 170, True),
    ((8, 2), 16, 70, 70, 3, True), ((4, 2), 16, 9, 130, 64, False), ((2, 1), 16, 100, 5000, 4950, True)])
@pytest.mark.parametrize("which", ["key", "value"])
def test_a_nan_block_reaches_the_rows_that_see_it(heads, page, q, kv, at, causal, which):
    def change(k, v, indptr, indices):
        scale_at(k if which == "key" else v, 0, indices[at // page], 0, at % page, 2, page)[:] = 255
    L, indptr, indices, k, v, qs, o, lse = attn_case(94, heads, page, [q], [kv], causal, change=change)
    G = heads[0] // heads[1]
    sees = np.array([not causal or kv - q + i >= at for i in range(q)])
    hit = np.zeros(o.shape, bool)
    hit[np.ix_(sees, np.arange(G), np.arange(D) if which == "key" else np.arange(64, 96))] = True
    np.testing.assert_array_equal(np.isnan(o.float().cpu().numpy()), hit)
    lhit = np.zeros(lse.shape, bool)
    if which == "key":
        lhit[np.ix_(sees, np.arange(G))] = True
    np.testing.assert_array_equal(np.isnan(lse.cpu().numpy()), lhit)
    # the other rows are as with a cache that holds zeros there
    pool = k if which == "key" else v
    pool[0, indices[at // page], 0, :64 * page].reshape(page, 64)[at % page, 32:48] = 0
    scale_at(pool, 0, indices[at // page], 0, at % page, 2, page)[:] = 0
    ref = attention(qs, rows_of(k[0], indptr, indices, 0, kv, page), rows_of(v[0], indptr, indices, 0, kv, page), D ** -0.5, causal)
    off = ((o.double().cpu() - ref[0]).abs() / ref[2]).numpy()
    assert (off[~hit] <= 1).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("heads,q,kv", [((8, 2), [1, 1], [300, 20]), ((32, 8), [9, 30], [100, 2000])])
def test_a_query_that_is_not_finite_stays_in_its_row(heads, q, kv, value):
    def q_change(x):
        x[0, 1, 77] = value
    L, indptr, indices, k, v, qs, o, lse = attn_case(95, heads, 16, q, kv, True, q_change=q_change)
    want = np.zeros(lse.shape, bool)
    want[0, 1] = True
    np.testing.assert_array_equal(np.isnan(lse.cpu().numpy()), want)
    np.testing.assert_array_equal(np.isnan(o.float().cpu().numpy()).all(-1), want)
    np.testing.assert_array_equal(np.isnan(o.float().cpu().numpy()).any(-1), want)


def test_missing_pages_read_as_zeros_and_are_reported():
    r = np.random.default_rng(96)
    L = lay((4, 2), 16, 8)
    k4, k = random_pool4(r, L)
    v4, v = random_pool4(r, L)
    q = rows(r, (3, 4, D))
    o, lse = torch.empty((3, 4, D), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 4), device="cuda")
    ctx = sa.Context(0)
    ip, ix = [0, 2, 4, 5], [1, 8, -1, 3, 2]                # a slot beyond the pool, a negative one, a table too short
    sa.sa_kvq_attn(ctx, L, 0, q.cuda(), k4, v4, [1, 1, 1], [30, 32, 40], dev(ip), dev(ix), D ** -0.5, o, lse)
    with pytest.raises(sa.SaError, match="SA_ERR_RANGE"):
        sa.sa_sync_check(ctx)
    for b, (kv, good) in enumerate(((30, {0: 1}), (32, {1: 3}), (40, {0: 2}))):
        rows_k, rows_v = np.zeros((2, 48, D)), np.zeros((2, 48, D))
        for p, s in good.items():
            rows_k[:, 16 * p:16 * p + 16], rows_v[:, 16 * p:16 * p + 16] = page_values(k[0, s], 16), page_values(v[0, s], 16)
        ref = attention(q[b:b + 1], rows_k[:, :kv], rows_v[:, :kv], D ** -0.5, True)
        assert ((o[b:b + 1].double().cpu() - ref[0]).abs() <= ref[2]).all()
        assert ((lse[b:b + 1].double().cpu() - ref[1]).abs() <= ref[3]).all()


def test_attention_gives_the_same_bits_again_and_on_another_stream():
    args = ((32, 8), 16, [1, 4, 1], [500, 90, 300], True)
    L, indptr, indices, k, v, q, o, lse = attn_case(97, *args)
    k4, v4 = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    again = torch.empty_like(o)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ctx = sa.Context(0)
    qd, ip, ix = q.cuda(), dev(indptr), dev(indices)
    side.wait_stream(torch.cuda.current_stream())
    sa.sa_kvq_attn(ctx, L, 0, qd, k4, v4, *args[2:4], ip, ix, D ** -0.5, again, stream=side)
    side.synchronize()
    assert torch.equal(o, again)


def test_two_contexts_at_once_on_two_streams():
    """Launches that join their own parts, and mixed ones, overlapping from two contexts: each as when alone."""
    cases = [((32, 8), 16, [1] * 4, [3000, 1000, 4096, 70], True), ((32, 8), 16, [1, 40], [6000, 5000], True)]
    made = []
    for i, args in enumerate(cases):
        L, indptr, indices, k, v, q, o, lse = attn_case(110 + i, *args)
        made.append((L, args, q.cuda(), torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), dev(indptr), dev(indices), o,
                     [torch.empty_like(o) for _ in range(20)], sa.Context(0), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for n in range(20):
        for L, args, q, k4, v4, ip, ix, o, outs, ctx, side in made:
            sa.sa_kvq_attn(ctx, L, 0, q, k4, v4, args[2], args[3], ip, ix, D ** -0.5, outs[n], stream=side)
    torch.cuda.synchronize()
    for L, args, q, k4, v4, ip, ix, o, outs, ctx, side in made:
        sa.sa_sync_check(ctx, side)
        for out in outs:
            assert torch.equal(out, o)


def test_reserved_contexts_and_timing_events():
    args = ((32, 8), 16, [1, 1, 33], [5000, 900, 4000], True)
    L, indptr, indices, k, v, q, o, lse = attn_case(112, *args)
    k4, v4, qd, ip, ix = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), q.cuda(), dev(indptr), dev(indices)
    ctx = sa.Context(0)
    sa.sa_reserve(ctx, 1 << 20, 1 << 24)
    free = torch.cuda.mem_get_info()[0]
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    stop.record()
    torch.cuda.synchronize()
    sa.sa_set_kernel_events(ctx, sa.TIMED_ATTN, start.cuda_event, stop.cuda_event)
    out = torch.empty_like(o)
    sa.sa_kvq_attn(ctx, L, 0, qd, k4, v4, *args[2:4], ip, ix, D ** -0.5, out)
    torch.cuda.synchronize()
    assert 0 < start.elapsed_time(stop) < 50
    assert torch.cuda.mem_get_info()[0] == free
    assert torch.equal(out, o)


def test_pools_beyond_4_gib():
    """Slots whose bytes lie past 2^32 of the pool."""
    heads, page = (8, 8), 32
    L = lay(heads, page, 260000, 1)                        # 4.5 GB a pool
    k4 = torch.zeros(sa.kvq_pool_shape(L), dtype=torch.uint8, device="cuda")
    v4 = torch.zeros_like(k4)
    r = np.random.default_rng(98)
    slots = np.array([259999, 3, 250001, 246725])
    xk, xv = (rows(r, (1, 4, 8, page, D)) for _ in range(2))
    near = lay(heads, page, 4, 1)
    ctx = sa.Context(0)
    sa.sa_kvq_pack(ctx, near, xk.cuda(), xv.cuda(), dev(np.arange(4)), k4, v4, dev(slots))
    q, kv = rows(r, (3, 8, D)), 120
    new = rows(r, (3, 8, D))
    ip, ix = dev([0, 4]), dev(slots)
    sa.sa_kvq_append(ctx, L, 0, new.cuda(), new.cuda(), k4, v4, [117], [3], ip, ix)
    o = torch.empty((3, 8, D), dtype=torch.bfloat16, device="cuda")
    sa.sa_kvq_attn(ctx, L, 0, q.cuda(), k4, v4, [3], [kv], ip, ix, D ** -0.5, o)
    back = [pool_bits(None, near, FILL) for _ in range(2)]
    sa.sa_kvq_unpack(ctx, near, k4, v4, dev(slots), *back, dev(np.arange(4)))
    sa.sa_sync_check(ctx)
    full = []
    for x in (xk, xv):
        x = x[0].double().numpy().transpose(1, 0, 2, 3).reshape(8, -1, D).copy()
        x[:, 117:120] = new.double().numpy().transpose(1, 0, 2)
        full.append(page_values(page_bytes(x[:, :, None]), 1).reshape(8, -1, D))
    got = back[0].view(torch.bfloat16)[0].double().cpu().numpy().transpose(1, 0, 2, 3).reshape(8, -1, D)
    np.testing.assert_array_equal(got, full[0])
    ref = attention(q, full[0][:, :kv], full[1][:, :kv], D ** -0.5, True)
    assert ((o.double().cpu() - ref[0]).abs() <= ref[2]).all()


def test_planned_calls_refuse_capture_and_leave_the_context_usable():
    args = ((8, 2), 16, [1], [50], True)
    L, indptr, indices, k, v, q, o, lse = attn_case(99, *args)
    k4, v4, qd, ip, ix = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), q.cuda(), dev(indptr), dev(indices)
    x, out, ctx = rows(np.random.default_rng(1), (1, 2, D)).cuda(), torch.empty_like(o), sa.Context(0)
    pool = pool_bits(None, L, 0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        mark = torch.zeros(4, device="cuda")
        for call in (lambda: sa.sa_kvq_attn(ctx, L, 0, qd, k4, v4, [1], [50], ip, ix, 0.1, out),
                     lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, v4, [50], [1], ip, ix),
                     lambda: sa.sa_kv_append_rope_axes(ctx, L, 0, sa.Rope(), [], qd, x, x, out, pool, pool, [50], [1], ip,
                                                       ix, ix[None])):
            with pytest.raises(sa.SaError, match="SA_ERR_UNSUPPORTED"):
                call()
        mark += 1
    g.replay()
    sa.sa_kvq_attn(ctx, L, 0, qd, k4, v4, [1], [50], ip, ix, D ** -0.5, out)
    sa.sa_sync_check(ctx)
    assert torch.equal(out, o)


def test_a_context_of_text_and_images_from_prompt_to_decode():
    """The calls together: a prompt's rows, rotated on three axes, into 4 bits; its attention; tokens one by one; the
    cache to bf16 and back; the bf16 attention over what it stands for; cross attention to the same rows."""
    r = np.random.default_rng(100)
    heads, page, T, steps = (8, 2), 16, 75, 5
    Hq, Hkv = heads
    n_pages = -(-(T + steps) // page)
    L = lay(heads, page, n_pages + 4)
    indptr, indices, _ = tables(r, [n_pages], L.num_slots)
    ip, ix = dev(indptr), dev(indices)
    x = rows(r, (T + steps, Hq + 2 * Hkv, D))
    pos = np.stack([np.arange(T + steps) // 16, np.arange(T + steps) // 4 % 4, np.arange(T + steps) % 4])
    axis = np.arange(64) * 3 // 64
    w = (1 + 0.2 * rows(r, (D,)).float()).to(torch.bfloat16).cuda()
    rope, ctx = sa.Rope(10000.0 ** (-np.arange(64) / 64), w, w), sa.Context(0)
    k4, v4 = pool4(L, 255), pool4(L, 255)
    on = x.cuda()
    turned = torch.empty((T + steps, Hq, D), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(turned)
    lse = torch.empty((T + steps, Hq), device="cuda")
    for a, n in [(0, T)] + [(T + i, 1) for i in range(steps)]:
        q, k, v = on[a:a + n].split([Hq, Hkv, Hkv], dim=1)
        sa.sa_kvq_append(ctx, L, 0, k, v, k4, v4, [a], [n], ip, ix, rope=rope, q=q, q_out=turned[a:a + n], axis=axis,
                         axis_pos=dev(pos[:, a:a + n]))
        sa.sa_kvq_attn(ctx, L, 0, turned[a:a + n], k4, v4, [n], [a + n], ip, ix, D ** -0.5, o[a:a + n], lse[a:a + n])
    sa.sa_sync_check(ctx)
    kh, vh = k4.cpu().numpy(), v4.cpu().numpy()
    full = [rows_of(p[0], indptr, indices, 0, T + steps, page) for p in (kh, vh)]
    ref = attention(turned.cpu(), *full, D ** -0.5, True)
    assert ((o.double().cpu() - ref[0]).abs() <= ref[2]).all() and ((lse.double().cpu() - ref[1]).abs() <= ref[3]).all()
    # the same cache in bf16: the segment attention's own roundings are the same
    kp, vp = pool_bits(None, L, 0), pool_bits(None, L, 0)
    mine = dev(indices)
    sa.sa_kvq_unpack(ctx, L, k4, v4, mine, kp, vp, mine)
    o16 = torch.empty_like(o)
    sa.sa_segment_prefill_attn(ctx, L, 0, turned, kp, vp, [T + steps], [T + steps], ip, ix, D ** -0.5, o16)
    sa.sa_sync_check(ctx)
    assert ((o16.double() - o.double()).cpu().abs() <= 2 * ref[2]).all()
    again = pool4(L, 255), pool4(L, 255)
    sa.sa_kvq_pack(ctx, L, kp, vp, mine, *again, mine)
    oc, lc = torch.empty_like(o), torch.empty_like(lse)
    sa.sa_kvq_attn(ctx, L, 0, turned, *again, [T + steps], [T + steps], ip, ix, D ** -0.5, oc, lc, causal=False)
    sa.sa_sync_check(ctx)
    ref = attention(turned.cpu(), *full, D ** -0.5, False)
    assert ((oc.double().cpu() - ref[0]).abs() <= ref[2]).all() and ((lc.double().cpu() - ref[1]).abs() <= ref[3]).all()


# ------------------------------------------------------------------------- the binding

def test_binding_refuses_other_types_and_sizes():
    L, ctx = lay((4, 2), 16, 4), sa.Context(0)
    k4 = pool4(L)
    x, q, t = torch.zeros((1, 2, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 4, D), dtype=torch.bfloat16, device="cuda"), dev([0, 1])
    kp = pool_bits(None, L, 0)
    rope = sa.Rope(np.ones(8))
    bad = [
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4.view(torch.int8), k4, [0], [1], t, t),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4[0, :3], k4, [0], [1], t, t),
        lambda: sa.sa_kvq_append(ctx, L, 0, x.float(), x, k4, k4, [0], [1], t, t),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, axis=[0], axis_pos=t[None]),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, rope=rope, axis=[0] * 8),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, rope=rope, axis=[0] * 7, axis_pos=t[None]),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, rope=rope, axis=[0] * 8, axis_pos=t),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, rope=rope, axis=[0] * 8, axis_pos=t[None].long()),
        lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [0], [1], t, t, rope=rope, q=q, q_out=q.float()),
        lambda: sa.sa_kv_append_rope_axes(ctx, L, 0, rope, [0] * 8, q, x, x, q, kp, kp, [0], [1], t, t, t[None][:, :0]),
        lambda: sa.sa_kvq_pack(ctx, L, kp, kp, t, k4, k4, t[:1]),
        lambda: sa.sa_kvq_pack(ctx, L, kp, kp, t, k4.view(-1)[:-16], k4, t),
        lambda: sa.sa_kvq_unpack(ctx, L, k4, k4[:, :2], t, kp, kp, t),
        lambda: sa.sa_kvq_attn(ctx, L, 0, q, kp, k4, [1], [1], t, t, 1.0, q),
        lambda: sa.sa_kvq_attn(ctx, L, 0, q, k4, k4, [1], [1], t, t, 1.0, q.float()),
        lambda: sa.sa_kvq_attn(ctx, L, 0, q, k4, k4, [1], [1, 1], t, t, 1.0, q),
        lambda: sa.sa_kvq_attn(ctx, L, 0, q.cpu(), k4, k4, [1], [1], t, t, 1.0, q),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)


DEBUG_CODE = """
import numpy as np, torch, paper_2607_00151_amd as sa
L = sa.Layout(num_q_heads=2, num_kv_heads=1, head_dim=128, page_size=16, num_layers=1, num_slots=4)
ctx = sa.Context(0)
i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
k = torch.zeros((1, 4, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
k4 = torch.zeros(sa.kvq_pool_shape(L), dtype=torch.uint8, device="cuda")
def refused(name, call):
    try:
        call()
    except sa.SaError as e:
        assert e.name == name, (name, e)
    else:
        raise AssertionError("not refused: " + name)
refused("SA_ERR_RANGE", lambda: sa.sa_kvq_pack(ctx, L, k, k, i32([0, 4]), k4, k4, i32([0, 1])))
refused("SA_ERR_RANGE", lambda: sa.sa_kvq_unpack(ctx, L, k4, k4, i32([0, -1]), k, k, i32([0, 1])))
refused("SA_ERR_OVERLAP", lambda: sa.sa_kvq_pack(ctx, L, k, k, i32([0, 1]), k4, k4, i32([2, 2])))
refused("SA_ERR_OVERLAP", lambda: sa.sa_kvq_unpack(ctx, L, k4, k4, i32([0, 1]), k, k, i32([2, 2])))
sa.sa_kvq_pack(ctx, L, k, k, i32([1, 1]), k4, k4, i32([2, 3]))
x = torch.zeros((2, 1, 128), dtype=torch.bfloat16, device="cuda")
refused("SA_ERR_OVERLAP", lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [3, 3], [1, 1], i32([0, 1, 2]), i32([2, 2])))
refused("SA_ERR_RANGE", lambda: sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [3, 3], [1, 1], i32([0, 1, 2]), i32([2, 4])))
sa.sa_kvq_append(ctx, L, 0, x, x, k4, k4, [3, 4], [1, 1], i32([0, 1, 2]), i32([2, 2]))
sa.sa_sync_check(ctx)
print("ALL OK")
"""


def test_debug_checks():
    r = subprocess.run([sys.executable, "-u", "-c", DEBUG_CODE], env=dict(os.environ, SA_DEBUG="1"), capture_output=True,
                       text=True, timeout=100, cwd=ROOT)
    assert r.returncode == 0 and "ALL OK" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]

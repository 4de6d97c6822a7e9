"""The 4-bit cache and attention over it, defined in numpy and float64 torch."""
import math

import numpy as np
import torch

D, ROW = 128, 68
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def scale_byte(amax):
    """The block's scale byte from its largest magnitude (float64; not finite: 255)."""
    with np.errstate(invalid="ignore"):
        m, e = np.frexp(np.where(np.isfinite(amax), amax, 1.0))      # m in [0.5, 1)
    s = e - 1 + (m >= 0.875) + 127 - 2
    return np.where(np.isfinite(amax), np.clip(np.where(amax > 0, s, 1), 1, 252), 255).astype(np.int64)


def quantise(x):
    """(codes [..., 128], scale bytes [..., 4]) of rows of finite or other values."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], 4, 32)
    amax = np.where(np.isfinite(b).all(-1), np.abs(np.where(np.isfinite(b), b, 0)).max(-1), np.inf)
    s = scale_byte(amax)
    y = np.abs(np.where(np.isfinite(b), b, 0)) / 2.0 ** np.where(s == 255, 0, s - 127)[..., None]
    up = np.clip(np.searchsorted(GRID, y), 0, 7)                     # first element that is not below
    low = np.maximum(up - 1, 0)
    near_up, near_low = GRID[up] - y, y - GRID[low]
    c = np.where((near_up < near_low) | ((near_up == near_low) & (up % 2 == 0)) | (near_up <= 0), up, low)
    c = np.where(s[..., None] == 255, 0, c + 8 * np.signbit(b))
    return c.reshape(x.shape), s


def page_bytes(x):
    """Pages [..., P * 68] of rows [..., P, 128]."""
    c, s = quantise(x)
    codes = (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    return np.concatenate([codes.reshape(*codes.shape[:-2], -1), s.astype(np.uint8).reshape(*s.shape[:-2], -1)], axis=-1)


def page_values(p, P):
    """The float64 rows [..., P, 128] that pages [..., P * 68] stand for."""
    b = p[..., :64 * P].reshape(*p.shape[:-1], P, 64).astype(np.int64)
    c = np.stack([b & 15, b >> 4], axis=-1).reshape(*p.shape[:-1], P, D)
    s = p[..., 64 * P:].reshape(*p.shape[:-1], P, 4).astype(np.float64)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    unit = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return (v.reshape(*c.shape[:-1], 4, 32) * unit[..., None]).reshape(c.shape)


def rows_of(pool, indptr, indices, b, n, P):
    """The first n cached rows of sequence b, float64 [Hkv][n][128], of one layer's pool [slots][Hkv][P * 68]."""
    slots = indices[indptr[b]:indptr[b + 1]][:-(-n // P)]
    v = page_values(pool[slots], P)
    return v.transpose(1, 0, 2, 3).reshape(pool.shape[1], -1, D)[:, :n]


def attention(q, k, v, scale, causal):
    """One sequence in float64: q [n][Hq][128]; k, v [Hkv][kv][128].  Returns o, lse, and what each may be off by.

    Probabilities are rounded to bf16 (2^-8 of sum p |v| / l = A) and so is the output (2^-8 |o|).  A score is off by
    e = scale (2^-14 sum over blocks of max |q| sum |k| + 128 2^-23 sum |q k|) at most: the query's pieces (the last of
    three leaves S / 2^13 of a block whose largest value is at least 3.75 S), and the fp32 sum; that moves every weight by a factor within exp(+-2 e).  The fp32 sums over n keys add n 2^-23 A."""
    n, Hq, kv = q.shape[0], q.shape[1], k.shape[1]
    G = Hq // k.shape[0]
    o, lse = torch.zeros((n, Hq, D), dtype=torch.float64), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    tol, ltol = torch.full_like(o, 1e-30), torch.full_like(lse, 1e-30)
    if kv == 0 or n == 0:
        return o, lse, tol, ltol
    q = torch.as_tensor(q).double().cuda()
    seen = torch.arange(kv, device="cuda")[None, :] < ((kv - n + 1 + torch.arange(n, device="cuda"))[:, None] if causal else kv)
    for h in range(Hq):
        kk, vv = torch.as_tensor(k[h // G]).cuda(), torch.as_tensor(v[h // G]).cuda()
        s = torch.where(seen, q[:, h] @ kk.t() * scale, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        w = p / total
        a = w @ vv.abs()
        out = w @ vv
        kb = kk.abs().reshape(kv, 4, 32).sum(-1)
        e = (q[:, h].abs().reshape(n, 4, 32).amax(-1) @ kb.t() * 2.0 ** -14 + q[:, h].abs() @ kk.abs().t() * 128 * 2.0 ** -23) * scale
        e = torch.where(seen, e, 0).amax(1, keepdim=True)
        o[:, h], lse[:, h] = out.cpu(), (top + torch.log(total))[:, 0].cpu()
        tol[:, h] = (2.0 ** -8 * (a + out.abs()) + (4 * e + (kv + 64) * 2.0 ** -23) * a).cpu() + 1e-30
        ltol[:, h] = (e[:, 0] + (kv + 64) * 2.0 ** -23 + 2.0 ** -22 * (top + torch.log(total))[:, 0].abs()).cpu()
    return o, lse, tol, ltol

"""Attention over a 4-bit cache in float64, with bounds that see one key's error: no term grows with the largest query dim,
and none with the number of keys beyond the additions that a lane makes."""
import math

import torch

D = 128
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"


def attention(q, k, v, scale, causal, inexact=False):
    """One sequence: q [n][Hq][128]; k, v [Hkv][kv][128].  Returns o, lse, the most each element of them may be off, and
    the most each row of o may be off as a vector.

    A score is off by s = scale 128 2^-23 sum |q k| (the fp32 sum of exact products) and by 2^-22 |score| (the
    scale in fp32, its product and the difference from the offset), its weight by 2^-22 for the exponential.  A lane adds
    a sixteenth of the keys at most one by one (four waves and, within 64 keys, four lanes share them, or the waves
    share the rows and a lane adds its 16 of a tile to each other first), 2^-24 each, and the joins of waves and parts some 64 times more.  Weights are
    rounded to bf16 and so is the output: 2^-8 of each at most.  As a vector the weights' roundings add up as
    independent ones, at most sqrt(sum (2^-8 w |v|)^2); twice that is allowed.

    inexact: what items of more than 32 rows may lose of small query dims, which of a block of 32 adds up to 2^-14 of the
    magnitudes of all but its largest, times the block's largest key."""
    n, Hq, kv = q.shape[0], q.shape[1], k.shape[1]
    G = Hq // k.shape[0]
    o, lse = torch.zeros((n, Hq, D), dtype=torch.float64), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    tol, ltol, row = torch.full_like(o, 1e-30), torch.full_like(lse, 1e-30), torch.full_like(lse, 1e-30)
    if kv == 0 or n == 0:
        return o, lse, tol, ltol, row
    q = torch.as_tensor(q).double().to(DEVICE)
    seen = torch.arange(kv, device=DEVICE)[None, :] < ((kv - n + 1 + torch.arange(n, device=DEVICE))[:, None] if causal else kv)
    for h in range(Hq):
        kk, vv = (torch.as_tensor(x[h // G]).double().to(DEVICE) for x in (k, v))
        s = torch.where(seen, q[:, h] @ kk.t() * scale, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        w = p / total
        out, a = w @ vv, w @ vv.abs()
        norm = torch.linalg.vector_norm(out, dim=1, keepdim=True)
        spread = torch.sqrt((w * w) @ (vv * vv).sum(1, keepdim=True))
        e = scale * 2.0 ** -16 * (q[:, h].abs() @ kk.abs().t()) + 2.0 ** -22 * (s.abs() + 1)
        if inexact:
            b = q[:, h].abs().reshape(n, 4, 32)
            e = e + scale * 2.0 ** -14 * ((b.sum(2) - b.amax(2)) @ kk.abs().reshape(kv, 4, 32).amax(2).t())
        e = torch.where(seen, e, 0).amax(1, keepdim=True) + (kv / 16 + 64) * 2.0 ** -24
        logs = (top + torch.log(total))[:, 0]
        o[:, h], lse[:, h] = out.cpu(), logs.cpu()
        tol[:, h] = (2.0 ** -8 * (a + out.abs()) + 2 * e * a).cpu() + 1e-30
        ltol[:, h] = (e[:, 0] + 2.0 ** -22 * logs.abs()).cpu()
        row[:, h] = (2 * 2.0 ** -8 * torch.sqrt(spread ** 2 + norm ** 2)
                     + 2 * e * torch.linalg.vector_norm(a, dim=1, keepdim=True))[:, 0].cpu() + 1e-30
    return o, lse, tol, ltol, row


def worst(got, got_lse, ref):
    """How far off, in units of what is allowed: elements, LSEs and rows (1 is the most)."""
    o, lse, tol, ltol, row = ref
    off = got.double().cpu() - o
    return ((off.abs() / tol).max().item(), ((got_lse.double().cpu() - lse).abs() / ltol).max().item(),
            (torch.linalg.vector_norm(off, dim=2) / row).max().item())


# ---- caches of known weights: keys of zeros, and values that tell which 64 keys they are of

def coded_values(kv):
    """[kv][128]: a one in the dim that its 64 keys have."""
    v = torch.zeros((kv, D), dtype=torch.float64)
    j = torch.arange(kv)
    v[j, j // 64 % D] = 1
    return v


def coded_worst(got, got_lse, kv, causal):
    """How far off the outputs [n][Hq][128] and LSEs of such a cache are, in units of what is allowed.  Row i sees
    kv - n + i + 1 keys (all, without a mask): its LSE is their number's logarithm, its output their counts by dim over it.

    Up to 2^16 keys a part's log2 is off by v_log's 2^-20 and as much comes back through the weights it gives its
    sums; the joined sum's log2 is off by 2^-20 and 2^-21, its product with ln 2 by 2^-21: 2.2e-6, twice that is
    allowed.  Outputs are rounded to bf16 and their parts' weights off as above."""
    n = got.shape[0]
    counts = torch.cumsum(coded_values(kv), 0)
    seen = [kv - n + i + 1 if causal else kv for i in range(n)]
    o = torch.stack([counts[s - 1] / s for s in seen])[:, None]
    lse = torch.tensor(seen, dtype=torch.float64).log()[:, None]
    return (((got.double().cpu() - o).abs() / ((2.0 ** -8 + 1e-5) * o + 1e-30)).max().item(),
            ((got_lse.double().cpu() - lse).abs() / 4.4e-6).max().item())

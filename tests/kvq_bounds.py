"""Attention over a 4-bit cache in float64, with bounds that see one key's error: no term grows with the largest query dim,
and none with the number of keys beyond the additions that a lane makes."""
import math

import torch

D = 128
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"


def attention(q, k, v, scale, causal):
    """One sequence: q [n][Hq][128]; k, v [Hkv][kv][128].  Returns o, lse, the most each element of them may be off, and
    the most each row of o may be off as a vector.

    A score is off by s = scale 128 2^-23 sum |q k| (the fp32 sum of exact products) and by 2^-22 |score| (the
    scale in fp32, its product and the difference from the offset), its weight by 2^-22 for the exponential.  A lane adds
    a sixteenth of the keys at most one by one (four waves and, within 64 keys, four lanes share them, or the waves
    share the rows and a lane adds its 16 of a tile to each other first), 2^-24 each, and the joins of waves and parts some 64 times more.  Weights are
    rounded to bf16 and so is the output: 2^-8 of each at most.  As a vector the weights' roundings add up as
    independent ones, at most sqrt(sum (2^-8 w |v|)^2); twice that is allowed."""
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

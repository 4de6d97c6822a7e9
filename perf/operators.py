"""The calls that keep several branches of one context alive, as timed cases, with their plain forms.

A case is a dict of plain values; `kind` names the calls that one pass makes:

  attn     sa_shared_prefix_attn: the members of each group share a prefix whose
           keys and values are read once for all of them
  rope     sa_kv_append_rope: norms of the query and key heads, their rotation by
           position, the key and value rows into their pages
  fork     sa_kv_fork and sa_kv_release: children of cached contexts are opened
           (shared pages, a copy of the partial one, fresh ones) and dropped again,
           with the list of free slots made anew
  compact  sa_kv_compact: the pages in use beyond a limit move into free slots below

With `own` false a pass computes the same in elementary torch operations, in 32 bits
(angles in 64), rounded once at the end.  Rows are N(0, 1) / 2 rounded to bf16 on a
shuffled page pool, the distribution of the configurations c1..c5, with 1% of the key
rows times 8 where `outliers` is set (c4's recipe).
"""
import math
import random

import numpy as np
import torch

own = False

D = 128


# ------------------------------------------------------------------------- cases

def _attn(name, heads, page, groups=1, members=(1, 1), pre=(0, 0), own_tokens=(1, 1), q=(1, 1), lens=1,
          outliers=False):
    c = {"kind": "attn", "Hq": heads[0], "Hkv": heads[1], "page": page, "groups": groups, "m_lo": members[0],
         "m_hi": members[1], "pre_lo": pre[0], "pre_hi": pre[1], "own_lo": own_tokens[0], "own_hi": own_tokens[1],
         "q_lo": q[0], "q_hi": q[1], "lens": lens, "outliers": outliers}
    return dict(c, name=name) if name else c


def _rope(name, heads, page, n=1, start=(0, 0), new=(1, 1), rot=128, interleaved=False, norm=True, fused=True,
          theta=1e6, far=0, lens=1):
    c = {"kind": "rope", "Hq": heads[0], "Hkv": heads[1], "page": page, "n": n, "start_lo": start[0],
         "start_hi": start[1], "new_lo": new[0], "new_hi": new[1], "rot": rot, "interleaved": interleaved,
         "norm": norm, "fused": fused, "theta": theta, "far": far, "lens": lens}
    return dict(c, name=name) if name else c


def _fork(name, heads, page, n=1, ctx=(1, 1), children=1, reserve=(0, 0), layers=1, spare=0, lens=1):
    c = {"kind": "fork", "Hq": heads[0], "Hkv": heads[1], "page": page, "n": n, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
         "children": children, "res_lo": reserve[0], "res_hi": reserve[1], "layers": layers, "spare": spare,
         "lens": lens}
    return dict(c, name=name) if name else c


def _compact(name, heads, page, slots=64, limit=32, tail=0.5, holes=0.5, layers=1):
    c = {"kind": "compact", "Hq": heads[0], "Hkv": heads[1], "page": page, "slots": slots, "limit": limit,
         "tail": tail, "holes": holes, "layers": layers}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of four lookahead branches of one short context: the smallest call of a serving loop
        _attn("branch_decode_few", (32, 8), 16, members=(4, 4), pre=(4096, 4096), own_tokens=(1, 64)),
        # a decode step of 32 sub-agents on one isolated 16K context (c5's prefill prefix)
        _attn("branch_decode", (32, 8), 16, members=(32, 32), pre=(16384, 16384), own_tokens=(16, 512)),
        # several contexts with a few branches each, ragged, one of them perhaps alone
        _attn("branch_groups", (32, 8), 16, groups=8, members=(1, 12), pre=(1000, 16000), own_tokens=(1, 700), lens=5),
        # 64 branches of c4's context and layout, outlier keys: 512 query rows on every key head
        _attn("branch_long_c4", (64, 8), 32, members=(64, 64), pre=(65536, 65536), own_tokens=(32, 1024),
              outliers=True),
        # short instruction chunks streamed onto 16 branches of a 16K context
        _attn("branch_segments", (32, 8), 16, members=(16, 16), pre=(16384, 16384), own_tokens=(64, 600), q=(16, 64)),
        # the new rows of one decode step of c5's 64 requests, out of a fused projection
        _rope("rope_decode_c5", (32, 8), 16, n=64, start=(4095, 16383), new=(1, 1)),
        # c1's segment: a small model, separate projections, rotation of interleaved pairs, no norms
        _rope("rope_segment_c1", (8, 2), 16, n=1, start=(512, 512), new=(256, 256), interleaved=True, norm=False,
              fused=False, theta=1e4),
        # c3's 16 ragged segments
        _rope("rope_ragged_c3", (32, 8), 16, n=16, start=(4096, 32768), new=(512, 4096), lens=3),
        # one context of ~4K tokens forked into four lookahead branches, eight layers of it
        _fork("fork_few", (32, 8), 16, n=1, ctx=(4001, 4001), children=4, reserve=(64, 64), layers=8, spare=1024),
        # c3's 16 contexts, four branches each
        _fork("fork_many_c3", (32, 8), 16, n=16, ctx=(4096, 32768), children=4, reserve=(512, 4096), layers=2,
              spare=8192, lens=3),
        # a small pool's last quarter is vacated
        _compact("compact_few", (32, 8), 16, slots=2048, limit=1536, tail=0.5, holes=0.3, layers=8),
        # half of a pool of 32K slots is vacated after most of its branches ended
        _compact("compact_many", (32, 8), 16, slots=32768, limit=16384, tail=0.4, holes=0.6, layers=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    return tuple(sorted((_log(rng, lo, hi), _log(rng, lo, hi))))


def draw(rng):
    """One more case of the ranges the listed ones span."""
    while True:
        kind = rng.choice(["attn", "attn", "rope", "fork", "compact"])
        heads, page = rng.choice([((32, 8), 16), ((64, 8), 32), ((8, 2), 16), ((32, 4), 32), ((24, 8), 16)])
        lens = rng.randrange(1 << 20)
        if kind == "attn":
            groups = _log(rng, 1, 12)
            q = (1, 1) if rng.random() < 0.6 else _span(rng, 1, 64)
            c = _attn(None, heads, page, groups=groups, members=_span(rng, 1, max(1, 64 // groups)),
                      pre=_span(rng, 64, 65536 // groups), own_tokens=_span(rng, q[1], 1024), q=q, lens=lens,
                      outliers=rng.random() < 0.2)
        elif kind == "rope":
            c = _rope(None, heads, page, n=_log(rng, 1, 64), start=_span(rng, 1, 32768), new=_span(rng, 1, 4096),
                      rot=rng.choice([128, 128, 64, 96, 32]), interleaved=rng.random() < 0.3,
                      norm=rng.random() < 0.7, fused=rng.random() < 0.6, theta=rng.choice([1e4, 5e5, 1e6]),
                      far=rng.choice([0, 0, _log(rng, 1000, 1 << 21)]), lens=lens)
        elif kind == "fork":
            c = _fork(None, heads, page, n=_log(rng, 1, 16), ctx=_span(rng, 1, 32768), children=rng.randint(1, 8),
                      reserve=_span(rng, 1, 2048), layers=rng.choice([1, 2, 4]), spare=_log(rng, 16, 8192), lens=lens)
        else:
            slots = _log(rng, 64, 32768)
            c = _compact(None, heads, page, slots=slots, limit=rng.randint(slots // 4, slots - 8),
                         tail=rng.uniform(0.05, 0.95), holes=rng.uniform(0.05, 0.95), layers=rng.choice([1, 2, 4]))
        w = work(c)
        if w["flops"] <= 1.8e11 and w["bytes"] <= 1.8e9 and _pool_bytes(c) <= 4e9:
            return c


# ------------------------------------------------------------------------- shapes

def _pages(x, P):
    return -(-np.asarray(x, dtype=np.int64) // P)


def _attn_lengths(case):
    """(group offsets, shared tokens per group, own tokens and query tokens per member)."""
    r = random.Random(case["lens"])
    sizes = [r.randint(case["m_lo"], case["m_hi"]) for _ in range(case["groups"])]
    shared = [r.randint(case["pre_lo"], case["pre_hi"]) for _ in range(case["groups"])]
    n = sum(sizes)
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(n)]
    mine = [max(x, r.randint(case["own_lo"], case["own_hi"])) for x in q]
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    return offsets, np.array(shared, dtype=np.int64), np.array(mine, dtype=np.int64), np.array(q, dtype=np.int64)


def _rope_lengths(case):
    r = random.Random(case["lens"])
    start = [r.randint(case["start_lo"], case["start_hi"]) for _ in range(case["n"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    return np.array(start, dtype=np.int64), np.array(new, dtype=np.int64)


def _fork_lengths(case):
    """(parent lengths, parent of every child, tokens every child reserves)."""
    r = random.Random(case["lens"])
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["n"])]
    parent = [b for b in range(case["n"]) for _ in range(case["children"])]
    reserve = [r.randint(case["res_lo"], case["res_hi"]) for _ in parent]
    return np.array(ctx, dtype=np.int64), np.array(parent, dtype=np.int64), np.array(reserve, dtype=np.int64)


def _fork_pages(case):
    """Per child: the parent's full pages, and all of the child's."""
    ctx, parent, reserve = _fork_lengths(case)
    P = case["page"]
    return ctx[parent] // P, _pages(ctx[parent] + reserve, P)


def _compact_counts(case):
    """Slots in use from the limit on, free slots below it, pages that move."""
    n_tail = case["slots"] - case["limit"]
    used = min(n_tail, max(1, round(case["tail"] * n_tail)))
    holes = min(case["limit"], max(1, round(case["holes"] * case["limit"])))
    return used, holes, min(used, holes)


def _num_slots(case):
    P = case["page"]
    if case["kind"] == "attn":
        off, shared, mine, _ = _attn_lengths(case)
        sh = np.repeat(shared, np.diff(off))
        need = int((shared // P).sum() + (_pages(sh + mine, P) - sh // P).sum())
        return max(16, need + need // 4)
    if case["kind"] == "rope":
        need = int(_pages(sum(_rope_lengths(case)), P).sum())
        return max(16, need + need // 4)
    if case["kind"] == "fork":
        ctx, _, _ = _fork_lengths(case)
        full, pages = _fork_pages(case)
        return max(16, int(_pages(ctx, P).sum() + (pages - full).sum()) + case["spare"])
    return case["slots"]


def _pool_bytes(case):
    return _num_slots(case) * case["Hkv"] * case["page"] * D * 2 * 2 * case.get("layers", 1)


def work(case):
    Hq, Hkv, P = case["Hq"], case["Hkv"], case["page"]
    row = Hkv * D * 2 * 2                                    # K and V of one token
    if case["kind"] == "attn":
        off, shared, mine, q = _attn_lengths(case)
        pre = np.repeat(shared, np.diff(off)) + mine - q
        pairs = int((q * pre + q * (q + 1) // 2).sum())
        keys = int(shared.sum() + mine.sum())                # the shared tokens once a group
        return {"bytes": float(keys * row + int(q.sum()) * Hq * (2 * D * 2 + 4)), "flops": 4.0 * D * Hq * pairs}
    if case["kind"] == "rope":
        _, new = _rope_lengths(case)
        n = int(new.sum())
        rows = n * (Hq + Hkv)
        return {"bytes": 2.0 * n * (Hq * D * 2 + row),
                "flops": float(rows * (3 * case["rot"] + (4 * D if case["norm"] else 0)))}
    if case["kind"] == "fork":
        ctx, parent, _ = _fork_lengths(case)
        full, pages = _fork_pages(case)
        copied = int((ctx[parent] % P).sum()) * row * case["layers"]
        # tables read and written, each child's counts raised and lowered, the counts read and the free list written
        words = int(_pages(ctx, P).sum()) + 6 * int(pages.sum()) + 2 * _num_slots(case)
        return {"bytes": 2.0 * copied + 4.0 * words, "flops": 0.0}
    used, holes, moved = _compact_counts(case)
    live = case["limit"] - holes + used
    # counts read and written, map written, table read and written
    words = 3 * case["slots"] + 2 * _compact_entries(case, live)
    return {"bytes": 2.0 * moved * P * row * case["layers"] + 4.0 * words, "flops": 0.0}


def _compact_entries(case, live):
    return live + live // 4                                  # a quarter of the pages are listed by two contexts


# ------------------------------------------------------------------------- inputs

def _rows(g, shape):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = t.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device="cuda").mul_(0.5)
    return t


def _outliers(g, k):
    flat = k.view(-1, D)
    hit = torch.randperm(flat.shape[0], generator=g, device="cuda")[:flat.shape[0] // 100]
    flat[hit] = flat[hit] * 8


def _table(lists):
    indptr = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
    return torch.from_numpy(indptr).cuda(), torch.cat(lists).contiguous()


def _attn_inputs(case, g, x):
    off, shared, mine, q = _attn_lengths(case)
    P, Hq = case["page"], case["Hq"]
    if case["outliers"]:
        _outliers(g, x["k"])
    perm = torch.randperm(x["num_slots"], generator=g, device="cuda").to(torch.int32)
    at, lists = 0, []
    for i, s in enumerate(shared.tolist()):
        common = perm[at:at + s // P]
        at += s // P
        first = None
        for b in range(int(off[i]), int(off[i + 1])):
            n = int(_pages(s + mine[b], P)) - s // P
            rest = perm[at:at + n]
            at += n
            if s % P and first is not None:                  # a fork's copy of the partial page
                for pool in (x["k"], x["v"]):
                    pool[0, rest[0].long(), :, :s % P] = pool[0, first, :, :s % P]
            elif s % P:
                first = rest[0].long()
            lists.append(torch.cat([common, rest]))
    x["indptr"], x["indices"] = _table(lists)
    x["groups"], x["shared"] = off.astype(np.int32), shared.astype(np.int32)
    x["q_len"] = q.astype(np.int32)
    x["kv_len"] = (np.repeat(shared, np.diff(off)) + mine).astype(np.int32)
    T = int(q.sum())
    x["q"] = _rows(g, (T, Hq, D))
    x["o"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    x["lse"] = torch.empty((T, Hq), dtype=torch.float32, device="cuda")


def _rope_inputs(case, g, x):
    start, new = _rope_lengths(case)
    P, Hq, Hkv, T = case["page"], case["Hq"], case["Hkv"], int(new.sum())
    perm = torch.randperm(x["num_slots"], generator=g, device="cuda").to(torch.int32)
    counts = _pages(start + new, P).tolist()
    x["indptr"], x["indices"] = _table(list(perm[:sum(counts)].split(counts)))
    x["start"], x["new_len"] = start.astype(np.int32), new.astype(np.int32)
    x["pos"] = (start + case["far"]).astype(np.int32) if case["far"] else None
    if case["fused"]:
        both = _rows(g, (T, Hq + 2 * Hkv, D))
        x["q"], x["k_new"], x["v_new"] = both.split([Hq, Hkv, Hkv], dim=1)
    else:
        x["q"], x["k_new"], x["v_new"] = _rows(g, (T, Hq, D)), _rows(g, (T, Hkv, D)), _rows(g, (T, Hkv, D))
    x["q_out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    x["inv_freq"] = case["theta"] ** (-2.0 * np.arange(case["rot"] // 2, dtype=np.float64) / case["rot"])
    x["q_weight"] = x["k_weight"] = None
    if case["norm"]:
        w = 1.0 + 0.2 * torch.randn((2, D), generator=g, device="cuda")
        x["q_weight"], x["k_weight"] = w.to(torch.bfloat16).unbind(0)


def _fork_inputs(case, g, x):
    ctx, parent, reserve = _fork_lengths(case)
    perm = torch.randperm(x["num_slots"], generator=g, device="cuda").to(torch.int32)
    counts = _pages(ctx, case["page"]).tolist()
    x["indptr"], x["indices"] = _table(list(perm[:sum(counts)].split(counts)))
    x["fresh"] = perm[sum(counts):].contiguous()
    x["src_len"], x["parent"], x["reserve"] = ctx.astype(np.int32), parent.astype(np.int32), reserve.astype(np.int32)
    pages = _fork_pages(case)[1]
    x["dst_indptr"] = torch.zeros(len(parent) + 1, dtype=torch.int32, device="cuda")
    x["dst_indices"] = torch.zeros(int(pages.sum()), dtype=torch.int32, device="cuda")
    x["ref"] = torch.bincount(x["indices"], minlength=x["num_slots"]).to(torch.int32)
    x["free"] = torch.zeros(x["num_slots"], dtype=torch.int32, device="cuda")
    x["num_free"] = torch.zeros(1, dtype=torch.int32, device="cuda")


def _compact_inputs(case, g, x):
    used, holes, _ = _compact_counts(case)
    low = torch.randperm(case["limit"], generator=g, device="cuda")[holes:]
    high = case["limit"] + torch.randperm(case["slots"] - case["limit"], generator=g, device="cuda")[:used]
    live = torch.cat([low, high])
    live = live[torch.randperm(len(live), generator=g, device="cuda")].to(torch.int32)
    table = torch.cat([live, live[:len(live) // 4]])
    x["indices"] = table.contiguous()
    x["ref"] = torch.bincount(table, minlength=case["slots"]).to(torch.int32)
    x["ref_out"] = torch.zeros_like(x["ref"])
    x["indices_out"] = torch.zeros_like(x["indices"])
    x["slot_map"] = torch.zeros_like(x["ref"])
    x["moved"] = torch.zeros(2, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    """Everything in plain torch and numpy: pools, tables, rows and host lengths."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    x = {"num_slots": _num_slots(case)}
    shape = (case.get("layers", 1), x["num_slots"], case["Hkv"], case["page"], D)
    x["k"], x["v"] = _rows(g, shape), _rows(g, shape)
    {"attn": _attn_inputs, "rope": _rope_inputs, "fork": _fork_inputs, "compact": _compact_inputs}[case["kind"]](case, g, x)
    return x


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2607_00151_amd as sa
        s["layout"] = sa.Layout(num_q_heads=case["Hq"], num_kv_heads=case["Hkv"], head_dim=D, page_size=case["page"],
                                num_layers=case.get("layers", 1), num_slots=s["num_slots"])
        s["ctx"] = sa.Context(0)
        if case["kind"] == "rope":
            s["rope"] = sa.Rope(inv_freq=s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                                interleaved=case["interleaved"])
    return s


# ------------------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"attn": _plain_attn, "rope": _plain_rope, "fork": _plain_fork, "compact": _plain_compact}[kind](s)
    import paper_2607_00151_amd as sa
    ctx, L = s["ctx"], s["layout"]
    if kind == "attn":
        sa.sa_shared_prefix_attn(ctx, L, 0, s["q"], s["k"], s["v"], s["q_len"], s["kv_len"], s["indptr"], s["indices"],
                                 s["groups"], s["shared"], D ** -0.5, s["o"], s["lse"])
        return [s["o"], s["lse"]]
    if kind == "rope":
        sa.sa_kv_append_rope(ctx, L, 0, s["rope"], s["q"], s["k_new"], s["v_new"], s["q_out"], s["k"], s["v"],
                             s["start"], s["new_len"], s["indptr"], s["indices"], pos=s["pos"])
        return [s["q_out"], s["k"], s["v"]]
    if kind == "fork":
        sa.sa_kv_fork(ctx, L, s["k"], s["v"], s["src_len"], s["parent"], s["reserve"], s["indptr"], s["indices"],
                      s["fresh"], s["dst_indptr"], s["dst_indices"], ref=s["ref"])
        sa.sa_kv_release(ctx, L, s["dst_indptr"], s["dst_indices"], s["ref"], s["free"], s["num_free"])
        return [s["k"], s["v"], s["dst_indptr"], s["dst_indices"], s["ref"], s["free"], s["num_free"]]
    sa.sa_kv_compact(ctx, L, s["k"], s["v"], s["case"]["limit"], s["ref"], s["ref_out"], s["indices"],
                     s["indices_out"], s["slot_map"], s["moved"])
    return [s["k"], s["v"], s["ref_out"], s["indices_out"], s["slot_map"], s["moved"]]


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


def _gather(pool, slots, n):
    """The first n tokens on these pages, [Hkv][n][D] in fp32."""
    x = pool[0][slots]                                       # [pages][Hkv][P][D]
    return x.transpose(0, 1).reshape(x.shape[1], -1, D)[:, :n].float()


def _plain_attn(s):
    """Per group: scores of all its rows on the shared keys, of each member's rows on its own, one softmax of both."""
    c, scale = s["case"], D ** -0.5
    Hkv, G, P = c["Hkv"], c["Hq"] // c["Hkv"], c["page"]
    q_len, kv_len = s["q_len"].tolist(), s["kv_len"].tolist()
    first = np.concatenate([[0], np.cumsum(_pages(s["kv_len"], P))]).tolist()
    indices = s["indices"].long()
    t0 = 0
    for i, n_shared in enumerate(s["shared"].tolist()):
        members = range(int(s["groups"][i]), int(s["groups"][i + 1]))
        if not members:
            continue
        b = members[0]
        slots = indices[first[b]:first[b + 1]][:-(-n_shared // P)]
        kt = _gather(s["k"], slots, n_shared).transpose(1, 2).contiguous()
        v = _gather(s["v"], slots, n_shared)
        for b in members:
            n, mine = q_len[b], kv_len[b] - n_shared
            skip = n_shared // P
            own_slots = indices[first[b]:first[b + 1]][skip:]
            k2 = _gather(s["k"], own_slots, kv_len[b] - skip * P)[:, n_shared - skip * P:]
            v2 = _gather(s["v"], own_slots, kv_len[b] - skip * P)[:, n_shared - skip * P:]
            q = s["q"][t0:t0 + n].float().view(n, Hkv, G, D).transpose(0, 1).reshape(Hkv, n * G, D) * scale
            a1 = q @ kt
            a2 = q @ k2.transpose(1, 2).contiguous()
            key = torch.arange(mine, device=q.device)
            last = torch.arange(mine - n, mine, device=q.device).repeat_interleave(G)
            a2 = torch.where(key[None, None, :] > last[None, :, None], -math.inf, a2)
            m = torch.maximum(a1.amax(2, keepdim=True), a2.amax(2, keepdim=True)) if n_shared else a2.amax(2, keepdim=True)
            p1, p2 = torch.exp(a1 - m), torch.exp(a2 - m)
            total = p1.sum(2, keepdim=True) + p2.sum(2, keepdim=True)
            o = (p1 @ v + p2 @ v2) / total
            s["o"][t0:t0 + n] = o.view(Hkv, n, G, D).transpose(0, 1).reshape(n, Hkv * G, D).to(torch.bfloat16)
            s["lse"][t0:t0 + n] = (m + torch.log(total)).view(Hkv, n, G).transpose(0, 1).reshape(n, Hkv * G)
            t0 += n
    return [s["o"], s["lse"]]


def _plain_rope(s):
    c = s["case"]
    P, new, start = c["page"], s["new_len"].astype(np.int64), s["start"].astype(np.int64)
    pos0 = start if s["pos"] is None else s["pos"].astype(np.int64)
    step = np.arange(int(new.sum())) - np.repeat(np.cumsum(new) - new, new)
    angle = _int(np.repeat(pos0, new) + step).double()[:, None] * torch.from_numpy(s["inv_freq"]).cuda()
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    half = c["rot"] // 2

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        y = x.clone()
        if c["interleaved"]:
            a, b = x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]
            y[..., 0:c["rot"]:2], y[..., 1:c["rot"]:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., :half], x[..., half:c["rot"]]
            y[..., :half], y[..., half:c["rot"]] = a * cos - b * sin, b * cos + a * sin
        return y.to(torch.bfloat16)

    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    at = _int(np.repeat(start, new) + step)
    first = np.cumsum(_pages(start + new, P)) - _pages(start + new, P)
    slot = s["indices"].long()[_int(np.repeat(first, new)) + at // P]
    s["k"][0].transpose(1, 2)[slot, at % P] = turned(s["k_new"], s["k_weight"])
    s["v"][0].transpose(1, 2)[slot, at % P] = s["v_new"]
    return [s["q_out"], s["k"], s["v"]]


def _plain_fork(s):
    c = s["case"]
    P, ctx, parent = c["page"], s["src_len"].astype(np.int64), s["parent"].astype(np.int64)
    full, pages = _fork_pages(c)
    base = np.cumsum(_pages(ctx, P)) - _pages(ctx, P)        # parents' offsets in the source table
    out = np.concatenate([[0], np.cumsum(pages)])
    taken = np.cumsum(pages - full) - (pages - full)         # children's offsets in the free list
    step = np.arange(int(pages.sum())) - np.repeat(out[:-1], pages)
    shared = step < np.repeat(full, pages)
    source = _int(np.where(shared, np.repeat(base[parent], pages) + step, 0))
    fresh = _int(np.where(shared, 0, np.repeat(taken - full, pages) + step))
    mask = torch.from_numpy(shared).cuda()
    s["dst_indptr"].copy_(_int(out))
    s["dst_indices"].copy_(torch.where(mask, s["indices"][source], s["fresh"][fresh]))
    s["ref"].index_add_(0, s["dst_indices"], torch.ones_like(s["dst_indices"]))
    part = np.flatnonzero(ctx[parent] % P)
    if len(part):
        src = s["indices"].long()[_int(base[parent[part]] + full[part])]
        dst = s["fresh"].long()[_int(taken[part])]
        keep = torch.arange(P, device="cuda")[None, :] < _int(ctx[parent[part]] % P)[:, None]
        for pool in (s["k"], s["v"]):
            pool[:, dst] = torch.where(keep[None, :, None, :, None], pool[:, src], pool[:, dst])
    # the children end: their counts go down again, and the free list is made anew
    s["ref"].index_add_(0, s["dst_indices"], torch.full_like(s["dst_indices"], -1))
    n = s["num_slots"]
    idle = s["ref"] == 0
    place = torch.where(idle, torch.cumsum(idle, 0) - 1, n)
    listed_free = torch.full((n + 1,), -1, dtype=torch.int32, device="cuda")
    listed_free.scatter_(0, place, torch.arange(n, dtype=torch.int32, device="cuda"))
    s["free"].copy_(listed_free[:n])
    s["num_free"].copy_(idle.sum())
    return [s["k"], s["v"], s["dst_indptr"], s["dst_indices"], s["ref"], s["free"], s["num_free"]]


def _plain_compact(s):
    limit, n = s["case"]["limit"], s["num_slots"]
    live = s["ref"] > 0
    hole = torch.nonzero(~live[:limit]).view(-1)
    high = limit + torch.nonzero(live[limit:]).view(-1)
    moved = min(len(hole), len(high))
    src, dst = high[:moved], hole[:moved]
    slot = torch.arange(n, device="cuda")
    to = torch.where(live, slot, -1)
    to[src] = dst
    for pool in (s["k"], s["v"]):
        pool[:, dst] = pool[:, src]
    s["slot_map"].copy_(to)
    s["indices_out"].copy_(s["slot_map"][s["indices"].long()])
    s["ref_out"].copy_(s["ref"])
    s["ref_out"][dst] = s["ref"][src]
    s["ref_out"][src] = 0
    s["moved"].copy_(torch.tensor([moved, len(high) - moved], dtype=torch.int32))
    return [s["k"], s["v"], s["ref_out"], s["indices_out"], s["slot_map"], s["moved"]]


# ------------------------------------------------------------------------- 64-bit reference

def exact(case, seed):
    """The outputs from the definitions, in float64; pages that only move have none."""
    if case["kind"] in ("fork", "compact"):
        return None
    x = _inputs(case, seed)
    return _exact_attn(case, x) if case["kind"] == "attn" else _exact_rope(case, x)


def _exact_attn(case, x):
    """Every sequence by itself over its whole context, head by head."""
    G = case["Hq"] // case["Hkv"]
    ip = x["indptr"].tolist()
    o = torch.empty(x["o"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(x["lse"].shape, dtype=torch.float64, device="cuda")
    t0 = 0
    for b, (n, kv) in enumerate(zip(x["q_len"].tolist(), x["kv_len"].tolist())):
        slots = x["indices"][ip[b]:ip[b + 1]].long()
        visible = kv - n + 1 + torch.arange(n, device="cuda")
        dead = torch.arange(kv, device="cuda")[None, :] >= visible[:, None]
        for h in range(case["Hkv"]):
            keys = x["k"][0, slots, h].reshape(-1, D)[:kv].double()
            values = x["v"][0, slots, h].reshape(-1, D)[:kv].double()
            for i in range(h * G, (h + 1) * G):
                scores = (x["q"][t0:t0 + n, i].double() @ keys.t()) / math.sqrt(D)
                scores[dead] = -math.inf
                lse[t0:t0 + n, i] = torch.logsumexp(scores, 1)
                o[t0:t0 + n, i] = torch.exp(scores - lse[t0:t0 + n, i, None]) @ values
        t0 += n
    return [o, lse]


def _exact_rope(case, x):
    """Pairs as complex numbers, turned by a unit number of the position's angle, sequence by sequence."""
    r, half = case["rot"], case["rot"] // 2
    freq = torch.from_numpy(x["inv_freq"]).cuda()

    def rotate(y, pos):
        unit = torch.polar(torch.ones_like(freq)[None, :].expand(len(pos), -1).contiguous(), pos[:, None] * freq[None, :])
        z = y[..., :r].reshape(*y.shape[:-1], half, 2) if case["interleaved"] else \
            torch.stack([y[..., :half], y[..., half:r]], dim=-1)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * unit[:, None, :])
        z = z.flatten(-2) if case["interleaved"] else torch.cat(z.unbind(-1), dim=-1)
        return torch.cat([z, y[..., r:]], dim=-1)

    def heads(t, w, pos):
        y = t.double()
        if w is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + 1e-6) * w.double()
        return rotate(y, pos)

    q = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    k, v = x["k"].double(), x["v"].double()
    ip, t0 = x["indptr"].tolist(), 0
    for b, (a, n) in enumerate(zip(x["start"].tolist(), x["new_len"].tolist())):
        at = torch.arange(a, a + n, device="cuda")
        pos = (at + case["far"]).double()
        slots = x["indices"][ip[b]:ip[b + 1]].long()[at // case["page"]]
        q[t0:t0 + n] = heads(x["q"][t0:t0 + n], x["q_weight"], pos)
        k[0, slots, :, at % case["page"]] = heads(x["k_new"][t0:t0 + n], x["k_weight"], pos)
        v[0, slots, :, at % case["page"]] = x["v_new"][t0:t0 + n].double()
        t0 += n
    return [q, k, v]

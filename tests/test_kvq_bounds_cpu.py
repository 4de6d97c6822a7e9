"""The bounds that the 4-bit attention is held to: right results pass them, results without a few of their keys do not."""
import numpy as np
import pytest
import torch

from kvq_bounds import D, attention, coded_values, coded_worst, worst


def plain(q, k, v, scale, keep):
    """float64 attention of one token over some of the keys, its output rounded to bf16."""
    s = np.einsum("hd,hnd->hn", q, k[:, keep]) * scale
    p = np.exp(s - s.max(1, keepdims=True))
    o = np.einsum("hn,hnd->hd", p / p.sum(1, keepdims=True), v[:, keep])
    return torch.from_numpy(o)[None].to(torch.bfloat16), torch.from_numpy(s.max(1) + np.log(p.sum(1)))[None]


@pytest.mark.parametrize("kv,lost", [(700, 1), (4096, 1), (4096, 16), (20000, 16), (60000, 16), (60000, 64)])
@pytest.mark.parametrize("where", ["first", "tile", "part", "last"])
def test_lost_keys_are_seen(kv, lost, where):
    r = np.random.default_rng(kv + lost)
    q, k, v = (r.standard_normal(s) * 0.5 for s in ((4, D), (4, kv, D), (4, kv, D)))
    q = torch.from_numpy(q).to(torch.bfloat16)
    ref = attention(q[None], k, v, D ** -0.5, True)
    keep = np.ones(kv, bool)
    assert max(worst(*plain(q.double().numpy(), k, v, D ** -0.5, keep), ref)) < 0.6
    at = {"first": 0, "tile": 320, "part": kv // 128 * 64 - lost, "last": kv - lost}[where]
    keep[at:at + lost] = False
    assert max(worst(*plain(q.double().numpy(), k, v, D ** -0.5, keep), ref)) > 1


@pytest.mark.parametrize("kv", [129, 4096, 40001, 65000])
def test_one_lost_or_doubled_key_of_a_cache_of_known_weights_is_seen(kv):
    v = coded_values(kv)

    def off(w):
        total = w.sum()
        return coded_worst((w @ v / total)[None, None].to(torch.bfloat16), total.log().float()[None, None], kv, True)
    assert max(off(torch.ones(kv, dtype=torch.float64))) < 0.6
    for at in (0, 63, 64, kv // 2, kv - 1):
        for weight in (0.0, 2.0):
            w = torch.ones(kv, dtype=torch.float64)
            w[at] = weight
            assert off(w)[1] > 1, (at, weight)
    w = torch.ones(kv, dtype=torch.float64)                  # 64 keys twice for 64 others: the LSE stays
    w[:64], w[64:128] = 0, 2
    assert off(w)[0] > 1

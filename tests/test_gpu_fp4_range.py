"""Attention over 4-bit pages whose values are near the end of bf16's range, against 64 bits: a row's result lies between
its values, so it is finite wherever they are, however its scores rise and fall."""
import numpy as np
import pytest
import torch

from cache_util import attend, check
from fp4_util import Cache4, bf16_of, key_codes, put_keys, put_values, value_codes
from gpu_util import lib

pytestmark = pytest.mark.gpu
LN2 = 0.6931471805599453  # with sm_scale LN2 / d and rows of ones, a key of a's has a score of a (log2)


def _scores(kind, n, rng):
    """Scores that the codes hold exactly (in units of log2): numbers of the E2M1 grid times powers of two."""
    if kind == "level":
        return np.ones(n)
    if kind == "rising":  # by less than what moves a reference at once
        return np.array([1, 1.5, 2, 3, 4, 6, 8])[np.minimum(np.arange(n) * 7 // n, 6)]
    if kind == "one":  # one token of a step far above the others, by just less than 2^8
        a = np.where(np.arange(n) % 64 == 5, 8.0, 0.5)
        a[:64] = 0.5
        return a
    return rng.choice([-6, -3, -1, 0, 0.5, 2, 4, 6, 8, 12], n).astype(float)


def _values(kind, n, d, rng):
    x = rng.standard_normal((n, d))
    if kind == "all":
        return x * 1e38
    if kind == "same":
        return np.full((n, d), 3e38) * np.sign(x[:, :1])
    if kind == "edge":  # around the scale from which on a weight is kept small: steps on either side of it
        return x * np.exp2(96 + 2 * (np.arange(n) // 64 % 2))[:, None]
    # large ones in a few tokens, ordinary ones around them
    return np.where((np.arange(n) % 97 == 3)[:, None], np.sign(x) * 2e38, x)


def _cache(lens, Hkv, d, P, scores, values, seed):
    rng = np.random.default_rng(seed)
    c = Cache4(lens, Hkv, d, P, seed=seed)
    for b, L in enumerate(c.lens):
        for h in range(Hkv):
            k = np.repeat(_scores(scores, int(L), rng)[:, None], d, 1)
            v = np.clip(_values(values, int(L), d, rng), -3.38e38, 3.38e38)
            for j in range(-(-int(L) // P)):
                at = np.arange(j * P, min(int(L), (j + 1) * P))
                put_keys(c.k[int(c.bt[b, j]), h].numpy(), at % P, *key_codes(bf16_of(k[at])))
                put_values(c.v[int(c.bt[b, j]), h].numpy(), at % P, *value_codes(bf16_of(v[at])))
    return c


@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
@pytest.mark.parametrize("scores", ["level", "rising", "one", "any"])
@pytest.mark.parametrize("values", ["all", "same", "edge", "few"])
def test_values_near_the_end_of_the_range(P, d, scores, values):
    print(f"[case] range P={P} d={d} {scores} {values}", flush=True)
    D, Hkv, G = lib(), 2, 3
    c = _cache([700, 64, 1, 2300, 0, 333], Hkv, d, P, scores, values, seed=P)
    B = len(c.lens)
    q = torch.ones(B, Hkv * G, d, dtype=torch.bfloat16)
    q[:, 1::2] = -1.0  # rows whose scores fall where the others' rise
    scale = LN2 / d
    want, spread = np.zeros(q.shape), np.zeros(q.shape)
    for b, L in enumerate(c.lens):
        o, s = attend(q[b].double().numpy()[None], *c.tokens(b, np.arange(int(L))), np.ones((1, int(L)), bool), scale)
        want[b], spread[b] = o[0], s[0]
    assert np.isfinite(want).all()
    dev, qd = c.gpu(), q.cuda()
    a = (dev["k"], dev["v"], dev["bt"], dev["lens"], None)
    for kw in ({}, {"num_waves": 3}, {"num_waves": 40, "min_range_pages": 1}):
        out = torch.full_like(qd, 7.0)
        D.dora_decode_attn(qd, *a, out, sm_scale=scale, **dev["kw"], **kw)
        check(out, want, spread, f"decode {kw}")
    n = -(-c.lens // P)
    width = int(n.max())
    lists = torch.arange(width, dtype=torch.int32).repeat(B, Hkv, 1).cuda()
    counts = torch.from_numpy(np.tile(n[:, None], (1, Hkv)).astype(np.int32)).cuda()
    out = torch.full_like(qd, 7.0)
    D.dora_decode_attn_pages(qd, lists, counts, *a, out, sm_scale=scale, **dev["kw"])
    check(out, want, spread, "lists in chunks")
    at = (torch.arange(600) % B).cuda()  # many lists: a wave each
    out = torch.full_like(qd[at], 7.0)
    D.dora_decode_attn_pages(qd[at].contiguous(), lists[at].contiguous(), counts[at].contiguous(), *a[:2], dev["bt"][at].contiguous(),
                             dev["lens"][at].contiguous(), None, out, sm_scale=scale, **dev["kw"])
    check(out[:B], want, spread, "a wave a list")
    assert all(torch.equal(out[i:i + B], out[:B]) for i in range(0, 600 - B, B))

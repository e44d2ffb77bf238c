"""dora_decode_attn_tree over rows that are cut between workgroups: longer than 2,048 tokens, for every
form of its kernels, and many of them."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check, odd_scales, random_trees, tree_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _run(c, T, G, counts, seed, roundings=1, **kw):
    print(f"[case] n={len(c.lens)} T={T} G={G} d={c.d} P={c.P} dt={c.dt} stride={c.bt.shape[1]} {kw}", flush=True)
    assert c.bt.shape[1] * c.P > 2048, "whole rows"
    B, g = len(c.lens), torch.Generator().manual_seed(seed)
    q, kd, vd = (torch.randn(B, T, h, c.d, generator=g).to(torch.bfloat16) for h in (c.Hkv * G, c.Hkv, c.Hkv))
    for b, n in enumerate(counts):
        for x in (q, kd, vd):
            x[b, n:] = float("nan")
    mask = random_trees(np.random.default_rng(seed), counts, T)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, counts, out)
    dev, got = c.gpu(), out.cuda()
    lib().dora_decode_attn_tree(q.cuda(), kd.cuda(), vd.cuda(), torch.from_numpy(mask.view(np.int64)).cuda(), dev["k"], dev["v"],
                                dev["bt"], dev["lens"], None, got, node_counts=torch.tensor(counts, dtype=torch.int32).cuda(),
                                **dev["kw"], **kw)
    torch.cuda.synchronize()
    check(got, want, spread, "tree", roundings=roundings)
    for b, n in enumerate(counts):
        assert torch.all(got[b, n:] == 7.0), "rows of nodes that are not there"


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 4), (2, 3), (4, 8), (33, 1), (6, 7), (12, 8), (20, 9)])
def test_every_form(T, G, d, P, dt):
    """One tile to two column blocks, long rows among empty and short ones."""
    counts = [T, T, 1, 0, T, max(1, T // 3), T]
    _run(Cache([2600, 0, 700, 31, 1, 4100, 2049], 2, d, P, dt, seed=T + P), T, G, counts, seed=G)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("T,G", [(2, 4), (8, 6), (13, 8)])
def test_more_sequences_than_threads(T, G, dt):
    """The lists of work of 300 and of 700 sequences take several passes of a workgroup's threads."""
    rng = np.random.default_rng(T)
    for n in (300, 700):
        lens = rng.integers(0, 60, n)
        lens[[5, n - 2]] = 2300, 2900
        counts = [int(x) for x in rng.integers(0, T + 1, n)]
        counts[n - 2] = T
        _run(Cache(lens, 1, 64, 16, dt, seed=n), T, G, counts, seed=n)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("T,G", [(2, 1), (5, 10)])
def test_several_launches(T, G, dt):
    """More sequences than a launch takes (2,048), cut in each."""
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 30, 2100)
    lens[[0, 2047, 2048, 2099]] = 2500, 2100, 2200, 900
    counts = [int(x) for x in rng.integers(0, T + 1, 2100)]
    counts[2047] = counts[2048] = T
    _run(Cache(lens, 1, 64, 16, dt, seed=16), T, G, counts, seed=T)


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(4, 4), (12, 4), (16, 8)])
def test_odd_scales(T, G, d, P):
    """Pages whose scales are 0, negative, infinite or far from 1 in some pieces of a row and not in others."""
    c = Cache([2600, 2100, 900, 2500, 640, 2300, 33], 1, d, P, 1, seed=d + P)
    odd_scales(c)
    _run(c, T, G, [T, T, 1, T - 1, T, 2, T], seed=T, roundings=2)

"""dora_decode_attn_tree where drafts hold infinities and NaN: they belong to the nodes that attend
them, and to no other."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check, random_trees, tree_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _inputs(B, T, Hkv, G, d, seed):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(B, T, h, d, generator=g).to(torch.bfloat16) for h in (Hkv * G, Hkv, Hkv))


def _check(c, q, kd, vd, mask, ns, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, ns, out)
    dev, got = c.gpu(), out.cuda()
    lib().dora_decode_attn_tree(q.cuda(), kd.cuda(), vd.cuda(), torch.from_numpy(mask.view(np.int64)).cuda(), dev["k"], dev["v"],
                                dev["bt"], dev["lens"], None, got, node_counts=torch.tensor(ns, dtype=torch.int32).cuda(),
                                **dev["kw"], **kw)
    torch.cuda.synchronize()
    check(got, want, spread, "tree")
    return got, want


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(5, 3), (40, 1), (12, 4), (20, 6), (64, 5)])
@pytest.mark.parametrize("lens", [[300, 0, 33, 0, 1], [3000, 0, 2300, 700, 0]])
def test_values_of_unattended_drafts_do_not_count(lens, T, G, d, P, dt):
    """One to three column tiles, one and two steps of drafts, rows whole and cut.  In each sequence
    some nodes have an infinite, a negative infinite and a NaN element of V, in dims of their own and in
    one that they share; another's K is NaN."""
    print(f"[case] lens={lens} T={T} G={G} d={d} P={P} dt={dt}", flush=True)
    c = Cache(lens, 2, d, P, dt, seed=T + P + dt)
    rng = np.random.default_rng(T + d)
    ns = [T, T, T - 1, max(1, T // 2), T]
    mask = random_trees(rng, ns, T)
    mask[1, ::2] = 0   # no cache and no bit: zeros
    mask[4, :3] = 0
    q, kd, vd = _inputs(5, T, 2, G, d, 3)
    for b, n in enumerate(ns):
        for x in (q, kd, vd):
            x[b, n:] = NAN
        for i, value in enumerate((INF, -INF, NAN)):
            j = int(rng.integers(0, n))
            vd[b, j, :, 7 * i:7 * i + 3] = value
            vd[b, j, 1, 40 + i] = value
            vd[b, int(rng.integers(0, n)), 0, 50] = value
        if n > 4:
            kd[b, n - 1, 0, 5] = NAN
    got, want = _check(c, q, kd, vd, mask, ns)
    assert np.isnan(want).any() and np.isposinf(want).any() and np.isfinite(want).any()
    assert torch.all(got[1, ::2] == 0)


@pytest.mark.parametrize("T,G", [(6, 4), (9, 6), (40, 4)])
def test_one_branch_does_not_change_the_others(T, G):
    """Two branches under node 0: V of the second is all NaN, or infinite in turn; the first is bitwise
    what it is beside finite ones."""
    c = Cache([500, 0, 2900], 1, 128, 16, 0, seed=2)
    half = T // 2
    first = [1 | (((1 << (i + 1)) - 1) & ~1) for i in range(half)]
    second = [1 | ((1 << (i + 1)) - (1 << half)) for i in range(half, T)]
    mask = np.array([first + second] * 3, np.uint64)
    q, kd, vd = _inputs(3, T, 1, G, 128, 4)
    clean, _ = _check(c, q, kd, vd, mask, [T] * 3)
    for odd in (torch.tensor(NAN), torch.tensor([INF, -INF]).repeat(64)):
        vd[:, half:] = odd.to(torch.bfloat16)
        got, _ = _check(c, q, kd, vd, mask, [T] * 3)
        assert torch.equal(got[:, :half].view(torch.int16), clean[:, :half].view(torch.int16))
        assert not torch.isfinite(got[:, half:].float()).any()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("waves", [1, 6, 40, 4000])
def test_ranges_that_end_between_drafts(waves, G, dt):
    """The two steps of 64 drafts in one workgroup's piece and in two's: a piece adds what is odd in its
    own, where another's may weigh nothing."""
    c = Cache([40, 7, 0, 700, 33], 2, 64, 16, dt, seed=9)
    mask = random_trees(np.random.default_rng(4), [64] * 5, 64)
    mask[2, 5] = 1 << 40  # a node that attends one of the second step alone
    mask[2, 6] = 1 << 3
    q, kd, vd = _inputs(5, 64, 2, G, 64, 6)
    for j, value in ((3, INF), (20, NAN), (40, -INF), (63, INF)):
        vd[:, j, :, j % 7:j % 7 + 2] = value
    _check(c, q, kd, vd, mask, [64] * 5, num_waves=waves)

"""Attention over listed pages where whole parts of a list attend nothing, or have scores of minus infinity: lists that one
workgroup takes, and lists that are cut into chunks and joined."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check
from fp4_util import FP4, make_cache, put_keys
from gpu_util import lib
from test_gpu_pages import TYPES, _q, _reference, _run

pytestmark = pytest.mark.gpu


def _chunked(c, B, Hkv, G, width):
    """Whether a call of this shape joins chunks: then its workspace holds partials."""
    D = lib()
    desc = D.make_decode_desc(num_seqs=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=c.d, page_size=c.P, block_table_stride=c.bt.shape[1],
                              num_pages=c.num_pages, kv_dtype=c.dt)
    return D.dora_decode_pages_workspace_bytes(desc, width) > 256


NOTHING = [-1, -2 ** 31, 2 ** 31 - 1, 10 ** 6]  # entries that are no page of any sequence


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P,d", [(16, 64), (32, 128), (16, 128), (32, 64)])
def test_chunks_that_attend_nothing(dt, P, d):
    """Lists cut into chunks, whose entries are no pages: all of them, or whole chunks of them first, in the middle and
    last; rows without tokens; counts of one chunk and of many."""
    Hkv, G, width = 2, 3, 2048 // P
    c = make_cache([2048, 2048, 0, 2048, 40, 2047, 1, 2048], Hkv, d, P, dt, seed=P + d)
    B = len(c.lens)
    assert _chunked(c, B, Hkv, G, width)
    rng = np.random.default_rng(d)
    part = width // 4  # several chunks: a chunk is 128 tokens here
    lists = np.tile(rng.permutation(width).astype(np.int32), (B, Hkv, 1))
    none = lambda b, at: lists[b, 1].__setitem__(at, rng.choice(NOTHING, len(lists[b, 1, at])))  # noqa: E731
    lists[0] = rng.choice(NOTHING, (Hkv, width))      # nothing at all
    none(1, slice(0, part))                           # first
    none(3, slice(part, 3 * part))                    # in the middle
    none(5, slice(2 * part, width))                   # last
    none(7, slice(0, width - 1))                      # all but the last entry
    counts = np.full((B, Hkv), width, np.int32)
    counts[7, 0] = 128 // P                           # one chunk
    counts[5, 0] = 128 // P + 1                       # and an entry more
    # rows 2, 4 and 6: entries past the sequence's end count for nothing
    q = _q(B, Hkv * G, d, 1)
    want, spread = _reference(c, q, lists, counts)
    assert not want[0].any() and not want[2].any() and want[1].any() and want[4].any()
    out = _run(c, q, lists, counts)
    assert not out[0].any() and not out[2].any()  # exactly 0
    check(out, want, spread, "chunks")


def _sink(c, b, pages):
    """Keys of the pages of sequence b whose score with rows that are 1 in dim 0 is below what fp32 holds."""
    for j in pages:
        page = int(c.bt[b, j])
        slot = np.arange(min(c.P, int(c.lens[b]) - j * c.P))
        if c.dt == FP4:  # -6 times 2^125, rows are 2^20 there
            codes, exps = np.zeros((len(slot), c.d), np.uint8), np.ones((len(slot), c.d // 32), np.uint8)
            codes[:, 0], exps[:, 0] = 15, 252
            for h in range(c.Hkv):
                put_keys(c.k[page, h].numpy(), slot, codes, exps)
        elif c.dt == 0:
            c.k[page, :, 0, :len(slot), 0] = float("-inf")
        else:  # -448 times the largest scale
            c.k[page] = 0
            c.k[page, :, 0, :len(slot), 0] = 0xFE
            c.ks[page] = 3e38


PLACES = {"first": lambda j, n: j < 8, "wave": lambda j, n: j % 4 == 1, "steps": lambda j, n: 4 <= j % 16 < 8,
          "chunk": lambda j, n: 8 <= j < 16, "all but the last": lambda j, n: j < n - 1, "some": lambda j, n: j * 7 % 5 < 2}


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
@pytest.mark.parametrize("place", sorted(PLACES))
def test_scores_of_minus_infinity(dt, P, d, place):
    """Pages whose scores are all minus infinity have no weight, wherever they are: all of a wave's, all of a chunk's."""
    print(f"[case] -inf dt={dt} P={P} d={d} {place}", flush=True)
    D, Hkv, G = lib(), 2, 3
    c = make_cache([1500, 40, 16 * P + 5, 700, 3 * P], Hkv, d, P, dt, seed=3)
    for b, L in enumerate(c.lens):
        n = -(-int(L) // P)
        _sink(c, b, [j for j in range(n) if PLACES[place](j, n) and n > 1 and not (place == "first" and n <= 8)])
    B = len(c.lens)
    q = _q(B, Hkv * G, d, 2)
    q[:, :, 0] = 2.0 ** 20 if dt == FP4 else 1.0
    if dt == FP4:  # the other pages' keys are 0 there
        for b, L in enumerate(c.lens):
            for t in range(int(L)):
                for h in range(Hkv):
                    tile = c.k[int(c.bt[b, t // P]), h].numpy()
                    at = (t % P) * 16
                    if tile[P * d // 2 + (t % P & ~15) + 4 * (t % P & 3) + (t % P >> 2 & 3)] != 252:
                        tile[at] &= 0xF0
    n = -(-c.lens // P)
    width = int(n.max())
    assert _chunked(c, B, Hkv, G, width)
    lists = np.tile(np.arange(width, dtype=np.int32), (B, Hkv, 1))
    counts = np.tile(n[:, None], (1, Hkv)).astype(np.int32)
    with np.errstate(all="ignore"):
        want, spread = _reference(c, q, lists, counts)
    assert np.isfinite(want).all()
    check(_run(c, q, lists, counts), want, spread, "chunks")
    short = min(width, 768 // P)  # not cut: the four waves of a workgroup take turns
    assert not _chunked(c, B, Hkv, G, short)
    for kw in ({}, {"reverse": True}):
        few = np.zeros((B, Hkv, short), np.int32)
        for b in range(B):
            m = min(int(n[b]), short)
            few[b, :, :m] = (n[b] - 1 - np.arange(m)) if kw else np.arange(m)
        few_counts = np.minimum(counts, short)
        with np.errstate(all="ignore"):
            want2, spread2 = _reference(c, q, few, few_counts)
        if place == "all but the last" and not kw:  # the last page is not listed: no row has a weight
            continue
        check(_run(c, q, few, few_counts), want2, spread2, f"a workgroup {kw}")
    dev, qd = c.gpu(), q.cuda()
    for kw in ({}, {"num_waves": 7}):
        out = torch.full_like(qd, 7.0)
        D.dora_decode_attn(qd, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"], **kw)
        check(out, want, spread, f"plain decode {kw}")


@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
def test_rows_whose_scores_are_all_minus_infinity(P, d):
    """There is no weight to share out: NaN, as the plain decode gives; a list without such pages is as it was."""
    D, Hkv = lib(), 1
    c = make_cache([1500, 60], Hkv, d, P, 0, seed=4)
    for b, L in enumerate(c.lens):
        _sink(c, b, range(-(-int(L) // P)))
    q = _q(2, 4, d, 2)
    q[:, :, 0] = 1.0
    n = -(-c.lens // P)
    lists = np.tile(np.arange(int(n.max()), dtype=np.int32), (2, 1, 1))
    assert bool(_run(c, q, lists, n[:, None].astype(np.int32)).isnan().all())
    dev, qd = c.gpu(), q.cuda()
    out = torch.zeros_like(qd)
    D.dora_decode_attn(qd, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"])
    assert bool(out.isnan().all())
    assert not _run(c, q, lists, np.zeros((2, 1), np.int32)).any()


def test_the_helper_of_these_tests():
    """A cache of each type keeps its other keys."""
    for dt in TYPES:
        c = make_cache([100], 1, 64, 16, dt, seed=1)
        before = c.tokens(0, np.arange(100))[0]
        _sink(c, 0, [1, 6])
        after = c.tokens(0, np.arange(100))[0]
        hit = np.zeros(100, bool)
        hit[16:32] = hit[96:] = True
        assert np.array_equal(before[~hit], after[~hit]) and (after[hit, 0, 0] <= -1e38).all()
        assert isinstance(c, Cache)

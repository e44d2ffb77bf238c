"""Attention over listed pages through the C ABI, against 64 bits: bf16, fp8 and 4-bit pages."""
import numpy as np
import pytest
import torch

from cache_util import attend, check
from fp4_util import FP4, make_cache
from gpu_util import lib

pytestmark = pytest.mark.gpu
TYPES = [0, 1, FP4]


def _q(B, Hq, d, seed):
    return torch.randn(B, Hq, d, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _reference(c, q, lists, counts, sm_scale=0.0):
    """Row by row: the tokens of the listed pages that the sequence has, as often as they are listed."""
    q = q.float().double().numpy()
    B, Hq, d = q.shape
    g = Hq // c.Hkv
    want, spread = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        k, v = c.tokens(b, np.arange(max(0, int(c.lens[b]))))
        for h in range(c.Hkv):
            n = min(max(int(counts[b, h]), 0), lists.shape[2])
            t = (lists[b, h, :n].astype(np.int64)[:, None] * c.P + np.arange(c.P)).ravel()
            t = t[(t >= 0) & (t < int(c.lens[b]))]
            if len(t) == 0:
                continue
            rows = slice(h * g, (h + 1) * g)
            o, s = attend(q[b, rows][None], k[t][:, h:h + 1], v[t][:, h:h + 1], np.ones((1, len(t)), bool), sm_scale or d ** -0.5)
            want[b, rows], spread[b, rows] = o[0], s[0]
    return want, spread


def _run(c, q, lists, counts, **kw):
    dev = c.gpu()
    out = torch.full_like(q, 7.0).cuda()
    lib().dora_decode_attn_pages(q.cuda(), torch.from_numpy(lists).cuda(), torch.from_numpy(counts).cuda(), dev["k"], dev["v"], dev["bt"],
                                 dev["lens"], None, out, **dev["kw"], **kw)
    torch.cuda.synchronize()
    return out


def _lists(rng, c, width, heads):
    """Random distinct pages in random order, the last page often among them; entries behind a count point outside."""
    n = -(-c.lens // c.P)
    lists = np.full((len(n), heads, width), 2 ** 31 - 1, np.int32)
    counts = np.zeros((len(n), heads), np.int32)
    for b in range(len(n)):
        for h in range(heads):
            m = min(int(rng.integers(0, width + 1)), int(n[b]))
            lists[b, h, :m] = rng.permutation(int(n[b]))[:m]
            counts[b, h] = m
            if m and rng.random() < 0.5 and n[b] - 1 not in lists[b, h, :m]:
                lists[b, h, rng.integers(0, m)] = n[b] - 1
    return lists, counts


def _hide(c, lists, counts):
    """Table entries of pages that no head lists point outside the pool."""
    for b in range(len(c.lens)):
        listed = set()
        for h in range(c.Hkv):
            listed.update(int(j) for j in lists[b, h, :max(0, int(counts[b, h]))])
        for j in range(c.bt.shape[1]):
            if j not in listed:
                c.bt[b, j] = 2 ** 31 - 1


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 64, 100, 300, 1000, 2050]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,width", [(1, 1), (4, 3), (7, 8), (16, 70)])
def test_lists(dt, P, d, G, width):
    print(f"[case] pages dt={dt} P={P} d={d} G={G} width={width}", flush=True)
    rng = np.random.default_rng(G + width)
    c = make_cache(LENS, 2, d, P, dt, seed=width)
    q = _q(len(LENS), 2 * G, d, G)
    lists, counts = _lists(rng, c, width, 2)
    want, spread = _reference(c, q, lists, counts)
    _hide(c, lists, counts)
    check(_run(c, q, lists, counts), want, spread, "pages")


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P", [16, 32])
def test_long_lists_in_chunks(dt, P):
    """Lists longer than a workgroup's pages, shorter ones and empty ones beside them."""
    print(f"[case] pages chunks dt={dt} P={P}", flush=True)
    rng = np.random.default_rng(P)
    c = make_cache([21000, 40, 0, 12000], 1, 64, P, dt, seed=P)
    q = _q(4, 4, 64, 3)
    n = -(-c.lens // P)
    lists = np.full((4, 1, 1250), -1, np.int32)
    counts = np.array([[min(int(x), 1250)] for x in n], np.int32)
    for b in range(4):
        lists[b, 0, :counts[b, 0]] = np.sort(rng.permutation(int(n[b]))[:counts[b, 0]])
    want, spread = _reference(c, q, lists, counts, 0.2)
    check(_run(c, q, lists, counts, sm_scale=0.2), want, spread, "pages in chunks")


@pytest.mark.parametrize("dt", TYPES)
def test_entries_that_are_no_pages_and_pages_listed_twice(dt):
    """Negative entries, entries at and behind the end, past the table, twice the same; counts outside the list."""
    c = make_cache([50, 33, 0, 200, 16], 2, 64, 16, dt, seed=1)
    q = _q(5, 4, 64, 2)
    lists = np.zeros((5, 2, 6), np.int32)
    lists[0] = [-1, 3, 3, 4, 2 ** 31 - 1, 0]
    lists[1] = [2, 2, 2, 2, 2, 2]
    lists[2] = [0, 0, 1, -7, -2 ** 31, 5]
    lists[3] = [12, 11, 13, 0, c.bt.shape[1], 12]
    lists[4] = [1, 2, 3, -1, 9, 1]
    counts = np.array([[6, 2], [9, -3], [6, 1], [6, 2 ** 31 - 1], [6, 0]], np.int32)
    want, spread = _reference(c, q, lists, counts)
    assert not want[2].any() and not want[4].any() and not want[1, 2:].any()
    check(_run(c, q, lists, counts), want, spread, "entries")


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
def test_all_pages_listed_is_the_plain_decode(dt, P, d):
    D = lib()
    c = make_cache([5, 100, 640, 0, 31, 1500], 2, d, P, dt, seed=3)
    q, dev = _q(6, 10, d, 4).cuda(), c.gpu()
    plain = torch.empty_like(q)
    D.dora_decode_attn(q, dev["k"], dev["v"], dev["bt"], dev["lens"], None, plain, **dev["kw"])
    width = c.bt.shape[1]
    lists = np.tile(np.arange(width, dtype=np.int32), (6, 2, 1))
    counts = np.tile((-(-c.lens // P))[:, None], (1, 2)).astype(np.int32)
    want, spread = _reference(c, q.cpu(), lists, counts)
    check(_run(c, q.cpu(), lists, counts), want, spread, "pages")
    check(plain, want, spread, "plain decode")


@pytest.mark.parametrize("dt", TYPES)
def test_scores_of_minus_infinity_and_nan(dt):
    """A NaN key reaches the rows of its head whose lists hold its page; a row that does not list it is as it was."""
    if dt == FP4:
        c = make_cache([64, 64], 1, 64, 16, dt, seed=5)
        c.k[int(c.bt[0, 2]), 0, 16 * 64 // 2 + 3] = 255  # an exponent of a token of page 2
    else:
        c = make_cache([64, 64], 1, 64, 16, dt, seed=5)
        c.k[int(c.bt[0, 2]), 0, 1, 3, 2] = float("nan") if dt == 0 else 0x7F
    q = _q(2, 4, 64, 6)
    lists = np.array([[[0, 2, 3]], [[0, 2, 3]]], np.int32)
    for counts, hit in (([[3], [3]], True), ([[1], [1]], False)):
        counts = np.array(counts, np.int32)
        out = _run(c, q, lists, counts).float()
        assert bool(out[0].isnan().all()) == hit and not out[1].isnan().any()


def test_two_streams_and_threads_do_not_share_a_workspace():
    """Calls of the same shape on two streams, interleaved, each equal to its own run alone."""
    D = lib()
    cases = []
    for i in range(2):
        c = make_cache([9000, 8000], 1, 64, 16, 0, seed=i)
        q = _q(2, 4, 64, i).cuda()
        lists = torch.arange(560, dtype=torch.int32).repeat(2, 1, 1).cuda()
        counts = torch.tensor([[560], [500]], dtype=torch.int32, device="cuda")
        dev = c.gpu()
        alone = torch.empty_like(q)
        D.dora_decode_attn_pages(q, lists, counts, dev["k"], dev["v"], dev["bt"], dev["lens"], None, alone, **dev["kw"])
        cases.append((q, lists, counts, dev, alone, torch.cuda.Stream(), torch.empty_like(q)))
    torch.cuda.synchronize()
    for _ in range(20):
        for q, lists, counts, dev, _, s, out in cases:
            D.dora_decode_attn_pages(q, lists, counts, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, stream=s, **dev["kw"])
    torch.cuda.synchronize()
    for *_, alone, _, out in cases:
        assert torch.equal(alone, out)


def test_validated_lists():
    D = lib()
    c = make_cache([50, 33], 2, 64, 16, 0, seed=1)
    q = _q(2, 4, 64, 2)
    lists = np.tile(np.array([0, 1, 2], np.int32), (2, 2, 1))
    good = np.full((2, 2), 3, np.int32)
    flags = dict(flags=D.DORA_FLAG_VALIDATE)
    assert torch.equal(_run(c, q, lists, good, **flags), _run(c, q, lists, good))

    def refused(lists, counts, c=c, **kw):
        with pytest.raises(D.DoraError) as e:
            _run(c, q, lists, counts, **flags, **kw)
        assert e.value.status == D.DORA_ERR_DEVICE_CHECK

    for value in (-1, 4, 2 ** 31 - 1):
        bad = lists.copy()
        bad[0, 1, 2] = value
        refused(bad, good)
    for value in (-1, 4):
        counts = good.copy()
        counts[1, 0] = value
        refused(lists, counts)
    c2 = make_cache([50, 33], 2, 64, 16, 0, seed=1)
    c2.bt[1, 2] = c2.num_pages
    refused(lists, good, c=c2)
    c2.lens[1] = 32  # the bad entry is no page of the sequence now, nor listed
    counts = good.copy()
    counts[1] = 2
    _run(c2, q, lists, counts, **flags)

"""The operators that read less of the cache over tables and lists of tens of thousands of pages, on a stream of their own, and
with tables that validation refuses."""
import numpy as np
import pytest
import torch

from cache_util import check
from fp4_util import FP4, make_cache
from gpu_util import lib
from test_gpu_fp4 import _reference as _dense_reference
from test_gpu_pages import TYPES, _q, _reference
from test_gpu_select import _choice, _scores, _select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [2049, 4097, 8193, 9000, 16385, 20001])
def test_choice_of_long_rows(pages):
    """Tables of as many pages as change how many scores a thread holds, and of more than it holds; rows that fill them and
    short ones."""
    print(f"[case] long choice {pages}", flush=True)
    _select([16 * (pages - 2), 16 * (pages - 3) - 7, 16 * 1500, 0, 90], 1, 2, 64, 16, 77, 1, 2, seed=pages, width=pages)
    _select([16 * (pages - 2) - 1], 2, 3, 64, 16, 3000, 0, 0, seed=pages, width=pages, scores=False)


def test_equal_scores_of_long_rows():
    def few(hi, lo, s, q):
        hi[:], lo[:] = 3, -2
        s[:] = 0.25 * 2.0 ** (np.arange(len(s)) % 3)[:, None]

    for pages in (9000, 20000):
        _select([16 * (pages - 2), 16 * 2000], 1, 2, 64, 16, 40, 2, 1, seed=2, make=few, width=pages)


def _repeated(c, times):
    """Sequence b's tokens `times[b]` times one behind the other, over the same pages: whole pages, so that attention over
    all of them is that over one copy."""
    assert all(n == 1 or L % c.P == 0 for n, L in zip(times, c.lens))
    width = max(n * -(-int(L) // c.P) for n, L in zip(times, c.lens))
    bt = np.zeros((len(times), width), np.int32)
    for b, n in enumerate(times):
        one = c.bt[b, :-(-int(c.lens[b]) // c.P)]
        bt[b, :n * len(one)] = np.tile(one, n)
    return torch.from_numpy(bt).cuda(), torch.from_numpy((np.asarray(times) * c.lens).astype(np.int32)).cuda()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P", [16, 32])
def test_rows_of_three_hundred_thousand_tokens(dt, P):
    """Lists of all pages, in chunks of the most that a workgroup takes too; of 4-bit pages the decode by every cut; the
    choice among equal copies."""
    print(f"[case] long rows dt={dt} P={P}", flush=True)
    D, Hkv, G, d = lib(), 2, 3, 64
    c = make_cache([2048, 1024, 70, 0, 512], Hkv, d, P, dt, seed=5)
    times = [150, 7, 1, 1, 33]
    bt, lens = _repeated(c, times)
    B, dev = len(c.lens), c.gpu()
    q = _q(B, Hkv * G, d, 3)
    want, spread = _dense_reference(c, q)
    n = (lens.cpu().numpy() + P - 1) // P
    counts = torch.from_numpy(np.tile(n[:, None], (1, Hkv)).astype(np.int32)).cuda()
    lists = torch.arange(bt.shape[1], dtype=torch.int32, device="cuda").repeat(B, Hkv, 1)
    out = torch.full_like(q, 7.0).cuda()
    args = (dev["k"], dev["v"], bt, lens, None)
    D.dora_decode_attn_pages(q.cuda(), lists, counts, *args, out, **dev["kw"])
    check(out, want, spread, "lists")
    rows = (torch.arange(70) % B).cuda()  # 140 segments: lists are cut by what a workgroup takes alone
    short = torch.minimum(counts, torch.tensor(1300, dtype=torch.int32, device="cuda"))[rows].contiguous()
    few = lists[rows][:, :, :1300].contiguous()
    many = torch.full((70, Hkv * G, d), 7.0, dtype=torch.bfloat16, device="cuda")
    D.dora_decode_attn_pages(q.cuda()[rows].contiguous(), few, short, dev["k"], dev["v"], bt[rows].contiguous(), lens[rows].contiguous(), None, many,
                             **dev["kw"])
    long = object.__new__(type(c))
    long.__dict__.update(c.__dict__)
    long.bt, long.lens = bt.cpu().numpy(), np.minimum(lens.cpu().numpy(), 1300 * P).astype(np.int32)
    want2, spread2 = _reference(long, q, few[:B].cpu().numpy(), short[:B].cpu().numpy())
    check(many[:B], want2, spread2, "many long lists")
    assert all(torch.equal(many[i:i + B], many[:B]) for i in range(0, 70, B))
    if dt == FP4:
        for kw in ({}, {"num_waves": 3}, {"num_waves": 1000}):
            out.fill_(7.0)
            D.dora_decode_attn(q.cuda(), *args, out, **dev["kw"], **kw)
            check(out, want, spread, f"decode {kw}")


def test_calls_on_a_stream_of_their_own():
    """Append, read, bounds, choice and attention given a stream, while the current one is busy, each equal to the same
    calls on the current stream."""
    D, Hkv, G, d, P, T, budget = lib(), 2, 4, 128, 32, 40, 4
    for dt in TYPES:
        c = make_cache([300, 17, 1000], Hkv, d, P, dt, seed=1, extra_tokens=T)
        lens = torch.from_numpy(c.lens + T).cuda()
        g = torch.Generator().manual_seed(2)
        kn, vn = (torch.randn(3, T, Hkv, d, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        q = torch.randn(3, Hkv * G, d, generator=g).to(torch.bfloat16).cuda()

        def run(stream):
            dev = c.gpu()
            torch.cuda.synchronize()
            bounds = torch.zeros(c.num_pages, D.dora_page_bounds_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
            rows = [torch.zeros_like(kn) for _ in range(2)]
            picked = torch.full((3, Hkv, budget), -1, dtype=torch.int32, device="cuda"), torch.zeros(3, Hkv, dtype=torch.int32, device="cuda")
            out = torch.zeros_like(q)
            torch.cuda.synchronize()
            if stream is not None:  # work that a call on the wrong stream would wait for
                busy = torch.randn(4096, 4096, device="cuda")
                for _ in range(20):
                    busy = busy @ busy * 1e-3
            kw = dev["kw"]
            D.dora_kv_append_path(kn, vn, dev["bt"], lens, dev["k"], dev["v"], stream=stream, **kw)
            D.dora_kv_read(dev["k"], dev["v"], dev["bt"], lens, *rows, stream=stream, **kw)
            bkw = {n: x for n, x in kw.items() if n != "v_scales"}
            D.dora_kv_page_bounds(dev["k"], dev["bt"], lens, bounds, num_tokens=T, head_dim=d, stream=stream, **bkw)
            D.dora_page_select(q, bounds, dev["bt"], lens, *picked, num_kv_heads=Hkv, page_size=P, stream=stream)
            D.dora_decode_attn_pages(q, *picked, dev["k"], dev["v"], dev["bt"], lens, None, out, stream=stream, **kw)
            if stream is not None:
                stream.synchronize()
            got = [x.clone() for x in (*rows, bounds, *picked, out)]
            torch.cuda.synchronize()
            return got

        side = torch.cuda.Stream()
        for a, b in zip(run(None), run(side)):
            assert torch.equal(a, b)


def test_validated_choice_bounds_and_reads():
    """Page ids outside the pool and pages of another version: the choice is refused and writes nothing; bounds and reads
    skip the page and report it."""
    D, Hkv, d, P = lib(), 2, 64, 16
    c = make_cache([100, 60], Hkv, d, P, 0, seed=6)
    dev = c.gpu()
    q = _q(2, 4, d, 1).cuda()
    record = D.dora_page_bounds_bytes(Hkv, d)
    owner = torch.full((c.num_pages,), 3, dtype=torch.int16, device="cuda")
    vers = torch.full((2,), 3, dtype=torch.int32, device="cuda")
    own = dict(version_ids=vers, page_owner=owner, flags=D.DORA_FLAG_VALIDATE)
    bad = dev["bt"].clone()
    bad[1, 2] = c.num_pages
    foreign = owner.clone()
    foreign[int(c.bt[1, 2])] = 9
    kw = dict(num_kv_heads=Hkv, page_size=P)
    bounds = torch.randint(0, 100, (c.num_pages, record), generator=torch.Generator().manual_seed(1), dtype=torch.uint8).cuda()
    for table, who, ok in ((dev["bt"], owner, True), (bad, owner, False), (dev["bt"], foreign, False)):
        lists = torch.full((2, Hkv, 3), -5, dtype=torch.int32, device="cuda")
        counts = torch.full((2, Hkv), -5, dtype=torch.int32, device="cuda")
        more = dict(own, page_owner=who)
        if ok:
            D.dora_page_select(q, bounds, table, dev["lens"], lists, counts, **kw, **more)
            assert bool((counts == 3).all()) and bool((lists >= 0).all())
        else:
            with pytest.raises(D.DoraError) as e:
                D.dora_page_select(q, bounds, table, dev["lens"], lists, counts, **kw, **more)
            assert e.value.status == D.DORA_ERR_DEVICE_CHECK and bool((counts == -5).all()) and bool((lists == -5).all())
        status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        taken = torch.full((c.num_pages, record), 0xEE, dtype=torch.uint8, device="cuda")
        D.dora_kv_page_bounds(dev["k"], table, dev["lens"], taken, num_tokens=100, head_dim=d, counts=dev["lens"], dev_status=status, **kw, **more)
        assert status.item() == (D.DORA_OK if ok else D.DORA_ERR_DEVICE_CHECK)
        changed = (taken != 0xEE).any(1).cpu().numpy()
        assert changed.sum() == 7 + 4 - (not ok) and changed[c.bt[1, 2]] == ok
        rows = [torch.full((2, 100, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        D.dora_kv_read(dev["k"], dev["v"], table, dev["lens"], *rows, counts=dev["lens"], dev_status=status, **kw, **more)
        assert status.item() == (D.DORA_OK if ok else D.DORA_ERR_DEVICE_CHECK)
        for x in rows:
            kept = (x == 7.0).flatten(2).all(2).cpu().numpy()  # rows that were not written
            assert not kept[0].any() and kept[1, 60:].all() and not kept[1, :32].any() and not kept[1, 48:60].any()
            assert kept[1, 32:48].all() == (not ok)


def test_scores_of_repeated_pages():
    """Pages that a table names many times have equal scores: the lowest places win."""
    D, Hkv, G, d, P, budget = lib(), 2, 3, 64, 16, 50
    c = make_cache([1600, 320], Hkv, d, P, 0, seed=8)
    bt, lens = _repeated(c, [180, 3])
    dev, rng = c.gpu(), np.random.default_rng(1)
    hi = rng.integers(0, 100, (c.num_pages, Hkv, d)).astype(np.int8)
    lo = -hi
    s = rng.uniform(0.1, 1, (c.num_pages, Hkv)).astype(np.float32)
    raw = np.zeros((c.num_pages, D.dora_page_bounds_bytes(Hkv, d)), np.uint8)
    raw[:, :Hkv * 2 * d] = np.stack([hi, lo], 2).reshape(c.num_pages, -1).view(np.uint8)
    raw[:, Hkv * 2 * d:Hkv * (2 * d + 4)] = s.view(np.uint8)
    q = _q(2, Hkv * G, d, 4)
    lists = torch.full((2, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    counts = torch.zeros(2, Hkv, dtype=torch.int32, device="cuda")
    D.dora_page_select(q.cuda(), torch.from_numpy(raw).cuda(), bt, lens, lists, counts, num_kv_heads=Hkv, page_size=P)
    for b in range(2):
        n = int(lens[b]) // P
        ids = bt[b, :n].cpu().numpy()
        sc = _scores(q[b].float().numpy().astype(np.float64), hi[ids], lo[ids], s[ids])
        for h in range(Hkv):
            assert int(counts[b, h]) == budget and np.array_equal(lists[b, h].cpu().numpy(), _choice(sc[h], n, budget, 1, 1))
    assert dev["bt"].shape[1] < bt.shape[1]

"""Bounds of pages and the choice of pages through the C ABI: every number equal to the definition's."""
import numpy as np
import pytest
import torch

from cache_util import check
from fp4_util import FP4, make_cache
from gpu_util import lib
from test_gpu_pages import TYPES, _reference

pytestmark = pytest.mark.gpu
MOST = np.float32(3.3895313892515355e38)
TINY = np.float32(2.0 ** -126)


def _finite(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isnan(x), 0.0, np.clip(x, -MOST, MOST))


def _bounds(x):
    """hi, lo int8 [Hkv][d], scale fp32 [Hkv] of keys [t][Hkv][d] (fp32 values in 64 bits)."""
    with np.errstate(all="ignore"):
        x = _finite(x).astype(np.float32)
        hi, lo = x.max(0), x.min(0)
        s = np.maximum(np.maximum(np.abs(hi), np.abs(lo)).max(1) / np.float32(127), TINY)
        hi, lo = np.ceil(hi / s[:, None]), np.floor(lo / s[:, None])
    return np.clip(hi, -127, 127).astype(np.int8), np.clip(lo, -127, 127).astype(np.int8), s


def _record(hi, lo, s):
    Hkv, d = hi.shape
    r = np.zeros(-(-Hkv * (2 * d + 4) // 16) * 16, np.uint8)
    r[:Hkv * 2 * d] = np.stack([hi, lo], 1).reshape(-1).view(np.uint8)
    r[Hkv * 2 * d:Hkv * (2 * d + 4)] = s.astype(np.float32).view(np.uint8)
    return r


def _tokens32(c, b, t):
    """Keys as the library's fp32 values, in 64 bits (an fp8 code times a scale is rounded)."""
    k, _ = c.tokens(b, t)
    with np.errstate(all="ignore"):
        k = k.astype(np.float32).astype(np.float64)
    if c.dt == FP4:  # a NaN block counts as 0, the other blocks of the token as they are
        k = np.where(np.isnan(k), 0.0, k)
    return k


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d,Hkv", [(64, 1), (64, 5), (128, 2), (128, 8)])
def test_bounds(dt, P, d, Hkv):
    print(f"[case] bounds dt={dt} P={P} d={d} Hkv={Hkv}", flush=True)
    D = lib()
    lens = np.array([0, 1, 15, 16, 17, 33, 64, 100, 203], np.int32)
    counts = np.array([0, 1, 15, 3, 1, 33, 0, 40, 150], np.int32)
    c = make_cache(lens, Hkv, d, P, dt, seed=d + P)
    if dt == 0:  # keys that are NaN, infinite, subnormal, zero
        c.k[int(c.bt[5, 0]), 0, :, 3] = float("nan")
        c.k[int(c.bt[5, 0]), Hkv - 1, 1, 2, 0] = float("-inf")
        c.k[int(c.bt[2, 0]), 0, :, :15] = 0.0
        c.k[int(c.bt[4, 0]), 0] = c.k[int(c.bt[4, 0]), 0] * 1e-38
    elif dt == 1:
        c.k[int(c.bt[5, 0]), 0, :, 3] = 0x7F
        c.ks[int(c.bt[5, 1])] = -0.25
    else:
        c.k[int(c.bt[5, 0]), 0, P * d // 2 + 1] = 255
    dev = c.gpu()
    rec = D.dora_page_bounds_bytes(Hkv, d)
    start = torch.randint(0, 256, (c.num_pages, rec), generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    bounds = start.cuda()
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    kw = {k: v for k, v in dev["kw"].items() if k != "v_scales"}
    D.dora_kv_page_bounds(dev["k"], dev["bt"], dev["lens"], bounds, num_tokens=150, head_dim=d, counts=torch.from_numpy(counts).cuda(),
                          dev_status=status, **kw)
    assert status.item() == 0
    want = start.numpy().copy()
    used = Hkv * (2 * d + 4)
    for b, (L, n) in enumerate(zip(lens, counts)):
        for j in range((L - n) // P, -(-int(L) // P)) if n else ():
            t = np.arange(j * P, min(int(L), (j + 1) * P))
            want[c.bt[b, j], :used] = _record(*_bounds(_tokens32(c, b, t)))[:used]
    assert np.array_equal(bounds.cpu().numpy()[:, :used], want[:, :used])


def test_bounds_skip_what_fits_no_row():
    D = lib()
    c = make_cache([20, 20, 20, 20], 2, 64, 16, 0, seed=1)
    c.bt[3, 1] = -1
    dev = c.gpu()
    counts = torch.tensor([3, -1, 21, 20], dtype=torch.int32, device="cuda")
    bounds = torch.full((c.num_pages, D.dora_page_bounds_bytes(2, 64)), 0xAB, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = {k: v for k, v in dev["kw"].items() if k != "v_scales"}
    D.dora_kv_page_bounds(dev["k"], dev["bt"], dev["lens"], bounds, num_tokens=32, head_dim=64, counts=counts, dev_status=status, **kw)
    assert status.item() == D.DORA_ERR_DEVICE_CHECK
    changed = (bounds != 0xAB).any(1).cpu().numpy()
    assert changed[c.bt[0, 1]] and changed[c.bt[3, 0]] and changed.sum() == 2


def _scores(q, hi, lo, s):
    """[Hkv][n] of rows q [Hq][d] (bf16 values) and bounds hi, lo [n][Hkv][d], s [n][Hkv]."""
    Hq, d = q.shape
    Hkv = hi.shape[1]
    q = _finite(q).astype(np.float32)
    step = np.maximum(np.abs(q).max(1) / np.float32(127), TINY)
    u = np.clip(np.rint(q / step[:, None]), -127, 127).astype(np.int64).reshape(Hkv, -1, d)
    hi, lo = hi.astype(np.int64), lo.astype(np.int64)
    out = np.zeros((Hkv, len(hi)), np.float32)
    with np.errstate(over="ignore"):
        for h in range(Hkv):
            total = np.maximum(u[h], 0) @ hi[:, h].T + np.minimum(u[h], 0) @ lo[:, h].T
            out[h] = (total.astype(np.float32) * step.reshape(Hkv, -1)[h][:, None]).max(0) * s[:, h]
    return out


def _choice(scores, n, budget, sinks, recent):
    if n <= budget:
        return np.arange(n)
    middle = np.arange(sinks, n - recent)
    order = np.lexsort((middle, -scores[sinks:n - recent].astype(np.float64)))
    return np.sort(np.concatenate([np.arange(sinks), middle[order[:budget - sinks - recent]], np.arange(n - recent, n)]))


def _select(lens, Hkv, G, d, P, budget, sinks, recent, seed, make=None, scores=True, width=0):
    """Scores, lists and counts against the definition.  A table of more than 1,024 pages takes two launches, a narrower
    one of as few rows as here one."""
    D = lib()
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    n = -(-lens // P)
    width = max(width, int(n.max()) + 2)
    pages = int(n.sum()) + 3
    hi = rng.integers(-40, 128, (pages, Hkv, d)).astype(np.int8)
    lo = np.minimum(hi, rng.integers(-127, 41, hi.shape)).astype(np.int8)
    s = rng.uniform(0.01, 0.03, (pages, Hkv)).astype(np.float32)
    q = torch.randn(len(lens), Hkv * G, d, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
    if make:
        make(hi, lo, s, q)
    table = np.full((len(lens), width), 2 ** 31 - 1, np.int32)
    perm = rng.permutation(pages)
    at = 0
    for b in range(len(lens)):
        table[b, :n[b]] = perm[at:at + n[b]]
        at += n[b]
    bounds = torch.from_numpy(np.stack([_record(hi[i], lo[i], s[i]) for i in range(pages)])).cuda()
    lists = torch.full((len(lens), Hkv, budget), -9, dtype=torch.int32, device="cuda")
    counts = torch.full((len(lens), Hkv), -9, dtype=torch.int32, device="cuda")
    sc = torch.full((len(lens), Hkv, width), 5.5, dtype=torch.float32, device="cuda") if scores else None
    D.dora_page_select(q.cuda(), bounds, torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), lists, counts, num_kv_heads=Hkv,
                       page_size=P, sink_pages=sinks, recent_pages=recent, scores=sc)
    lists, counts = lists.cpu().numpy(), counts.cpu().numpy()
    for b in range(len(lens)):
        ids = table[b, :n[b]]
        want = _scores(q[b].float().numpy().astype(np.float64), hi[ids], lo[ids], s[ids])
        if scores:
            assert np.array_equal(sc[b, :, :n[b]].cpu().numpy(), want), b
            assert (sc[b, :, n[b]:] == 5.5).all()
        for h in range(Hkv):
            pick = _choice(want[h], int(n[b]), budget, sinks, recent)
            assert counts[b, h] == len(pick)
            assert np.array_equal(lists[b, h, :len(pick)], pick), (b, h)
            assert (lists[b, h, len(pick):] == -9).all()


LENS = [0, 1, 16, 17, 100, 255, 256, 257, 500, 1000, 4000]


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(1, 1), (2, 7), (5, 16), (8, 4)])
@pytest.mark.parametrize("width", [0, 1025])
def test_choice(P, d, Hkv, G, width):
    print(f"[case] select P={P} d={d} Hkv={Hkv} G={G} width={width}", flush=True)
    _select(LENS, Hkv, G, d, P, 9, 1, 2, seed=P + d + G, width=width)
    _select(LENS, Hkv, G, d, P, 1, 0, 0, seed=P + d + G, scores=False, width=width)


@pytest.mark.parametrize("pages", [255, 256, 257, 1023, 1024])
@pytest.mark.parametrize("d", [64, 128])
def test_one_launch_at_its_widest(pages, d):
    _select([16 * (pages - 2) - 15, 16 * (pages - 2), 16 * 200, 5], 3, 5, d, 16, 33, 1, 2, seed=pages, width=pages)


@pytest.mark.parametrize("rows", [32, 33, 64, 65])
@pytest.mark.parametrize("width", [40, 300])
def test_rows_around_a_round_of_workgroups(rows, width):
    _select([16 * (5 + i % 31) for i in range(rows)], 8, 2, 64, 16, 7, 0, 1, seed=rows, width=width, scores=rows % 2 == 0)


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 1), (1, 1, 0), (5, 2, 3), (16, 0, 0), (100, 3, 7), (3000, 1, 1)])
def test_budgets(budget, sinks, recent):
    """Budgets that the kept pages fill, that hold every page, that are wider than the table."""
    _select([0, 30, 400, 1600, 5000, 47000], 2, 4, 64, 16, budget, sinks, recent, seed=budget)


def test_rows_of_many_tiles():
    """More pages than one round of a workgroup holds, several times over."""
    _select([16 * 1024, 16 * 1025, 16 * 5000 + 1, 16 * 2047], 1, 2, 64, 16, 700, 1, 1, seed=3)


def test_equal_scores_go_to_the_lower_page():
    def same(hi, lo, s, q):
        hi[:], lo[:], s[:] = 3, -2, 0.5

    def two_kinds(hi, lo, s, q):
        hi[:], lo[:], s[:] = 3, -2, np.where(np.arange(len(s)) % 3 == 0, 0.5, 0.25)[:, None]

    def zeros(hi, lo, s, q):  # scores of 0 and -0
        hi[:], lo[:] = 0, 0
        hi[::2] = -1
        lo[::2] = -1
        s[:] = 2.0 ** -126
        q *= 1e-38

    for make in (same, two_kinds, zeros):
        _select([800, 5000, 17000], 2, 3, 64, 16, 20, 2, 1, seed=1, make=make)
        _select([800, 5000, 16000], 2, 3, 64, 16, 20, 2, 1, seed=1, make=make)


def test_scores_below_zero_and_past_the_range():
    def negative(hi, lo, s, q):
        hi[:] = np.minimum(hi, -1)
        lo[:] = np.minimum(lo, hi)
        q[:] = q.abs()

    def huge(hi, lo, s, q):
        s[::3] = 3e38
        q *= 1e30

    def odd(hi, lo, s, q):
        q[0, 0, 3] = float("nan")
        q[1, 1] = 0
        q[2, 2, 5] = float("inf")
        q[2, 3, 5] = float("-inf")

    for make in (negative, huge, odd):
        for width in (0, 1025):
            _select([300, 2000, 700], 2, 3, 128, 32, 8, 0, 1, seed=2, make=make, width=width)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
def test_bounds_choice_and_attention_together(dt, P, d):
    """Prompts are appended, their bounds taken, pages chosen and attended; then a token a step.  The scores bound what
    the rows give every token of a page, but for the rounding of the row to 8 bits."""
    D, Hkv, G, budget = lib(), 2, 4, 6
    lens = np.array([1, 40, 700, 90, 300], np.int32)
    steps = 3
    c = make_cache(np.zeros_like(lens), Hkv, d, P, dt, seed=1, extra_tokens=int(lens.max()) + steps)
    dev = c.gpu()
    if dt == 1:
        dev["kw"]["k_scales"].fill_(1.0)
        dev["kw"]["v_scales"].fill_(1.0)
    g = torch.Generator().manual_seed(2)
    kn, vn = (torch.randn(len(lens), 700, Hkv, d, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    bounds = torch.zeros(c.num_pages, D.dora_page_bounds_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    lists = torch.full((len(lens), Hkv, budget), -1, dtype=torch.int32, device="cuda")
    counts = torch.zeros(len(lens), Hkv, dtype=torch.int32, device="cuda")
    bkw = {k: v for k, v in dev["kw"].items() if k != "v_scales"}
    for step in range(steps + 1):
        now = lens + step
        ln = torch.from_numpy(now).cuda()
        new = ln if step == 0 else torch.ones_like(ln)
        D.dora_kv_append_path(kn, vn, dev["bt"], ln, dev["k"], dev["v"], counts=new, **dev["kw"])
        D.dora_kv_page_bounds(dev["k"], dev["bt"], ln, bounds, num_tokens=700, head_dim=d, counts=new, **bkw)
        q = torch.randn(len(lens), Hkv * G, d, generator=g).to(torch.bfloat16)
        scores = torch.zeros(len(lens), Hkv, dev["bt"].shape[1], device="cuda")
        D.dora_page_select(q.cuda(), bounds, dev["bt"], ln, lists, counts, num_kv_heads=Hkv, page_size=P, scores=scores)
        out = torch.empty_like(q).cuda()
        D.dora_decode_attn_pages(q.cuda(), lists, counts, dev["k"], dev["v"], dev["bt"], ln, None, out, **dev["kw"])
        c.lens = now
        c.k, c.v = dev["k"].cpu(), dev["v"].cpu()
        if dt == 1:
            c.ks, c.vs = dev["kw"]["k_scales"].cpu(), dev["kw"]["v_scales"].cpu()
        li, co, sc = lists.cpu().numpy(), counts.cpu().numpy(), scores.cpu().numpy()
        check(out, *_reference(c, q, li, co), "chosen pages")
        for b in range(len(lens)):
            k, _ = c.tokens(b, np.arange(now[b]))
            n = -(-int(now[b]) // P)
            want = []
            for j in range(n):
                want.append(_bounds(_tokens32(c, b, np.arange(j * P, min(int(now[b]), (j + 1) * P)))))
            hi, lo, s = (np.stack(x) for x in zip(*want))
            qb = q[b].float().numpy().astype(np.float64)
            assert np.array_equal(sc[b, :, :n], _scores(qb, hi, lo, s))
            dots = np.einsum("hgd,thd->hgt", qb.reshape(Hkv, G, d), k).max(1)  # [Hkv][t]
            # a row's value is off by half of its step, a key is at most 127 steps of its page's scale
            slack = 0.5 * (np.abs(qb).max(1) / 127).reshape(Hkv, G).max(1)[:, None] * d * 127 * s.T * 1.001
            for j in range(n):
                assert (dots[:, j * P:(j + 1) * P].max(1) <= sc[b, :, j] + slack[:, j]).all()
            for h in range(Hkv):
                assert np.array_equal(li[b, h, :co[b, h]], _choice(sc[b, h], n, budget, 1, 1))

"""dora_kv_append_path through the C ABI: pages and scales bit for bit what as many single
appends of the oracle leave."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _np(t, dt):
    t = t.contiguous().cpu()
    return t.view(torch.int16).numpy().view(np.uint16).copy() if dt == 0 else t.view(torch.uint8).numpy().copy()


def _same(a, b, dt):
    """Bit for bit; a NaN code's sign, which the fp8 policy leaves open (the single append
    keeps it, the oracle does not), apart."""
    if dt == 1:
        a, b = (np.where((x & 0x7F) == 0x7F, 0x7F, x) for x in (a, b))
    return np.array_equal(a, b)


def _pool(n, Hkv, d, P, dt, g):
    X = wl.chunk_elems(dt)
    shapes = (n, Hkv, d // X, P, X), (n, Hkv, d, P)
    if dt == 0:
        k, v = (torch.randint(0, 65536, s, generator=g, dtype=torch.int32).to(torch.int16).view(torch.bfloat16) for s in shapes)
        return k, v, None, None
    k, v = (torch.randint(0, 256, s, generator=g, dtype=torch.int32).to(torch.uint8) for s in shapes)
    scales = [torch.rand(n, generator=g) * 0.02 + 1e-3 for _ in range(2)]
    return k, v, scales[0], scales[1]


def _case(before, counts, T, Hkv, d, P, dt, seed, path=None, spread=0.8, values=None, given=True):
    print(f"[case] append path T={T} Hkv={Hkv} d={d} P={P} dt={dt}", flush=True)
    g = torch.Generator().manual_seed(seed)
    B = len(before)
    before, counts = np.asarray(before, np.int32), np.asarray(counts, np.int32)
    lens = (before + counts).astype(np.int32)
    n = int(wl.pages_needed(lens, P).sum()) + 3
    bt, _ = wl.place_pages(lens, P, n, seed=seed + 1)
    k, v, ks, vs = _pool(n, Hkv, d, P, dt, g)
    mags = torch.exp(torch.randn(B, T, 1, 1, generator=g) * spread)
    kn, vn = ((torch.randn(B, T, Hkv, d, generator=g) * mags).to(torch.bfloat16) for _ in range(2))
    if values is not None:
        values(kn, vn)
    hk, hv = _np(k, dt), _np(v, dt)
    hks, hvs = (None if x is None else x.numpy().copy() for x in (ks, vs))
    rows = np.tile(np.arange(T), (B, 1)) if path is None else path
    kb, vb = _np(kn, 0), _np(vn, 0)
    for i in range(int(counts.max()) if B else 0):
        now = np.where(i < counts, before + i + 1, 0).astype(np.int32)
        at = np.clip(rows[:, min(i, T - 1)], 0, T - 1)
        assert oracle.kv_append(kb[np.arange(B), at], vb[np.arange(B), at], bt, now, hk, hv, kv_dtype=dt, page_size=P,
                                k_scales=hks, v_scales=hvs) == 0
    dk, dv = k.cuda(), v.cuda()
    dks, dvs = (None if x is None else x.cuda() for x in (ks, vs))
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    lib().dora_kv_append_path(kn.cuda(), vn.cuda(), torch.from_numpy(bt).cuda(), torch.from_numpy(lens).cuda(), dk, dv,
                              num_kv_heads=Hkv, page_size=P, kv_dtype=dt, k_scales=dks, v_scales=dvs,
                              path=None if path is None else torch.from_numpy(path.astype(np.int32)).cuda(),
                              counts=torch.from_numpy(counts).cuda() if given else None, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert _same(_np(dk, dt), hk, dt) and _same(_np(dv, dt), hv, dt)
    if dt == 1:
        assert np.array_equal(dks.cpu().numpy().view(np.uint32), hks.view(np.uint32))
        assert np.array_equal(dvs.cpu().numpy().view(np.uint32), hvs.view(np.uint32))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("Hkv,d", [(1, 64), (4, 128), (8, 128), (3, 64)])
def test_paths(dt, P, Hkv, d):
    """Ascending, repeated and backward paths; every slot a page can be entered at."""
    T, B = 12, 40
    rng = np.random.default_rng(P + d + dt)
    path = rng.integers(0, T, (B, T))
    counts = rng.integers(0, T + 1, B)
    counts[:4] = [0, 1, T, T]
    path[np.arange(T)[None, :] >= counts[:, None]] = 10 ** 6  # not read
    _case(np.arange(B), counts, T, Hkv, d, P, dt, seed=d + P, path=path)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("T", [1, 17, 90])
def test_runs_in_order(dt, P, T):
    counts = [T, T, max(0, T - 1), T // 2, T, T]
    _case([0, 5, 31, 100, 16, 47], counts, T, 2, 128, P, dt, seed=T + P)
    _case([0, 5, 31], [T] * 3, T, 2, 64, P, dt, seed=T + P + 1, given=False)


def test_scales_that_grow_with_every_token():
    """31 growths of one page, down to codes that vanish, and up from zeros."""
    def rising(kn, vn):
        for i in range(kn.shape[1]):
            kn[:, i] *= 1.3 ** i
            vn[:, i] *= 2.0 ** (i % 9)
        kn[1, 0] = 0
        vn[1, :3] = 0
    _case([0, 0, 3, 30], [32, 32, 29, 33], 33, 2, 64, 32, 1, seed=5, spread=0.0, values=rising)
    _case([0, 0, 3, 14], [16, 16, 13, 19], 33, 2, 64, 16, 1, seed=6, spread=0.0, values=rising)


@pytest.mark.parametrize("dt", [0, 1])
def test_equals_single_appends(dt):
    """Against dora_kv_append itself, NaN codes and tokens with NaN and infinities included."""
    D = lib()
    g = torch.Generator().manual_seed(8 + dt)
    B, T, Hkv, d, P = 30, 20, 2, 64, 16
    k, v, ks, vs = _pool(4 * B, Hkv, d, P, dt, g)
    kn, vn = ((torch.randn(B, T, Hkv, d, generator=g) * torch.exp(torch.randn(B, T, 1, 1, generator=g))).to(torch.bfloat16).cuda()
              for _ in range(2))
    for x in (kn, vn):
        x[3, 7, 1, 2], x[5, 1, 0, 9], x[6, 3, 1, 1] = float("nan"), float("inf"), -float("inf")
    bt = torch.randperm(4 * B, generator=g).to(torch.int32).view(B, 4).cuda()
    before = torch.arange(B, dtype=torch.int32).cuda()
    pools = [[None if x is None else x.cuda() for x in (k, v, ks, vs)] for _ in range(2)]
    kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=dt)
    for i in range(T):
        a = pools[0]
        D.dora_kv_append(kn[:, i].contiguous(), vn[:, i].contiguous(), bt, before + i + 1, a[0], a[1], k_scales=a[2], v_scales=a[3], **kw)
    a = pools[1]
    D.dora_kv_append_path(kn, vn, bt, before + T, a[0], a[1], k_scales=a[2], v_scales=a[3], **kw)
    torch.cuda.synchronize()
    for x, y in zip(*pools):
        if x is not None:
            dtype = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
            assert torch.equal(x.view(dtype), y.view(dtype))


@pytest.mark.parametrize("scale", [float("nan"), 0.0, 2.0 ** -126, 2.0 ** -81, 2.0 ** -80 * 1.3, 2.0 ** -40, (5 * 2 ** 20 - 1) * 2.0 ** -23,
                                   (9 * 2 ** 20 + 1) * 2.0 ** -30, 0.75, 1.0, 2.0 ** 60 * 1.7, 2.0 ** 99, 2.0 ** 101, float("inf")])
def test_every_magnitude_over_every_scale(scale):
    """Against dora_kv_append: random bit patterns under a page scale that is given, quotients next to
    and on the ties of two codes, zeros of both signs, and what is far below or above the scale."""
    D = lib()
    g = torch.Generator().manual_seed(3)
    B, T, Hkv, d, P = 24, 15, 4, 128, 16
    k, v, ks, vs = _pool(2 * B, Hkv, d, P, 1, g)
    s = scale if 0 < scale < 1e38 else 1.0
    ks[:], vs[:] = scale, scale
    new = []
    for _ in range(2):
        ties = (torch.randint(0, 512, (B, T, Hkv, d), generator=g).double() - 256) * s * 2.0 ** torch.randint(-8, 1, (B, T, Hkv, d), generator=g).double()
        wide = torch.randn(B, T, Hkv, d, generator=g).double() * s * 2.0 ** torch.randint(-20, 7, (B, T, 1, 1), generator=g).double()
        x = torch.where(torch.rand(B, T, Hkv, d, generator=g) < 0.5, ties, wide).to(torch.bfloat16)
        bits = torch.randint(0, 65536, x.shape, generator=g, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
        x = torch.where(torch.rand(B, T, 1, 1, generator=g) < 0.05, bits, x)
        new.append(torch.where(torch.rand(x.shape, generator=g) < 0.02, x * 0, x).cuda())
    bt = torch.randperm(2 * B, generator=g).to(torch.int32).view(B, 2).cuda()
    before = (torch.arange(B, dtype=torch.int32) % 17).cuda()
    pools = [[x.cuda() for x in (k, v, ks, vs)] for _ in range(2)]
    kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=1)
    for i in range(T):
        a = pools[0]
        D.dora_kv_append(new[0][:, i].contiguous(), new[1][:, i].contiguous(), bt, before + i + 1, a[0], a[1], k_scales=a[2], v_scales=a[3], **kw)
    a = pools[1]
    D.dora_kv_append_path(new[0], new[1], bt, before + T, a[0], a[1], k_scales=a[2], v_scales=a[3], **kw)
    torch.cuda.synchronize()
    for x, y in zip(*pools):
        if x.element_size() == 1:
            # apart from a NaN code's sign: under a NaN scale the old code's value is a product of two
            # NaNs, whose sign IEEE 754 leaves open
            assert _same(x.cpu().numpy(), y.cpu().numpy(), 1)
        else:
            assert torch.equal(x.view(torch.int32), y.view(torch.int32))


def test_infinities_and_nan():
    def odd(kn, vn):
        kn[0, 2, 0, 5] = float("inf")
        vn[0, 1, 1, 7] = float("nan")
        kn[1, 1, 1, 3] = -float("inf")
    for dt in (0, 1):
        _case([4, 0], [5, 4], 5, 2, 64, 16, dt, seed=7, values=odd)


@pytest.mark.parametrize("dt", [0, 1])
def test_graph_replays_and_streams(dt):
    """A page copy and a path append, captured together and replayed with new tokens, against eager
    calls, on the current stream and on another."""
    D = lib()
    g = torch.Generator().manual_seed(11 + dt)
    B, T, Hkv, d, P = 9, 20, 2, 64, 16
    start = [None if x is None else x.cuda() for x in _pool(5 * B, Hkv, d, P, dt, g)]
    kn, vn = (torch.zeros(B, T, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    perm = torch.randperm(5 * B, generator=g).to(torch.int32).numpy()
    bt, src, dst = i32(perm[:4 * B].reshape(B, 4)), i32(perm[4 * B:]), i32(perm[:4 * B].reshape(B, 4)[:, 0])
    before = torch.arange(B, dtype=torch.int32, device="cuda")
    path = torch.randint(0, T, (B, T), generator=g, dtype=torch.int32).cuda()
    counts = (torch.arange(B, dtype=torch.int32, device="cuda") * 3) % (T + 1)
    lens = before + counts

    def calls(pool, status, stream=None):
        kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=dt, k_scales=pool[2], v_scales=pool[3], dev_status=status, stream=stream)
        D.dora_kv_page_copy(pool[0], pool[1], src, dst, head_dim=d, **kw)
        D.dora_kv_append_path(kn, vn, bt, lens, pool[0], pool[1], path=path, counts=counts, **kw)

    clone = lambda: [None if x is None else x.clone() for x in start]  # noqa: E731
    captured, status = clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    calls(clone(), status)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(captured, status)
    for step in range(4):
        for x in (kn, vn):
            x.copy_((torch.randn(x.shape, generator=g) * 2.0 ** (step - 1)).to(torch.bfloat16))
        for x, y in zip(captured, start):
            if x is not None:
                x.copy_(y)
        status.fill_(9)
        graph.replay()
        eager, other = clone(), clone()
        calls(eager, None)
        torch.cuda.synchronize()
        calls(other, None, stream=torch.cuda.Stream())
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for x, y, z in zip(captured, eager, other):
            if x is not None:
                dtype = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
                assert torch.equal(x.view(dtype), y.view(dtype)) and torch.equal(z.view(dtype), y.view(dtype)), step


def test_what_may_not_be_written_is_skipped_and_reported():
    """Bad page ids, lengths, counts and path entries: those pages (or sequences) stay as they
    were, the others are written, and the status says so."""
    D = lib()
    for dt in (0, 1):
        g = torch.Generator().manual_seed(dt)
        Hkv, d, P, T, B, n = 2, 64, 16, 20, 7, 40
        k, v, ks, vs = _pool(n, Hkv, d, P, dt, g)
        kn, vn = (torch.randn(B, T, Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2))
        bt = np.arange(B * 4, dtype=np.int32).reshape(B, 4)
        lens = np.array([20, 20, 65, 20, 3, 40, 30], np.int32)
        counts = np.array([20, 20, 20, -1, 5, 21, 20], np.int32)
        path = np.tile(np.arange(T, dtype=np.int32), (B, 1))
        bt[1, 1] = n        # its second page
        path[6, 19] = T     # its second page (positions 16 .. 29 hold rows 6 .. 19)
        hk, hv = _np(k, dt), _np(v, dt)
        hks, hvs = (None if x is None else x.numpy().copy() for x in (ks, vs))
        kb, vb = _np(kn, 0), _np(vn, 0)
        ok = {0: range(20), 1: range(16), 6: range(6)}
        for b, rows in ok.items():
            first = int(lens[b] - counts[b])
            for i in rows:
                now = np.zeros(B, np.int32)
                now[b] = first + i + 1
                t2 = np.where(bt == n, 0, bt)
                assert oracle.kv_append(kb[:, i], vb[:, i], t2, now, hk, hv, kv_dtype=dt, page_size=P, k_scales=hks,
                                        v_scales=hvs) == 0
        dk, dv = k.cuda(), v.cuda()
        dks, dvs = (None if x is None else x.cuda() for x in (ks, vs))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        D.dora_kv_append_path(kn.cuda(), vn.cuda(), torch.from_numpy(bt).cuda(), torch.from_numpy(lens).cuda(), dk, dv,
                              num_kv_heads=Hkv, page_size=P, kv_dtype=dt, k_scales=dks, v_scales=dvs,
                              path=torch.from_numpy(path).cuda(), counts=torch.from_numpy(counts).cuda(),
                              dev_status=status)
        assert int(status.item()) == D.DORA_ERR_DEVICE_CHECK
        assert _same(_np(dk, dt), hk, dt) and _same(_np(dv, dt), hv, dt)


def test_another_versions_page_is_skipped():
    D = lib()
    g = torch.Generator().manual_seed(1)
    k, v, _, _ = _pool(4, 1, 64, 16, 0, g)
    kn, vn = (torch.randn(2, 3, 1, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    dk, dv = k.cuda(), v.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    D.dora_kv_append_path(kn, vn, i32([[0], [1]]), i32([3, 3]), dk, dv, num_kv_heads=1, page_size=16, version_ids=i32([0, 0]),
                          page_owner=torch.tensor([0, 1, 0, 0], dtype=torch.int16, device="cuda"), flags=D.DORA_FLAG_VALIDATE,
                          dev_status=status)
    assert int(status.item()) == D.DORA_ERR_DEVICE_CHECK
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(dk[1:].cpu(), k[1:]) and same(dv[1:].cpu(), v[1:])
    assert same(dk[0, :, :, :3].permute(2, 0, 1, 3).reshape(3, 1, 64).cpu(), kn[0].cpu())

"""4-bit pages through the C ABI: what appends write bit for bit, what reads give back, decode
attention against 64 bits, packing and copies."""
import numpy as np
import pytest
import torch

import workloads as wl
from cache_util import attend, check
from fp4_util import FP4, Cache4, bf16_of, bf16_value, get_keys, get_values, key_codes, put_keys, put_values, tile_bytes, value_codes
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def _odd_rows(rng, shape):
    """bf16 bits: ordinary rows, rows of very large, very small and subnormal numbers, of zeros, of numbers that tie, and
    rows with infinities and NaN."""
    x = bf16_of(rng.standard_normal(shape) * np.exp(rng.normal(0, 3, shape[:-1] + (1,))))
    flat = x.reshape(-1, shape[-1])
    n = len(flat)
    kinds = rng.integers(0, 12, n)
    for i in range(n):
        r = flat[i]
        if kinds[i] == 0:
            r[:] = bf16_of(rng.standard_normal(len(r)) * 1e38)
        elif kinds[i] == 1:
            r[:] = rng.integers(0, 0x0100, len(r)) | (rng.integers(0, 2, len(r)) << 15)
        elif kinds[i] == 2:
            r[:] = rng.integers(0, 2, len(r)) << 15
        elif kinds[i] == 3:  # halves and quarters: ties of every code
            r[:] = bf16_of(rng.integers(-28, 29, len(r)) / 4.0)
        elif kinds[i] == 4:
            r[rng.integers(0, len(r))] = rng.choice([0x7F80, 0xFF80])
        elif kinds[i] == 5:
            r[rng.integers(0, len(r))] = rng.choice([0x7FC0, 0xFFC1, 0x7F81])
        elif kinds[i] == 6:  # one large number among small ones
            r[rng.integers(0, len(r))] = 0x4F00
        elif kinds[i] == 7:
            r[:] = bf16_of(np.full(len(r), 1.75)) | (rng.integers(0, 2, len(r)) << 15)
    return x


def _expect(c, bits_k, bits_v, rows, counts, lens):
    """The pool's bytes after the tokens (row rows[b][i] of bits [B][T][Hkv][d]) are in."""
    k, v = c.k.numpy().copy(), c.v.numpy().copy()
    for b in range(len(lens)):
        for i in range(counts[b]):
            t = lens[b] - counts[b] + i
            page, slot = int(c.bt[b, t // c.P]), np.array([t % c.P])
            for h in range(c.Hkv):
                put_keys(k[page, h], slot, *key_codes(bits_k[b, rows[b][i], h][None]))
                put_values(v[page, h], slot, *value_codes(bits_v[b, rows[b][i], h][None]))
    return k, v


def _bf16(bits):
    return torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).cuda()


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
def test_single_appends_write_these_bytes(P, d, Hkv):
    print(f"[case] append4 P={P} d={d} Hkv={Hkv}", flush=True)
    rng = np.random.default_rng(P + d + Hkv)
    lens = np.array([0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 64, 5, 7, 8], np.int32)
    c = Cache4(np.maximum(lens - 1, 0), Hkv, d, P, seed=1, extra_tokens=1)
    bits = [_odd_rows(rng, (len(lens), 1, Hkv, d)) for _ in range(2)]
    want = _expect(c, *bits, [[0]] * len(lens), np.minimum(lens, 1), lens)
    dev = c.gpu()
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    lib().dora_kv_append(_bf16(bits[0][:, 0]), _bf16(bits[1][:, 0]), dev["bt"], torch.from_numpy(lens).cuda(), dev["k"], dev["v"],
                         dev_status=status, **dev["kw"])
    assert status.item() == 0
    assert np.array_equal(dev["k"].cpu().numpy(), want[0])
    assert np.array_equal(dev["v"].cpu().numpy(), want[1])


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d,Hkv", [(64, 2), (128, 1), (128, 5)])
@pytest.mark.parametrize("T,path", [(1, False), (9, True), (70, False), (33, True)])
def test_appends_along_a_path_write_these_bytes_and_read_back(P, d, Hkv, T, path):
    print(f"[case] path4 P={P} d={d} Hkv={Hkv} T={T} path={path}", flush=True)
    rng = np.random.default_rng(P + d + Hkv + T)
    base = np.array([0, 0, 1, 5, 15, 16, 17, 31, 32, 47, 200], np.int32)
    counts = np.minimum(T, np.array([0, T, 1, 2, T // 2, T, 3, T, 17, 16, T])).astype(np.int32)
    lens = base + counts
    c = Cache4(base, Hkv, d, P, seed=2, extra_tokens=T)
    rows = [rng.integers(0, T, n) if path else np.arange(n) for n in counts]
    table = np.full((len(lens), T), 2 ** 31 - 1, np.int32)
    for b, r in enumerate(rows):
        table[b, :len(r)] = r
    bits = [_odd_rows(rng, (len(lens), T, Hkv, d)) for _ in range(2)]
    want = _expect(c, *bits, rows, counts, lens)
    dev = c.gpu()
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    lib().dora_kv_append_path(_bf16(bits[0]), _bf16(bits[1]), dev["bt"], i32(lens), dev["k"], dev["v"], path=i32(table) if path else None,
                              counts=i32(counts), dev_status=status, **dev["kw"])
    assert status.item() == 0
    assert np.array_equal(dev["k"].cpu().numpy(), want[0])
    assert np.array_equal(dev["v"].cpu().numpy(), want[1])
    # and back: K's values are bf16 numbers, V's are rounded to them
    out = [torch.full((len(lens), T, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib().dora_kv_read(dev["k"], dev["v"], dev["bt"], i32(lens), *out, counts=i32(counts), dev_status=status, **dev["kw"])
    assert status.item() == 0
    for x, pool, get in ((out[0], want[0], get_keys), (out[1], want[1], get_values)):
        x = _bits(x)
        for b in range(len(lens)):
            assert (x[b, counts[b]:] == 0x40E0).all()
            for i in range(counts[b]):
                t = lens[b] - counts[b] + i
                for h in range(Hkv):
                    y = get(pool[c.bt[b, t // P], h], np.array([t % P]), d)[0]
                    nan = np.isnan(y)
                    assert (np.isnan(bf16_value(x[b, i, h])) == nan).all()
                    # (a code of -0 is -0)
                    assert np.array_equal(np.where(nan, 0, x[b, i, h]), np.where(nan, 0, bf16_of(y)))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
def test_reads_of_bf16_and_fp8_pages(dt, P, d):
    from cache_util import Cache
    Hkv, T = 3, 40
    lens, counts = np.array([0, 1, 40, 77, 100], np.int32), np.array([0, 1, 40, 3, 33], np.int32)
    c = Cache(lens, Hkv, d, P, dt, seed=3)
    dev = c.gpu()
    out = [torch.full((len(lens), T, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib().dora_kv_read(dev["k"], dev["v"], dev["bt"], dev["lens"], *out, counts=torch.from_numpy(counts).cuda(), **dev["kw"])
    for b in range(len(lens)):
        k, v = c.tokens(b, np.arange(lens[b] - counts[b], lens[b]))
        for x, y in zip(out, (k, v)):
            # the fp32 product of a code (4 bits) and a scale, rounded to bf16: the 64-bit product has at most 28
            # bits, so rounding it to fp32 first is the same
            assert np.array_equal(_bits(x[b, :counts[b]]), bf16_of(y))
            assert (_bits(x[b, counts[b]:]) == 0x40E0).all()


def _decode(c, q, **kw):
    dev = c.gpu()
    out = torch.full_like(q, 7.0).cuda()
    lib().dora_decode_attn(q.cuda(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"], **kw)
    torch.cuda.synchronize()
    return out


def _reference(c, q, sm_scale=0.0):
    q = q.float().double().numpy()
    want, spread = np.zeros(q.shape), np.zeros(q.shape)
    for b, L in enumerate(c.lens):
        k, v = c.tokens(b, np.arange(max(0, int(L))))
        o, s = attend(q[b][None], k, v, np.ones((1, len(k)), bool), sm_scale or c.d ** -0.5)
        want[b], spread[b] = o[0], s[0]
    return want, spread


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 300, 1025]


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 7, 16])
@pytest.mark.parametrize("waves", [0, 1, 13, 300])
def test_decode(P, d, G, waves):
    """Whole rows and rows cut anywhere (waves > 0), tails of NaN behind every sequence."""
    print(f"[case] decode4 P={P} d={d} G={G} waves={waves}", flush=True)
    c = Cache4(LENS, 2, d, P, seed=G)
    q = torch.randn(len(LENS), 2 * G, d, generator=torch.Generator().manual_seed(G)).to(torch.bfloat16)
    want, spread = _reference(c, q)
    check(_decode(c, q, num_waves=waves, min_range_pages=1 if waves else 0), want, spread, "decode4")


@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
@pytest.mark.parametrize("lens", [[5000], [3000, 20, 0, 9000], [700] * 40, list(range(0, 600, 3))])
def test_decode_long_and_many(P, d, lens):
    print(f"[case] decode4 P={P} d={d} n={len(lens)} max={max(lens)}", flush=True)
    c = Cache4(lens, 1, d, P, seed=7)
    q = torch.randn(len(lens), 5, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    want, spread = _reference(c, q, 0.3)
    for kw in ({}, {"num_waves": 37}, {"num_waves": 700, "min_range_pages": 2}):
        check(_decode(c, q, sm_scale=0.3, **kw), want, spread, f"decode4 {kw}")


def test_queries_far_from_one_and_odd_keys():
    """Query rows whose values spread over 30 powers of two, zero rows, keys that are zero; a NaN key or value reaches
    its head's rows alone, and a NaN or infinite query its own."""
    c = Cache4([40, 130, 64, 9], 2, 128, 16, seed=5)
    q = torch.randn(4, 8, 128, generator=torch.Generator().manual_seed(1))
    q[0] *= torch.exp2(torch.randint(-28, 3, q[0].shape, generator=torch.Generator().manual_seed(2)).float())
    q[1, :3] = 0
    q[1, 3] *= 1e-30
    q = q.to(torch.bfloat16)
    for h in range(2):
        x = np.zeros((1, 128), np.uint16)
        put_keys(c.k[int(c.bt[1, 2]), h].numpy(), np.array([5]), *key_codes(x))
    want, spread = _reference(c, q)
    check(_decode(c, q), want, spread, "far")
    q[2, 6, 3] = float("nan")
    q[2, 7, 100] = float("inf")
    x = np.full((1, 128), 0x7FC0, np.uint16)
    put_keys(c.k[int(c.bt[0, 1]), 0].numpy(), np.array([2]), *key_codes(x))
    put_values(c.v[int(c.bt[1, 0]), 1].numpy(), np.array([15]), *value_codes(x))
    want[2, 6:] = np.nan
    want[0, :4] = np.nan
    want[1, 4:] = np.nan
    for kw in ({}, {"num_waves": 5}):
        check(_decode(c, q, **kw), want, spread, f"odd {kw}")


def test_noalloc_prepared_and_validated_calls_equal_the_plain_one():
    D = lib()
    c = Cache4([700, 0, 33, 1200], 2, 128, 32, seed=9)
    q = torch.randn(4, 12, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    dev = c.gpu()
    outs = [torch.empty_like(q) for _ in range(4)]
    a = (q, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
    D.dora_decode_attn(*a, outs[0], **dev["kw"])
    D.dora_decode_attn_noalloc(*a, outs[1], **dev["kw"])
    D.PreparedDecode(*a, outs[2], **dev["kw"])()
    D.dora_decode_attn(*a, outs[3], flags=D.DORA_FLAG_VALIDATE, **dev["kw"])
    assert all(torch.equal(outs[0], x) for x in outs[1:])
    bad = dev["bt"].clone()
    bad[3, 7] = c.num_pages
    with pytest.raises(D.DoraError) as e:
        D.dora_decode_attn(q, dev["k"], dev["v"], bad, dev["lens"], None, outs[3], flags=D.DORA_FLAG_VALIDATE, **dev["kw"])
    assert e.value.status == D.DORA_ERR_DEVICE_CHECK


@pytest.mark.parametrize("P,d,Hkv", [(16, 64, 1), (32, 128, 8), (16, 128, 3)])
def test_pages_pack_unpack_and_copy_as_bytes(P, d, Hkv):
    D = lib()
    g = torch.Generator().manual_seed(P)
    n, size = 37, tile_bytes(d, P)
    pool = [torch.randint(0, 256, (n, Hkv, size), generator=g, dtype=torch.uint8) for _ in range(2)]
    kw = dict(num_kv_heads=Hkv, page_size=P, head_dim=d, kv_dtype=FP4)
    k, v = (x.cuda() for x in pool)
    src, dst = torch.randperm(n, generator=g)[:20].to(torch.int32), torch.randperm(n, generator=g)[:20].to(torch.int32)
    desc = D.make_pack_desc(kv_dtype=FP4, page_size=P, num_kv_heads=Hkv, head_dim=d, num_pages=n, policy_version=0)
    need = D.dora_kv_packed_bytes(desc, 20)
    assert need == 256 + 2 * 20 * Hkv * size
    packed = torch.empty(need, dtype=torch.uint8, device="cuda")
    D.dora_kv_page_pack(k, v, src.cuda(), packed, **kw)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    D.dora_kv_page_unpack(packed, dst.cuda(), k2, v2, src_version=0, **kw)
    for x, y in ((k2, pool[0]), (v2, pool[1])):
        assert torch.equal(x[dst.long().cuda()].cpu(), y[src.long()])
    a, b = torch.tensor([1, 5, 1], dtype=torch.int32), torch.tensor([30, 31, 32], dtype=torch.int32)
    D.dora_kv_page_copy(k, v, a.cuda(), b.cuda(), **kw)
    for x, y in ((k, pool[0]), (v, pool[1])):
        y = y.clone()
        y[b.long()] = y[a.long()]
        assert torch.equal(x.cpu(), y)


def test_pages_behind_four_gigabytes():
    """Pages whose byte offsets pass 32 bits, written, read back and attended."""
    D, P, d, Hkv, n = lib(), 32, 128, 8, 260000  # 4.5 GB of K
    size = tile_bytes(d, P)
    k, v = (torch.empty((n, Hkv, size), dtype=torch.uint8, device="cuda") for _ in range(2))
    bt = torch.tensor([[n - 1, 7, 250001, 130000], [n - 3, 247000, 3, n - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([100, 128], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(4)
    kn, vn = (torch.randn(2, 128, Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2))
    kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=FP4)
    D.dora_kv_append_path(kn.cuda(), vn.cuda(), bt, lens, k, v, counts=lens, **kw)
    ko, vo = torch.zeros_like(kn).cuda(), torch.zeros_like(vn).cuda()
    D.dora_kv_read(k, v, bt, lens, ko, vo, counts=lens, **kw)
    c = Cache4([100, 128], 1, 64, 32)  # only its helpers
    q = torch.randn(2, 16, d, generator=g).to(torch.bfloat16)
    out = torch.empty_like(q).cuda()
    D.dora_decode_attn(q.cuda(), k, v, bt, lens, None, out, **kw)
    want, spread = np.zeros(q.shape), np.zeros(q.shape)
    for b, L in enumerate((100, 128)):
        kb, vb = _bits(kn[b, :L]), _bits(vn[b, :L])
        codes, e = key_codes(kb)
        from fp4_util import dec4
        kk = dec4(codes) * np.repeat(np.exp2(e - 127.0), 32, axis=-1)
        codes, s = value_codes(vb)
        vv = dec4(codes) * np.repeat(bf16_value(s).astype(np.float64), 64, axis=-1)
        assert np.array_equal(_bits(ko[b, :L]), bf16_of(kk)) and np.array_equal(_bits(vo[b, :L]), bf16_of(vv))
        o, sp = attend(q[b].float().double().numpy()[None], kk, vv, np.ones((1, L), bool), d ** -0.5)
        want[b], spread[b] = o[0], sp[0]
    check(out, want, spread, "far pages")
    assert c.num_pages > 0


def test_what_is_skipped_stays():
    """Counts and lengths that fit no row, pages outside the pool, path entries that are no row: reported, nothing
    written; the rest is."""
    D, P, d, Hkv, T = lib(), 16, 64, 2, 20
    base = np.array([0, 10, 30, 5, 16, 3], np.int32)
    counts = np.array([-1, 21, 5, 8, 20, 4], np.int32)
    lens = np.array([10, 31, 3, 13, 36, 7], np.int32)  # (2: fewer than its count)
    c = Cache4(base, Hkv, d, P, seed=2, extra_tokens=T)
    c.bt[4, 1] = -5
    rng = np.random.default_rng(1)
    bits = [_odd_rows(rng, (6, T, Hkv, d)) for _ in range(2)]
    path = np.tile(np.arange(T, dtype=np.int32), (6, 1))
    path[5, 2] = T
    rows = [[]] * 3 + [path[3], path[4], []]
    good = c.bt.copy()
    good[4, 1] = 0
    keep = c.bt
    some = np.array([0, 0, 0, 8, 20, 0], np.int32)
    k0, v0 = c.k.numpy().copy(), c.v.numpy().copy()
    # sequence 4: tokens 16 .. 31 lie in the bad page, 32 .. 35 behind it are written
    c.bt = good
    want = _expect(c, *bits, [r if i != 4 else [] for i, r in enumerate(rows)], np.where(np.arange(6) == 4, 0, some), lens)
    c.k, c.v = torch.from_numpy(want[0]), torch.from_numpy(want[1])
    want = _expect(c, *bits, [path[b][16:] if b == 4 else [] for b in range(6)], np.array([0, 0, 0, 0, 4, 0]), lens)
    c.k, c.v, c.bt = torch.from_numpy(k0), torch.from_numpy(v0), keep
    dev = c.gpu()
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    D.dora_kv_append_path(_bf16(bits[0]), _bf16(bits[1]), dev["bt"], i32(lens), dev["k"], dev["v"], path=i32(path), counts=i32(counts),
                          dev_status=status, **dev["kw"])
    assert status.item() == D.DORA_ERR_DEVICE_CHECK
    assert np.array_equal(dev["k"].cpu().numpy(), want[0]) and np.array_equal(dev["v"].cpu().numpy(), want[1])
    out = [torch.full((6, T, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dora_kv_read(dev["k"], dev["v"], dev["bt"], i32(lens), *out, counts=i32(counts), dev_status=status, **dev["kw"])
    assert status.item() == D.DORA_ERR_DEVICE_CHECK
    for x in out:
        x = _bits(x) != 0x40E0
        assert not x[:3].any() and x[3, :8].any() and not x[3, 8:].any()
        assert not x[4, :16].any() and x[4, 16:].any()


def test_page_owners():
    D = lib()
    c = Cache4([20, 20], 2, 64, 16, seed=2, extra_tokens=4)
    dev = c.gpu()
    owner = np.full(c.num_pages, 3, np.int16)
    owner[c.bt[1, 1]] = 9
    kw = dict(version_ids=torch.tensor([3, 3], dtype=torch.int32, device="cuda"), page_owner=torch.from_numpy(owner).cuda(),
              flags=D.DORA_FLAG_VALIDATE, **dev["kw"])
    k0 = dev["k"].clone()
    x = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor([21, 21], dtype=torch.int32, device="cuda")
    D.dora_kv_append(x, x, dev["bt"], lens, dev["k"], dev["v"], dev_status=status, **kw)
    assert status.item() == D.DORA_ERR_DEVICE_CHECK
    changed = (dev["k"] != k0).flatten(1).any(1).cpu().numpy()
    assert changed[c.bt[0, 1]] and changed.sum() == 1


def test_captured_steps_replayed():
    """Append, bounds, selection and attention over the listed pages, captured once and replayed with other inputs: each
    replay equals the eager calls bit for bit, with eager work between."""
    D, B, Hkv, Hq, d, P, steps, budget = lib(), 5, 2, 8, 128, 16, 5, 4
    L0 = np.array([0, 15, 64, 300, 1000], np.int32)
    c = Cache4(L0, Hkv, d, P, seed=4, extra_tokens=steps)
    g = torch.Generator().manual_seed(5)
    qs, kn, vn = (torch.randn(steps, B, h, d, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    lens = [torch.from_numpy(L0 + 1 + s).cuda() for s in range(steps)]
    rec = D.dora_page_bounds_bytes(Hkv, d)

    def state():
        dev = c.gpu()
        bounds = torch.zeros(c.num_pages, rec, dtype=torch.uint8, device="cuda")
        full = torch.from_numpy(L0).cuda()
        D.dora_kv_page_bounds(dev["k"], dev["bt"], full, bounds, num_tokens=1000, head_dim=d, counts=full, num_kv_heads=Hkv, page_size=P, kv_dtype=FP4)
        return dict(dev, bounds=bounds, q=torch.empty_like(qs[0]), kn=torch.empty_like(kn[0]), vn=torch.empty_like(vn[0]),
                    ln=lens[0].clone(), out=torch.zeros_like(qs[0]), dense=torch.zeros_like(qs[0]),
                    lists=torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda"),
                    counts=torch.zeros(B, Hkv, dtype=torch.int32, device="cuda"))

    def step(s):
        kw = s["kw"]
        D.dora_kv_append(s["kn"], s["vn"], s["bt"], s["ln"], s["k"], s["v"], **kw)
        D.dora_kv_page_bounds(s["k"], s["bt"], s["ln"], s["bounds"], num_tokens=1, head_dim=d, num_kv_heads=Hkv, page_size=P, kv_dtype=FP4)
        D.dora_page_select(s["q"], s["bounds"], s["bt"], s["ln"], s["lists"], s["counts"], num_kv_heads=Hkv, page_size=P)
        D.dora_decode_attn_pages(s["q"], s["lists"], s["counts"], s["k"], s["v"], s["bt"], s["ln"], None, s["out"], **kw)
        D.dora_decode_attn(s["q"], s["k"], s["v"], s["bt"], s["ln"], None, s["dense"], **kw)

    def inputs(s, i):
        for name, x in (("q", qs), ("kn", kn), ("vn", vn), ("ln", lens)):
            s[name].copy_(x[i])

    captured, eager = state(), state()
    for s in (captured, eager):
        inputs(s, 0)
        step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for i in range(1, steps):
        inputs(captured, i)
        inputs(eager, i)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for name in ("k", "v", "bounds", "lists", "counts", "out", "dense"):
            assert torch.equal(captured[name], eager[name]), (i, name)
        float(torch.randn(1000, device="cuda").sum())

"""4-bit and listed pages in batches of more sequences than a launch covers, by every route of the 4-bit decode, and with
neighbours at work: other streams, graphs, empty rows."""
import numpy as np
import pytest
import torch

from cache_util import bound, check
from fp4_util import FP4, Cache4, bf16_of, bf16_value, dec4, key_codes, make_cache, value_codes
from gpu_util import lib
from test_gpu_fp4 import _reference as _dense_reference
from test_gpu_pages import LENS, TYPES, _hide, _lists, _q, _reference
from test_gpu_select import _bounds, _record, _select, _tokens32

pytestmark = pytest.mark.gpu


def _tiled(c, B):
    """The sequences of c again and again up to B rows, over the same pages."""
    at = np.arange(B) % len(c.lens)
    dev = c.gpu()
    dev["bt"], dev["lens"] = (dev[n][torch.from_numpy(at).cuda()].contiguous() for n in ("bt", "lens"))
    return dev, torch.from_numpy(at)


def _check_tiled(out, at, want, spread, what):
    """Every row against the 64-bit row that it repeats."""
    got = out.float().cpu().double()
    limit = torch.from_numpy(bound(want, spread))
    assert not got.isnan().any()
    off = (got - torch.from_numpy(want)[at]).abs() - limit[at]
    assert float(off.max()) <= 0, f"{what}: {float(off.max())} beyond the bound"


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("B", [8192, 8193, 20000])
def test_more_sequences_than_a_launch_covers(dt, B):
    print(f"[case] batches dt={dt} B={B}", flush=True)
    D, Hkv, G, d, P, budget = lib(), 2, 2, 64, 16, 3
    c = make_cache([0, 1, 40, 17, 100, 64, 300], Hkv, d, P, dt, seed=3)
    dev, at = _tiled(c, B)
    q = _q(len(c.lens), Hkv * G, d, 1)
    qd = q[at].cuda().contiguous()
    bounds = torch.zeros(c.num_pages, D.dora_page_bounds_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    small = c.gpu()
    bkw = {k: v for k, v in dev["kw"].items() if k != "v_scales"}
    D.dora_kv_page_bounds(small["k"], small["bt"], small["lens"], bounds, num_tokens=300, head_dim=d, counts=small["lens"], **bkw)
    lists = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    counts = torch.full((B, Hkv), -1, dtype=torch.int32, device="cuda")
    few = torch.full((7, Hkv, budget), -1, dtype=torch.int32, device="cuda"), torch.full((7, Hkv), -1, dtype=torch.int32, device="cuda")
    args = dict(num_kv_heads=Hkv, page_size=P)
    D.dora_page_select(q.cuda(), bounds, small["bt"], small["lens"], *few, **args)
    for scores in (False, True):
        lists.fill_(-1)
        sc = torch.zeros(B, Hkv, dev["bt"].shape[1], device="cuda") if scores else None
        D.dora_page_select(qd, bounds, dev["bt"], dev["lens"], lists, counts, scores=sc, **args)
        assert torch.equal(lists.cpu(), few[0].cpu()[at]) and torch.equal(counts.cpu(), few[1].cpu()[at])
    want, spread = _reference(c, q, few[0].cpu().numpy(), few[1].cpu().numpy())
    out = torch.full_like(qd, 7.0)
    D.dora_decode_attn_pages(qd, lists, counts, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"])
    _check_tiled(out, at, want, spread, "pages")
    D.dora_decode_attn_pages(qd, lists, counts, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, flags=D.DORA_FLAG_VALIDATE,
                             **dev["kw"])
    _check_tiled(out, at, want, spread, "validated pages")
    if dt == FP4:
        out.fill_(7.0)
        D.dora_decode_attn(qd, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"])
        _check_tiled(out, at, *_dense_reference(c, q), "decode4")
    last = counts.clone()
    last[B - 1, 1] = budget + 1  # in the last launch
    with pytest.raises(D.DoraError) as e:
        D.dora_decode_attn_pages(qd, lists, last, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, flags=D.DORA_FLAG_VALIDATE,
                                 **dev["kw"])
    assert e.value.status == D.DORA_ERR_DEVICE_CHECK


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,width", [(1, 1), (4, 3), (16, 8), (7, 150)])
def test_lists_of_many_segments(dt, P, d, G, width):
    """As many lists as make a wave each the better way where they are short."""
    print(f"[case] many lists dt={dt} P={P} d={d} G={G} width={width}", flush=True)
    c = make_cache(LENS, 2, d, P, dt, seed=width)
    q = _q(len(LENS), 2 * G, d, G)
    lists, counts = _lists(np.random.default_rng(G + width), c, width, 2)
    want, spread = _reference(c, q, lists, counts)
    _hide(c, lists, counts)
    dev, at = _tiled(c, 330)
    out = torch.full((330, 2 * G, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lib().dora_decode_attn_pages(q[at].cuda().contiguous(), torch.from_numpy(lists)[at].cuda().contiguous(),
                                 torch.from_numpy(counts)[at].cuda().contiguous(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, out,
                                 **dev["kw"])
    _check_tiled(out, at, want, spread, "pages")


@pytest.mark.parametrize("one", [False, True])
def test_stores_and_reads_of_more_sequences_than_a_launch_covers(one):
    """33,000 sequences with a page of their own: stored bit for bit as their rows say, read back, and bounded."""
    D, B, d, P = lib(), 33000, 64, 16
    T = 1 if one else 3
    rng = np.random.default_rng(4)
    bits = [bf16_of(rng.standard_normal((B, T, 1, d))) for _ in range(2)]
    perm = rng.permutation(B).astype(np.int32)
    dev = {n: torch.full((B, 1, P * d * 17 // 32), 0xFF, dtype=torch.uint8, device="cuda") for n in "kv"}
    bt = torch.from_numpy(perm[:, None]).cuda()
    lens = torch.full((B,), T, dtype=torch.int32, device="cuda")
    kw = dict(num_kv_heads=1, page_size=P, kv_dtype=FP4)
    new = [torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda() for x in bits]
    if one:
        D.dora_kv_append(new[0][:, 0], new[1][:, 0], bt, lens, dev["k"], dev["v"], **kw)
    else:
        D.dora_kv_append_path(*new, bt, lens, dev["k"], dev["v"], **kw)
    out = [torch.zeros(B, T, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dora_kv_read(dev["k"], dev["v"], bt, lens, *out, **kw)
    ck, ek = key_codes(bits[0])
    cv, sv = value_codes(bits[1])
    k = dec4(ck) * np.repeat(np.exp2(ek.astype(np.float64) - 127), 32, axis=-1)
    v = dec4(cv) * np.repeat(bf16_value(sv).astype(np.float64), 64, axis=-1)
    for x, y in zip(out, (k, v)):
        assert np.array_equal(x.cpu().view(torch.int16).numpy().view(np.uint16), bf16_of(y))
    bounds = torch.zeros(B, D.dora_page_bounds_bytes(1, d), dtype=torch.uint8, device="cuda")
    D.dora_kv_page_bounds(dev["k"], bt, lens, bounds, num_tokens=T, head_dim=d, **kw)
    got = bounds.cpu().numpy()
    for b in (0, 8191, 8192, 32767, 32768, B - 1):
        assert np.array_equal(got[perm[b], :2 * d + 4], _record(*_bounds(k[b]))[:2 * d + 4])
    seen = got[perm, 2 * d:2 * d + 4].copy().view(np.float32)[:, 0]  # every page's scale
    top = np.abs(k).max((1, 2, 3)).astype(np.float32) / np.float32(127)
    assert np.array_equal(seen, top)


ROUTES = [  # rows, KV heads, longest row, pages of 16 tokens in a workgroup: whole rows (None), chunks, and 0
    (5, 2, 900, None), (2000, 1, 60, None), (5, 2, 1500, 16), (100, 2, 2300, None), (6, 2, 6000, 32), (40, 1, 4500, 64), (12, 2, 15000, 64),
    (3, 1, 32000, 32), (300, 2, 2700, 0), (1100, 2, 200, None), (700, 1, 740, None), (400, 8, 1500, None), (400, 8, 1600, 0)]


@pytest.mark.parametrize("B,Hkv,longest,pages", ROUTES)
@pytest.mark.parametrize("d", [64, 128])
def test_routes_of_the_4_bit_decode(B, Hkv, longest, pages, d):
    print(f"[case] route B={B} Hkv={Hkv} longest={longest} d={d}", flush=True)
    D, G = lib(), 3
    c = Cache4([longest, 0, longest // 3, 1, longest // 2 + 1], Hkv, d, 16, seed=5)
    dev, at = _tiled(c, B)
    q = _q(5, Hkv * G, d, 2)
    qd = q[at].cuda().contiguous()
    width = dev["bt"].shape[1]
    desc = D.make_decode_desc(num_seqs=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, page_size=16, block_table_stride=width,
                              num_pages=c.num_pages, kv_dtype=FP4)
    assert D.dora_decode_segment_pages(desc) == (width if pages is None else pages)
    want, spread = _dense_reference(c, q)
    out = torch.full_like(qd, 7.0)
    D.dora_decode_attn(qd, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"])
    _check_tiled(out, at, want, spread, "decode4")


def test_two_graphs_on_two_streams():
    """Two captured runs over chunked lists and cut rows, replayed at once on streams of their own, with eager calls of
    the same shapes between: each equals its own eager run."""
    D = lib()
    runs = []
    for i in range(2):
        c = make_cache([9000, 300, 5000], 2, 64, 16, FP4, seed=i)
        dev = c.gpu()
        if i:  # a table so wide that the choice takes two launches and their workspace
            dev["bt"] = torch.nn.functional.pad(dev["bt"], (0, 1100 - dev["bt"].shape[1])).contiguous()
        q = _q(3, 8, 64, i).cuda()
        n = -(-c.lens // 16)
        width = int(n.max())
        lists = torch.arange(width, dtype=torch.int32).repeat(3, 2, 1).cuda()
        counts = torch.from_numpy(np.tile(n[:, None], (1, 2)).astype(np.int32)).cuda()
        bounds = torch.randint(0, 100, (c.num_pages, D.dora_page_bounds_bytes(2, 64)), generator=torch.Generator().manual_seed(i),
                               dtype=torch.uint8).cuda()
        picked = torch.zeros(3, 2, 9, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda")
        outs = [torch.zeros_like(q) for _ in range(2)]

        def step(c=c, dev=dev, q=q, lists=lists, counts=counts, bounds=bounds, picked=picked, outs=outs, stream=None):
            D.dora_page_select(q, bounds, dev["bt"], dev["lens"], *picked, num_kv_heads=2, page_size=16, stream=stream)
            D.dora_decode_attn_pages(q, lists, counts, dev["k"], dev["v"], dev["bt"], dev["lens"], None, outs[0], stream=stream, **dev["kw"])
            D.dora_decode_attn(q, dev["k"], dev["v"], dev["bt"], dev["lens"], None, outs[1], stream=stream, **dev["kw"])

        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in (*outs, *picked)]
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            step()
        runs.append((graph, stream, step, (*outs, *picked), eager))
    for _ in range(5):
        for _, _, _, outs, _ in runs:
            for x in outs:
                x.zero_()
        torch.cuda.synchronize()
        for graph, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, _, outs, eager in runs:
            assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        for _, _, step, outs, eager in runs:
            step()
        torch.cuda.synchronize()
        for _, _, _, outs, eager in runs:
            assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@pytest.mark.parametrize("dt", TYPES)
def test_far_pages_are_read_as_near_ones(dt):
    """The same pages within 4 GB of the pool's start and behind: reads, bounds, attention over lists (four waves and one a
    list) and, of 4-bit pages, the decode by ranges are equal bit for bit."""
    D, Hkv, d, P = lib(), 2, 128, 32
    c = make_cache([900, 33, 0, 257], Hkv, d, P, dt, seed=9)
    near = c.gpu()
    page = near["k"][0].numel() * near["k"].element_size()
    far = (1 << 32) // page + 5  # the first page that begins behind 4 GB
    pool = {}
    for n in "kv":
        big = torch.empty((far + c.num_pages, *near[n].shape[1:]), dtype=near[n].dtype, device="cuda")
        big[far:] = near[n]
        pool[n] = big
    kw = dict(near["kw"])
    if dt == 1:
        for n in ("k_scales", "v_scales"):
            kw[n] = torch.cat([torch.full((far,), float("nan"), device="cuda"), near["kw"][n]])
    bt = (near["bt"] + far).contiguous()
    lens = near["lens"]
    rec = D.dora_page_bounds_bytes(Hkv, d)
    bounds = [torch.zeros(n, rec, dtype=torch.uint8, device="cuda") for n in (c.num_pages, far + c.num_pages)]
    rows = [[torch.zeros(4, 900, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    for i, (k, v, t, w) in enumerate(((near["k"], near["v"], near["bt"], near["kw"]), (pool["k"], pool["v"], bt, kw))):
        D.dora_kv_read(k, v, t, lens, *rows[i], counts=lens, **w)
        D.dora_kv_page_bounds(k, t, lens, bounds[i], num_tokens=900, head_dim=d, counts=lens, **{n: x for n, x in w.items() if n != "v_scales"})
    assert torch.equal(bounds[0], bounds[1][far:])
    for a, b in zip(*rows):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    for B in (4, 330):
        at = (torch.arange(B) % 4).cuda()
        q = _q(4, Hkv * 3, d, 2).cuda()[at].contiguous()
        lists = torch.arange(6, dtype=torch.int32, device="cuda").repeat(B, Hkv, 1).contiguous()
        counts = torch.full((B, Hkv), 6, dtype=torch.int32, device="cuda")
        outs = [torch.zeros_like(q) for _ in range(4)]
        D.dora_decode_attn_pages(q, lists, counts, near["k"], near["v"], near["bt"][at].contiguous(), lens[at].contiguous(), None, outs[0], **near["kw"])
        D.dora_decode_attn_pages(q, lists, counts, pool["k"], pool["v"], bt[at].contiguous(), lens[at].contiguous(), None, outs[1], **kw)
        D.dora_decode_attn(q, near["k"], near["v"], near["bt"][at].contiguous(), lens[at].contiguous(), None, outs[2], num_waves=9, **near["kw"])
        D.dora_decode_attn(q, pool["k"], pool["v"], bt[at].contiguous(), lens[at].contiguous(), None, outs[3], num_waves=9, **kw)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3]) and not outs[0].isnan().any()


@pytest.mark.parametrize("dt", TYPES)
def test_as_many_kv_heads_as_there_may_be(dt):
    """127 KV heads: waves of a workgroup take several, the choice its last pair alone."""
    D, Hkv, d, P = lib(), 127, 64, 16
    c = make_cache([40, 0, 17], Hkv, d, P, dt, seed=2)
    dev = c.gpu()
    bounds = torch.zeros(c.num_pages, D.dora_page_bounds_bytes(Hkv, d), dtype=torch.uint8, device="cuda")
    D.dora_kv_page_bounds(dev["k"], dev["bt"], dev["lens"], bounds, num_tokens=40, head_dim=d, counts=dev["lens"],
                          **{n: x for n, x in dev["kw"].items() if n != "v_scales"})
    for b, j in ((0, 0), (0, 2), (2, 1)):
        t = np.arange(j * P, min(int(c.lens[b]), (j + 1) * P))
        used = Hkv * (2 * d + 4)
        assert np.array_equal(bounds[int(c.bt[b, j])].cpu().numpy()[:used], _record(*_bounds(_tokens32(c, b, t)))[:used])
    out = [torch.zeros(3, 40, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    D.dora_kv_read(dev["k"], dev["v"], dev["bt"], dev["lens"], *out, counts=dev["lens"], **dev["kw"])
    for b, L in enumerate(c.lens):
        for x, y in zip(out, c.tokens(b, np.arange(L))):
            assert np.array_equal(x[b, :L].cpu().view(torch.int16).numpy().view(np.uint16), bf16_of(y))
    q = _q(3, Hkv * 2, d, 4)
    lists = np.tile(np.array([2, 0], np.int32), (3, Hkv, 1))
    counts = np.full((3, Hkv), 2, np.int32)
    want, spread = _reference(c, q, lists, counts)
    got = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    D.dora_decode_attn_pages(q.cuda(), torch.from_numpy(lists).cuda(), torch.from_numpy(counts).cuda(), dev["k"], dev["v"], dev["bt"],
                             dev["lens"], None, got, **dev["kw"])
    check(got, want, spread, "pages")
    if dt == FP4:
        for waves in (0, 40):
            D.dora_decode_attn(q.cuda(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, got, num_waves=waves, **dev["kw"])
            check(got, *_dense_reference(c, q), "decode4")
        k, v = torch.full_like(dev["k"], 0xFF), torch.full_like(dev["v"], 0xFF)
        D.dora_kv_append_path(*out, dev["bt"], dev["lens"], k, v, counts=dev["lens"], **dev["kw"])
        again = [torch.zeros_like(x) for x in out]
        D.dora_kv_read(k, v, dev["bt"], dev["lens"], *again, counts=dev["lens"], **dev["kw"])
        # a block's largest K is at least 4 steps and at most 6, so that K's values are stored again as they are
        assert torch.equal(out[0].view(torch.int16), again[0].view(torch.int16))
    for width in (0, 1025):
        _select([300, 77, 0], Hkv, 1, d, P, 5, 1, 1, seed=3, width=width)

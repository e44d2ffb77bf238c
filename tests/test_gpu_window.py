"""dora_decode_attn_window through the C ABI against the operator written down in 64 bits."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check, odd_scales, window_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _q(B, Hq, d, seed):
    return torch.randn(B, Hq, d, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _hide(c, window, sinks):
    """NaN in every slot that does not count; entries of pages without one that does point
    outside the pool."""
    for b, L in enumerate(c.lens):
        for j in range(-(-int(L) // c.P)):
            t = np.arange(j * c.P, min((j + 1) * c.P, int(L)))
            off = t[~((t < sinks) | (t >= int(L) - window))]
            pg = int(c.bt[b, j])
            for x in (off % c.P):
                c.k[pg, :, :, x] = float("nan") if c.dt == 0 else 0x7F
                c.v[pg, :, :, x] = float("nan") if c.dt == 0 else 0x7F
            if len(off) == len(t):
                c.bt[b, j] = 2 ** 31 - 1


def _case(lens, window, sinks, Hkv, G, d, P, dt, seed, **kw):
    print(f"[case] window={window} sinks={sinks} Hkv={Hkv} G={G} d={d} P={P} dt={dt} n={len(lens)} {kw}", flush=True)
    c = Cache(lens, Hkv, d, P, dt, seed=seed)
    q = _q(len(lens), Hkv * G, d, seed + 1)
    want, spread = window_reference(c, q, window, sinks, kw.get("sm_scale", 0.0))
    _hide(c, window, sinks)
    dev = c.gpu()
    out = torch.full_like(q, 7.0).cuda()
    lib().dora_decode_attn_window(q.cuda(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, window=window,
                                  sinks=sinks, **dev["kw"], **kw)
    torch.cuda.synchronize()
    check(out, want, spread, "window")
    return out


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 300, 1000, 1025]


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (33, 16), (100, 40), (512, 1), (2000, 7)])
def test_windows(dt, P, d, window, sinks):
    _case(LENS, window, sinks, 2, 4, d, P, dt, seed=window + sinks + P + dt)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("G", [1, 7, 16])
def test_groups_and_many_segments(dt, G):
    """More (sequence, KV head) segments than workgroups fit the chip at once."""
    rng = np.random.default_rng(G)
    _case(rng.integers(0, 200, 300), 50, 5, 2, G, 64, 16, dt, seed=G)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
def test_wide_windows_in_chunks(dt, P):
    """Windows wider than a workgroup's pages, over rows shorter and longer."""
    _case([9000, 20, 5200, 0, 12000], 5000, 100, 1, 4, 64, P, dt, seed=P + dt)


def test_window_past_every_row_is_the_plain_decode():
    D = lib()
    c = Cache([5, 100, 640, 0, 31], 2, 128, 16, 0, seed=3)
    q, dev = _q(5, 8, 128, 4).cuda(), c.gpu()
    out, plain = torch.empty_like(q), torch.empty_like(q)
    a = (q, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
    for window, sinks in ((2 ** 31 - 1, 0), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1), (640, 0)):
        D.dora_decode_attn_window(*a, out, window=window, sinks=sinks, **dev["kw"])
        D.dora_decode_attn(*a, plain, **dev["kw"])
        want, spread = window_reference(c, q.cpu(), 640, 0)
        check(out, want, spread)
        check(plain, want, spread)


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 150])
def test_odd_scales(d, P, n):
    """n = 150: many segments."""
    c = Cache([300, 100, 90, 211, 64, 50, 33] * n, 4, d, P, 1, seed=d + P)
    odd_scales(c)
    q = _q(7 * n, 8, d, P)
    want, spread = window_reference(c, q, 70, 20)
    dev = c.gpu()
    out = torch.empty_like(q).cuda()
    lib().dora_decode_attn_window(q.cuda(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, window=70, sinks=20, **dev["kw"])
    check(out, want, spread, "window", roundings=2)


def test_infinite_scores():
    """Keys of -inf inside the window, and +inf and NaN outside of it."""
    c = Cache([100, 300], 1, 64, 16, 0, seed=5)
    q = _q(2, 2, 64, 6)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    c.k[c.bt[0, 5], :, 0, :, 0] = -float("inf")
    c.k[c.bt[1, 3], :, 0, :, 0] = float("inf")
    for window in (40, 20):  # (the page of -inf alone in the second's front)
        want, spread = window_reference(c, q, window, 2)
        dev = c.gpu()
        out = torch.empty_like(q).cuda()
        lib().dora_decode_attn_window(q.cuda(), dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, window=window,
                                      sinks=2, **dev["kw"])
        assert np.isfinite(want).all()
        check(out, want, spread)


def test_validate_looks_at_what_is_read():
    D = lib()
    c = Cache([300], 1, 64, 16, 0, seed=7)
    q, out = _q(1, 2, 64, 8).cuda(), torch.empty(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    c.bt[0, 5] = -1  # between the sinks and the window
    owner = torch.full((c.num_pages,), 2, dtype=torch.int16, device="cuda")
    vers = torch.tensor([2], dtype=torch.int32, device="cuda")
    kw = dict(window=100, sinks=4, flags=D.DORA_FLAG_VALIDATE, page_owner=owner)
    dev = c.gpu()
    D.dora_decode_attn_window(q, dev["k"], dev["v"], dev["bt"], dev["lens"], vers, out, **kw, **dev["kw"])
    for j, bad in ((15, c.num_pages), (0, -1)):
        bt = dev["bt"].clone()
        bt[0, j] = bad
        with pytest.raises(D.DoraError) as e:
            D.dora_decode_attn_window(q, dev["k"], dev["v"], bt, dev["lens"], vers, out, **kw, **dev["kw"])
        assert e.value.status == D.DORA_ERR_DEVICE_CHECK
    owner[int(c.bt[0, 18])] = 1
    with pytest.raises(D.DoraError):
        D.dora_decode_attn_window(q, dev["k"], dev["v"], dev["bt"], dev["lens"], vers, out, **kw, **dev["kw"])
    with pytest.raises(D.DoraError):
        D.dora_decode_attn_window(q, dev["k"], dev["v"], dev["bt"], dev["lens"] + 20, vers, out, **kw, **dev["kw"])


def test_many_sequences_take_several_launches():
    rng = np.random.default_rng(9)
    _case(rng.integers(0, 40, 8200), 10, 1, 1, 1, 64, 16, 0, seed=10)


def test_graph_replays_and_streams():
    D = lib()
    sets = []
    for n, (lens, window) in enumerate([([3000, 20, 900], 1500), ([70, 1200, 5, 5], 600)]):
        c = Cache(lens, 2, 64, 16, 1, seed=25 + n)
        dev, q = c.gpu(), _q(len(lens), 8, 64, n).cuda()
        a = (q, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
        kw = dict(dev["kw"], window=window, sinks=3)
        out = D.dora_decode_attn_window(*a, torch.empty_like(q), **kw)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.dora_decode_attn_window(*a, out, **kw)
        sets.append((a, out, graph, kw))
    s = torch.cuda.Stream()
    for step in range(4):
        for a, out, graph, kw in sets:
            a[0].copy_(torch.randn_like(a[0].float()).to(torch.bfloat16))
            out.fill_(9.0)
            graph.replay()
        torch.cuda.synchronize()
        for a, out, graph, kw in sets:
            eager = D.dora_decode_attn_window(*a, torch.empty_like(out), stream=s, **kw)
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), step

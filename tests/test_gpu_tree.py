"""dora_decode_attn_tree through the C ABI against the operator written down in 64 bits."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check, odd_scales, random_trees, tree_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _drafts(B, T, Hkv, G, d, counts, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, T, Hkv * G, d, generator=g).to(torch.bfloat16)
    kd = torch.randn(B, T, Hkv, d, generator=g).to(torch.bfloat16)
    vd = torch.randn(B, T, Hkv, d, generator=g).to(torch.bfloat16)
    for b, n in enumerate(counts):  # what belongs to no node may be anything
        for x in (q, kd, vd):
            x[b, n:] = float("nan")
    return q, kd, vd


def _run(c, q, kd, vd, mask, counts, out, **kw):
    D, dev = lib(), c.gpu()
    got = out.cuda()
    D.dora_decode_attn_tree(q.cuda(), kd.cuda(), vd.cuda(), torch.from_numpy(mask.view(np.int64)).cuda(),
                            dev["k"], dev["v"], dev["bt"], dev["lens"], None, got,
                            node_counts=None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda(),
                            **dev["kw"], **kw)
    torch.cuda.synchronize()
    return got


def _case(lens, counts, T, Hkv, G, d, P, dt, seed, masks=None, stride=None, **kw):
    print(f"[case] tree lens={list(lens)[:6]}.. T={T} Hkv={Hkv} G={G} d={d} P={P} dt={dt} {kw}", flush=True)
    c = Cache(lens, Hkv, d, P, dt, seed=seed, stride=stride)
    rng = np.random.default_rng(seed)
    ns = [T] * len(lens) if counts is None else counts
    mask = random_trees(rng, ns, T) if masks is None else masks
    q, kd, vd = _drafts(len(lens), T, Hkv, G, d, ns, seed + 5)
    out = torch.full((len(lens), T, Hkv * G, d), 7.0, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, ns, out, kw.get("sm_scale", 0.0))
    got = _run(c, q, kd, vd, mask, counts, out, **kw)
    check(got, want, spread, "tree")
    for b, n in enumerate(ns):
        assert torch.all(got[b, n:] == 7.0), "rows of nodes that are not there"
    return got


SHORT = [0, 1, 15, 16, 17, 31, 32, 33, 100, 250]
MIXED = [700, 0, 1, 33, 129, 512, 513, 1300, 64]


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (5, 7), (8, 8), (24, 4), (64, 2)])
def test_short_rows(dt, P, d, T, G):
    """Tables short enough for a workgroup per (sequence, KV head); one to four column tiles."""
    counts = [T, 1, T // 2, T, 0, T, max(1, T - 1), T, 1, T]
    _case(SHORT, counts, T, 2, G, d, P, dt, seed=T * 100 + P + dt)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(2, 3), (9, 6), (33, 3)])
def test_cut_rows(dt, P, d, T, G):
    """Longer tables: ranges that cut segments anywhere, joined again."""
    counts = [T, T, 1, 0, T, max(1, T // 3), T, T, T]
    _case(MIXED, counts, T, 2, G, d, P, dt, seed=T * 10 + P + dt)


@pytest.mark.parametrize("waves", [1, 4, 12, 28, 400])
def test_any_number_of_workgroups_gives_the_same(waves):
    """One range over everything (a page window is refilled: 20,000 tokens), and many."""
    for dt, P in ((0, 16), (1, 32)):
        _case([20000, 3, 500, 0, 40], [6, 6, 2, 6, 6], 6, 1, 4, 64, P, dt, seed=9, num_waves=waves)


@pytest.mark.parametrize("dt", [0, 1])
def test_column_blocks(dt):
    """64 nodes of 16 heads: 1,024 columns in blocks, ragged counts that leave blocks out."""
    _case([90, 700, 17], [64, 20, 3], 64, 1, 16, 64, 16, dt, seed=3)


def test_no_counts_and_a_scale():
    _case([40, 600], None, 7, 2, 4, 128, 16, 0, seed=11, sm_scale=0.25)


def test_masks_that_leave_rows_empty():
    """No bit at all: zeros without a cache, the cache alone with one; bits of one other node
    only; every bit; nodes past 31."""
    T = 40
    masks = np.zeros((4, T), np.uint64)
    masks[1] = np.uint64(2 ** 64 - 1)
    masks[2] = np.uint64(1) << np.uint64(39)
    masks[3, ::2] = np.uint64(1)
    got = _case([0, 0, 5, 0], [T, T, T, T], T, 1, 2, 64, 16, 0, seed=12, masks=masks)
    assert torch.all(got[0] == 0) and torch.all(got[3, 1::2] == 0)
    _case([0, 700, 5, 0], [T, T, T, T], T, 1, 2, 64, 32, 1, seed=13, masks=masks, stride=60)


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(4, 4), (12, 4), (16, 8)])
def test_odd_scales(d, P, T, G):
    c = Cache([300, 100, 90, 211, 64, 50, 33], 2, d, P, 1, seed=d + P)
    odd_scales(c)
    ns = [T, T, 1, T - 1, T, 2, T]
    mask = random_trees(np.random.default_rng(T), ns, T)
    q, kd, vd = _drafts(7, T, 2, G, d, ns, T)
    out = torch.full((7, T, 2 * G, d), 7.0, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, ns, out)
    check(_run(c, q, kd, vd, mask, ns, out), want, spread, "tree", roundings=2)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_of_any_magnitude(dt, P, d):
    """Elements of 2^-14 to 4 of their row's scale, rows of zeros, of subnormals, of one large element,
    and with an infinity or a NaN, which make the row NaN.  Scores: what the fp8 products leave of a
    query is 2^-21 of its largest element (8), so 8 * 2^-21 * sum |k| (128 of 0.8) is below 2^-11, with
    the softmax scale and log2(e) below 2^-13."""
    T, G, lens = 16, 8, [2500, 3000, 100, 0]
    c = Cache(lens, 1, d, P, dt, seed=d + P)
    q, kd, vd = _drafts(4, T, 1, G, d, [T] * 4, 7)
    g = torch.Generator().manual_seed(9)
    q = (q.float() * 2.0 ** torch.randint(-14, 2, q.shape, generator=g)).clamp(-8, 8)
    q[0, 1], q[0, 2] = 0.0, q[0, 2] * 2.0 ** -132
    q[0, 3] *= 2.0 ** -9
    q[0, 3, :, 5] = 8.0
    q[1, 4, 3, 7], q[1, 5, 0, d - 1], q[2, 6, 1, 0] = float("inf"), -float("inf"), float("nan")
    q = q.to(torch.bfloat16)
    mask = random_trees(np.random.default_rng(3), [T] * 4, T)
    out = torch.zeros(4, T, G, d, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, [T] * 4, out)
    check(_run(c, q, kd, vd, mask, None, out), want, spread, "tree")


def test_infinite_scores():
    """Keys of -inf: no weight; of all visible tokens: NaN, as the definition gives."""
    for lens in ([40, 600], [40, 30]):
        c = Cache(lens, 1, 64, 16, 0, seed=14)
        q, kd, vd = _drafts(2, 3, 1, 2, 64, [3, 3], 15)
        q[:, :, :, 0] = q[:, :, :, 0].abs() + 0.5
        c.k[c.bt[0, 0], :, 0, 3, 0] = -float("inf")
        c.k[c.bt[1, 1], :, 0, :, 0] = -float("inf")
        kd[0, :, :, 0] = -float("inf")
        for j in range(3):
            c.k[c.bt[0, j], :, 0, :, 0] = -float("inf")
        mask = np.full((2, 3), 7, np.uint64)
        out = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
        want, spread = tree_reference(c, q, kd, vd, mask, [3, 3], out)
        assert np.isnan(want[0]).all() and np.isfinite(want[1]).all()
        check(_run(c, q, kd, vd, mask, [3, 3], out), want, spread)


def test_many_sequences_take_several_launches():
    """More sequences than a launch takes (2,048), with and without cuts."""
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 30, 2100)
    lens[2060] = 900
    counts = [int(x) for x in rng.integers(0, 3, 2100)]
    for stride in (57, 60):
        _case(lens, counts, 2, 1, 1, 64, 16, 0, seed=16, stride=stride)


def test_far_pages():
    """Page offsets past 32 bits: the sequence's pages are the last of a pool of 9 GB."""
    D = lib()
    Hkv, d, P, n = 8, 128, 32, 70000
    c = Cache([130, 700], Hkv, d, P, 0, seed=17)
    far = n - c.num_pages
    k = torch.empty((n,) + c.k.shape[1:], dtype=torch.bfloat16, device="cuda")
    v = torch.empty((n,) + c.v.shape[1:], dtype=torch.bfloat16, device="cuda")
    k[far:], v[far:] = c.k.cuda(), c.v.cuda()
    q, kd, vd = _drafts(2, 3, Hkv, 2, d, [3, 3], 18)
    mask = np.full((2, 3), 7, np.uint64)
    out = torch.zeros(2, 3, 16, d, dtype=torch.bfloat16)
    want, spread = tree_reference(c, q, kd, vd, mask, [3, 3], out)
    got = out.cuda()
    D.dora_decode_attn_tree(q.cuda(), kd.cuda(), vd.cuda(), torch.from_numpy(mask.view(np.int64)).cuda(), k, v,
                            torch.from_numpy(c.bt + far).cuda(), torch.from_numpy(c.lens).cuda(), None, got,
                            num_kv_heads=Hkv, page_size=P)
    check(got, want, spread)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("T,G", [(2, 8), (5, 8), (9, 8)])
def test_rows_past_the_ids_held_at_a_time(dt, T, G):
    """Around 512 pages of 16 tokens, whose ids a workgroup holds at once, and twice that, whole rows
    in one range and cut."""
    lens = [8191, 8192, 8193, 8224, 16400]
    _case(lens, None, T, 1, G, 64, 16, dt, seed=T + dt, num_waves=4)
    _case(lens, None, T, 1, G, 64, 16, dt, seed=T + dt)


def test_workspaces_of_different_sizes_in_turn():
    """Batches whose calls need less, more and less again than the workspace that is kept."""
    D = lib()
    runs = []
    for n, (lens, T) in enumerate([([4000, 20], 4), ([3000, 2500, 4100], 40), ([2100], 9)]):
        c = Cache(lens, 2, 64, 16, 0, seed=41 + n)
        dev = c.gpu()
        q, kd, vd = (x.cuda() for x in _drafts(len(lens), T, 2, 4, 64, [T] * len(lens), 43 + n))
        mask = torch.from_numpy(random_trees(np.random.default_rng(n), [T] * len(lens), T).view(np.int64)).cuda()
        a = (q, kd, vd, mask, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
        desc = D.make_decode_desc(num_seqs=len(lens), num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16,
                                  block_table_stride=dev["bt"].shape[1], num_pages=c.num_pages)
        ws = torch.empty(D.dora_decode_tree_workspace_bytes(desc, T), dtype=torch.uint8, device="cuda")
        want = D.dora_decode_attn_tree(*a, torch.empty_like(q), workspace=ws, **dev["kw"])
        runs.append((a, dev, want))
    for n in (0, 1, 2, 1, 0):
        a, dev, want = runs[n]
        got = D.dora_decode_attn_tree(*a, torch.empty_like(want), **dev["kw"])
        assert torch.equal(got.view(torch.int16), want.view(torch.int16)), n


def test_one_node_without_drafts_of_others_equals_the_decode():
    """A tree of one node over a cache, against the plain decode with that token appended."""
    D = lib()
    lens = np.array([5, 100, 640, 31], np.int32)
    c = Cache(lens, 2, 128, 16, 0, seed=19, extra_tokens=1)
    q, kd, vd = _drafts(4, 1, 2, 4, 128, [1] * 4, 20)
    got = _run(c, q, kd, vd, np.ones((4, 1), np.uint64), None, torch.zeros(4, 1, 8, 128, dtype=torch.bfloat16))
    dev = c.gpu()
    after = dev["lens"] + 1
    D.dora_kv_append(kd[:, 0].contiguous().cuda(), vd[:, 0].contiguous().cuda(), dev["bt"], after, dev["k"], dev["v"],
                     num_kv_heads=2, page_size=16)
    one = torch.empty(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    D.dora_decode_attn(q[:, 0].contiguous().cuda(), dev["k"], dev["v"], dev["bt"], after, None, one,
                       num_kv_heads=2, page_size=16)
    # both round their weights and results to bf16
    assert (got[:, 0].float() - one.float()).abs().max() <= 4 * 2.0 ** -8 * 4


def test_validate_reports_bad_tables():
    D = lib()
    c = Cache([40, 600], 1, 64, 16, 0, seed=21)
    q, kd, vd = _drafts(2, 2, 1, 1, 64, [2, 2], 22)
    mask = np.full((2, 2), 3, np.uint64)
    out = torch.full((2, 2, 1, 64), 3.0, dtype=torch.bfloat16)
    c.bt[1, 5] = c.num_pages
    with pytest.raises(D.DoraError) as e:
        _run(c, q, kd, vd, mask, None, out, flags=D.DORA_FLAG_VALIDATE)
    assert e.value.status == D.DORA_ERR_DEVICE_CHECK


def test_repeated_calls_streams_and_workspaces():
    """Bitwise the same again, on another stream, and with a workspace of the caller's."""
    D = lib()
    c = Cache([3000, 20, 900], 2, 128, 16, 0, seed=23)
    dev = c.gpu()
    q, kd, vd = (x.cuda() for x in _drafts(3, 5, 2, 7, 128, [5] * 3, 24))
    mask = torch.from_numpy(random_trees(np.random.default_rng(1), [5] * 3, 5).view(np.int64)).cuda()
    a = (q, kd, vd, mask, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
    first = D.dora_decode_attn_tree(*a, torch.empty_like(q), **dev["kw"]).clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [torch.empty_like(q) for _ in range(4)]
    for o in outs[:2]:
        D.dora_decode_attn_tree(*a, o, **dev["kw"])
        D.dora_decode_attn_tree(*a, outs[2], stream=s, **dev["kw"])
    desc = D.make_decode_desc(num_seqs=3, num_q_heads=14, num_kv_heads=2, head_dim=128, page_size=16,
                              block_table_stride=dev["bt"].shape[1], num_pages=c.num_pages)
    need = D.dora_decode_tree_workspace_bytes(desc, 5)
    ws = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    D.dora_decode_attn_tree(*a, outs[3], workspace=ws[:need], **dev["kw"])
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.view(torch.int16), first.view(torch.int16))
    assert torch.all(ws[need:] == 0xAB)
    with pytest.raises(D.DoraError) as e:
        D.dora_decode_attn_tree(*a, outs[3], workspace=ws[:need - 256], **dev["kw"])
    assert e.value.status == D.DORA_ERR_WORKSPACE_TOO_SMALL


def test_two_threads_on_one_stream():
    """Calls of two launches each, from two threads on the same stream at once: each thread has a
    workspace of its own."""
    import threading
    D = lib()
    sets = []
    for n in range(2):
        c = Cache([3000 + 700 * n, 2100], 2, 64, 16, 0, seed=31 + n)
        dev = c.gpu()
        q, kd, vd = (x.cuda() for x in _drafts(2, 5, 2, 4, 64, [5] * 2, 33 + n))
        mask = torch.from_numpy(random_trees(np.random.default_rng(n), [5] * 2, 5).view(np.int64)).cuda()
        a = (q, kd, vd, mask, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
        want = D.dora_decode_attn_tree(*a, torch.empty_like(q), **dev["kw"])
        sets.append((a, dev, want, [torch.empty_like(q) for _ in range(40)]))
    torch.cuda.synchronize()
    errors = []

    def work(a, dev, outs):
        try:
            for o in outs:
                D.dora_decode_attn_tree(*a, o, **dev["kw"])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(a, dev, outs)) for a, dev, _, outs in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for _, _, want, outs in sets:
        for o in outs:
            assert torch.equal(o.view(torch.int16), want.view(torch.int16))


def test_graph_replays():
    """Captured with the library's workspace, two graphs of different sizes, replayed in turn
    with new inputs between."""
    D = lib()
    sets = []
    for n, (lens, T) in enumerate([([3000, 20, 900], 5), ([70, 1200], 9)]):
        c = Cache(lens, 2, 64, 16, 0, seed=25 + n)
        dev = c.gpu()
        q, kd, vd = (x.cuda() for x in _drafts(len(lens), T, 2, 4, 64, [T] * len(lens), 27 + n))
        mask = torch.from_numpy(random_trees(np.random.default_rng(n), [T] * len(lens), T).view(np.int64)).cuda()
        out = torch.empty_like(q)
        a = (q, kd, vd, mask, dev["k"], dev["v"], dev["bt"], dev["lens"], None)
        D.dora_decode_attn_tree(*a, out, **dev["kw"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.dora_decode_attn_tree(*a, out, **dev["kw"])
        sets.append((a, out, graph, dev))
    for step in range(4):
        for a, out, graph, dev in sets:
            a[0].copy_(torch.randn_like(a[0].float()).to(torch.bfloat16))
            out.fill_(9.0)
            graph.replay()
        torch.cuda.synchronize()
        for a, out, graph, dev in sets:
            eager = D.dora_decode_attn_tree(*a, torch.empty_like(out), **dev["kw"])
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), step

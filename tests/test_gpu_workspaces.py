"""Workspaces that the binding makes where the caller gives none: no larger than the call uses, and a captured graph's its
own."""
import pytest
import torch

import workloads as wl
from cache_util import Cache
from fp4_util import FP4, Cache4
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _recorded(monkeypatch, D, name, at):
    """The arguments `at` of the library's function in each call from here on."""
    seen, call = [], getattr(D.library(), name)

    def record(*args):
        seen.append(tuple(args[i] for i in at))
        return call(*args)

    monkeypatch.setattr(D.library(), name, record)
    return seen


def test_a_choice_with_scores_keeps_no_second_buffer(monkeypatch):
    """Scores that the caller takes need no room in the workspace; lists are equal with them and without."""
    D, B, Hkv, d, P, width, budget = lib(), 20, 4, 64, 16, 3000, 9
    g = torch.Generator().manual_seed(1)
    pages = 5000
    bounds = torch.randint(0, 100, (pages, D.dora_page_bounds_bytes(Hkv, d)), generator=g, dtype=torch.uint8).cuda()
    bt = torch.randint(0, pages, (B, width), generator=g, dtype=torch.int32).cuda()
    lens = torch.randint(0, width * P + 1, (B,), generator=g, dtype=torch.int32).cuda()
    q = torch.randn(B, Hkv * 2, d, generator=g).to(torch.bfloat16).cuda()
    scores = torch.zeros(B, Hkv, width, device="cuda")
    picked = [[torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")]
              for _ in range(3)]
    stream = torch.cuda.Stream()  # one that no call has a workspace for yet
    torch.cuda.synchronize()
    seen = _recorded(monkeypatch, D, "dora_page_select", (-2,))
    for out, sc in zip(picked, (scores, None, scores)):
        D.dora_page_select(q, bounds, bt, lens, *out, num_kv_heads=Hkv, page_size=P, scores=sc, stream=stream)
    torch.cuda.synchronize()
    assert seen[0] == (256,)
    desc = D.make_decode_desc(num_seqs=B, num_q_heads=Hkv * 2, num_kv_heads=Hkv, head_dim=d, page_size=P, block_table_stride=width, num_pages=pages)
    full = D.dora_page_select_workspace_bytes(desc)
    assert full == 256 + B * Hkv * width * 4 and seen[-1] == (full,)  # (one that is there and large enough serves)
    for out in picked[1:]:
        assert torch.equal(out[0], picked[0][0]) and torch.equal(out[1], picked[0][1])
    # a captured call's is new each time
    seen.clear()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.dora_page_select(q, bounds, bt, lens, *picked[2], num_kv_heads=Hkv, page_size=P, scores=scores)
    assert seen == [(256,)]
    for _ in range(3):
        picked[2][0].fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(picked[2][0], picked[0][0])


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("dt", [0, 1, FP4])
def test_two_graphs_of_one_stream_have_a_workspace_each(dt, grouped, monkeypatch):
    """Two decodes captured on the same stream, replayed at once on two others beside an eager one: each equals its own
    eager run."""
    if dt == FP4 and grouped:
        return  # refused
    D = lib()
    name = "dora_decode_attn_grouped" if grouped else "dora_decode_attn"
    seen = _recorded(monkeypatch, D, name, (-3,))
    capture = torch.cuda.Stream()
    runs = []
    for i in range(2):
        if grouped:
            M = 4
            w = wl.Workload("g", 2 * M, 8, 2, 128, 16, dt, 8192, "lognormal", 3000, 0.5, 1, 6000)
            b, _ = wl.make_grpo_batch(w, group_size=M, prompt_range=(300, 900), device="cuda", seed_index=i)
            out = torch.zeros_like(b.q)
            b.block_table = torch.nn.functional.pad(b.block_table, (0, 600 - b.block_table.shape[1])).contiguous()  # workspaces of one size

            def step(b=b, out=out, **kw):
                D.dora_decode_attn_grouped(b.q, b.k_pages, b.v_pages, b.block_table, b.seq_lens, None, out, group_size=4, num_kv_heads=2,
                                           page_size=16, kv_dtype=dt, k_scales=b.k_scales, v_scales=b.v_scales, **kw)
        else:
            c = (Cache4 if dt == FP4 else lambda *a, **k: Cache(*a, dt, **k))([9000, 300, 5000], 2, 64, 16, seed=i)
            dev = c.gpu()
            q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda()
            out = torch.zeros_like(q)

            def step(dev=dev, q=q, out=out, **kw):
                D.dora_decode_attn(q, dev["k"], dev["v"], dev["bt"], dev["lens"], None, out, **dev["kw"], **kw)

        step()
        torch.cuda.synchronize()
        eager = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=capture):
            step()
        runs.append((graph, torch.cuda.Stream(), step, out, eager))
    seen.append(None)
    for _, _, step, out, eager in runs:  # and the stream's eager calls have another
        out.zero_()
        torch.cuda.synchronize()
        step(stream=capture)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    first, second = seen[1], seen[3]
    assert first != second and not {first, second} & set(seen[seen.index(None) + 1:])
    for _ in range(5):
        for _, _, _, out, _ in runs:
            out.zero_()
        torch.cuda.synchronize()
        for graph, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, eager) for *_, out, eager in runs)
        float(torch.randn(1000, device="cuda").sum())

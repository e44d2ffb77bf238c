"""Workspaces that the binding makes where the caller gives none: no larger than the call uses, and a captured graph's its
own."""
import pytest
import torch

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

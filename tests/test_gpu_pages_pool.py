"""Bounds of a pool's pages through forks and compactions: what the caller copies and what it takes again."""
import numpy as np
import pytest
import torch

import workloads as wl
from cache_util import Cache, check
from fp4_util import FP4, Cache4, tile_bytes
from gpu_util import lib
from test_gpu_pages import TYPES, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("P,d", [(16, 64), (32, 128)])
def test_bounds_follow_forks_and_compactions(dt, P, d):
    """Prompts are forked, whole and from the middle of a page, responses appended, some freed, the pool compacted.  Shared
    pages keep their bounds, a fork's own page takes them again, moved pages' records are copied: after each the bounds
    equal those taken from nothing, and chosen pages are attended as the definition says."""
    D, Hkv, G, pages, budget = lib(), 2, 3, 160, 5
    g = torch.Generator().manual_seed(P + dt)
    pool = D.Pool(pages, P, 2, seed=3)
    X = wl.chunk_elems(dt) if dt != FP4 else 0
    shapes = ((pages, Hkv, tile_bytes(d, P)),) * 2 if dt == FP4 else ((pages, Hkv, d // X, P, X), (pages, Hkv, d, P))
    k, v = (torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") if dt == 0 else
            torch.full(s, 0x7F if dt == 1 else 0xFF, dtype=torch.uint8, device="cuda") for s in shapes)
    ks, vs = (torch.full((pages,), float("nan"), device="cuda") if dt == 1 else None for _ in range(2))
    kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=dt)
    scales = dict(k_scales=ks, v_scales=vs)
    record = D.dora_page_bounds_bytes(Hkv, d)
    bounds = torch.full((pages, record), 0x55, dtype=torch.uint8, device="cuda")
    used = Hkv * (2 * d + 4)
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731

    def take(ids, counts, into):
        table, lens, vers = pool.block_table(ids)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        D.dora_kv_page_bounds(k, gpu(table), gpu(lens), into, num_tokens=int(max(counts)), head_dim=d, counts=gpu(np.asarray(counts, np.int32)),
                              k_scales=ks, version_ids=gpu(vers), page_owner=gpu(pool.page_owner()), flags=D.DORA_FLAG_VALIDATE,
                              dev_status=status, **kw)
        assert int(status.item()) == 0

    def append(ids, counts):
        n = int(max(counts))
        new = [torch.randn(len(ids), n, Hkv, d, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
        table, lens, _ = pool.block_table(ids)
        D.dora_kv_append_path(*new, gpu(table), gpu(lens), k, v, counts=gpu(np.asarray(counts, np.int32)), **kw, **scales)
        take(ids, counts, bounds)

    def grow(ids, counts):
        _, lens, _ = pool.block_table(ids)
        for sid, L, n in zip(ids, lens, counts):
            pool.extend_seq(sid, int(L) + int(n))
        append(ids, counts)

    def move(src, dst):
        D.dora_kv_page_copy(k, v, gpu(src), gpu(dst), head_dim=d, **kw, **scales)

    def agree(ids, what):
        table, lens, _ = pool.block_table(ids)
        again = torch.full_like(bounds, 0xAA)
        take(ids, lens, again)
        for b, L in enumerate(lens):
            at = torch.from_numpy(table[b, :-(-int(L) // P)].astype(np.int64)).cuda()
            assert torch.equal(bounds[at][:, :used], again[at][:, :used]), (what, b)
        c = object.__new__(Cache4 if dt == FP4 else Cache)
        c.bt, c.lens, c.Hkv, c.d, c.P, c.dt = table, lens, Hkv, d, P, dt
        c.k, c.v = k.cpu(), v.cpu()
        c.ks, c.vs = (None if x is None else x.cpu() for x in (ks, vs))
        q = torch.randn(len(ids), Hkv * G, d, generator=g).to(torch.bfloat16)
        lists = torch.full((len(ids), Hkv, budget), -1, dtype=torch.int32, device="cuda")
        counts = torch.zeros(len(ids), Hkv, dtype=torch.int32, device="cuda")
        D.dora_page_select(q.cuda(), bounds, gpu(table), gpu(lens), lists, counts, num_kv_heads=Hkv, page_size=P)
        out = torch.zeros_like(q).cuda()
        D.dora_decode_attn_pages(q.cuda(), lists, counts, k, v, gpu(table), gpu(lens), None, out, **kw, **scales)
        check(out, *_reference(c, q, lists.cpu().numpy(), counts.cpu().numpy()), what)

    prompts = [pool.add_seq(1, 5 * P + 3), pool.add_seq(1, 9 * P), pool.add_seq(1, 12 * P + P - 1)]
    append(prompts, [5 * P + 3, 9 * P, 12 * P + P - 1])
    agree(prompts, "prompts")
    ids, tails = [], []
    for p in prompts:
        for n in (None, 2 * P + 5, 3 * P, 4 * P + 1):  # whole, and from the middle or the end of a page
            sid, src, dst = pool.fork_seq(p, n)
            if len(src):
                move(src, dst)
            ids.append(sid)
            _, L, _ = pool.block_table([sid])
            tails.append(int(L[0]) % P)  # tokens in a page of the fork's own: those of its source may be more
    take(ids, tails, bounds)
    agree(ids + prompts, "forks")
    for sid in prompts:
        pool.free_seq(sid)
    grow(ids, np.arange(len(ids)) * 3 + 1)
    agree(ids, "responses")
    for sid in ids[1::3]:
        pool.free_seq(sid)
    ids = [s for i, s in enumerate(ids) if i % 3 != 1]
    src, dst = pool.compact()
    assert len(src) > 0
    move(src, dst)
    bounds[torch.from_numpy(np.asarray(dst, np.int64)).cuda()] = bounds[torch.from_numpy(np.asarray(src, np.int64)).cuda()]
    agree(ids, "compacted")
    grow(ids, [2] * len(ids))
    agree(ids, "a step behind it")

"""dora_kv_page_copy through the C ABI, and the pool's forks, releases and compaction with
the attention that reads what they leave."""
import numpy as np
import pytest
import torch

import workloads as wl
from cache_util import Cache, check, random_trees, tree_reference, window_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu


def _bytes(t):
    return t.contiguous().view(torch.uint8) if t.dtype != torch.uint8 else t


def _pool(n, Hkv, d, P, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = wl.chunk_elems(dt)
    out = []
    for s in ((n, Hkv, d // X, P, X), (n, Hkv, d, P)):
        t = torch.randint(0, 256, s[:-1] + (s[-1] * (2 if dt == 0 else 1),), generator=g, device="cuda", dtype=torch.uint8)
        out.append(t.view(torch.bfloat16) if dt == 0 else t)
    return out


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("Hkv,d,P", [(1, 64, 16), (4, 128, 16), (8, 128, 32), (3, 64, 32), (5, 16, 8)])
def test_copies(dt, Hkv, d, P):
    """Bit for bit: pages copied once, to many places and onto themselves; others untouched;
    pairs with an id outside the pool skipped and reported."""
    D = lib()
    print(f"[case] page copy dt={dt} Hkv={Hkv} d={d} P={P}", flush=True)
    n = 60
    k, v = _pool(n, Hkv, d, P, dt, seed=Hkv + d)
    ks, vs = (torch.rand(n, device="cuda") for _ in range(2))
    rng = np.random.default_rng(dt)
    perm = rng.permutation(n)
    src = np.concatenate([perm[:10], np.repeat(perm[10], 7), perm[58:59]]).astype(np.int32)
    dst = np.concatenate([perm[20:37], perm[58:59]]).astype(np.int32)
    want = [x.clone() for x in (k, v, ks, vs)]
    for x in want:
        x[torch.from_numpy(dst.astype(np.int64)).cuda()] = x[torch.from_numpy(src.astype(np.int64)).cuda()]
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    kw = dict(num_kv_heads=Hkv, page_size=P, head_dim=d, kv_dtype=dt, k_scales=ks if dt else None, v_scales=vs if dt else None,
              dev_status=status)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    D.dora_kv_page_copy(k, v, i32(src), i32(dst), **kw)
    assert int(status.item()) == 0
    for got, x in zip((k, v) + ((ks, vs) if dt else ()), want):
        assert torch.equal(_bytes(got), _bytes(x))
    D.dora_kv_page_copy(k, v, i32([n, -1, 0, 1]), i32([40, 41, n, -5]), **kw)
    assert int(status.item()) == D.DORA_ERR_DEVICE_CHECK
    D.dora_kv_page_copy(k, v, i32([]), i32([]), **kw)
    assert int(status.item()) == 0
    for got, x in zip((k, v), want):
        assert torch.equal(_bytes(got), _bytes(x))


def test_many_and_far_pages():
    """More pages than a grid layer holds, and offsets past 32 bits."""
    D = lib()
    n = 70000
    k, v = _pool(n, 1, 64, 16, 1, seed=1)
    scales = torch.rand(n, device="cuda")
    at = torch.randperm(n, device="cuda").to(torch.int32)
    src, dst = at[:n // 2].contiguous(), at[n // 2:].contiguous()
    want = k.clone(), v.clone()
    for x in want:
        x[dst.long()] = x[src.long()]
    D.dora_kv_page_copy(k, v, src, dst, num_kv_heads=1, page_size=16, head_dim=64, kv_dtype=1, k_scales=scales, v_scales=scales.clone())
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    big = torch.zeros((n, 8, 16, 32, 8), dtype=torch.bfloat16, device="cuda")  # 4.6 GB
    vals = torch.zeros((n, 8, 128, 32), dtype=torch.bfloat16, device="cuda")
    big[3], vals[3] = 1.5, 2.5
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    D.dora_kv_page_copy(big, vals, i32([3, n - 1]), i32([n - 2, 5]), num_kv_heads=8, page_size=32, head_dim=128)
    assert torch.all(big[n - 2] == 1.5) and torch.all(vals[n - 2] == 2.5) and torch.all(big[n - 3] == 0)


@pytest.mark.parametrize("dt", [0, 1])
def test_fork_draft_accept_release_compact(dt):
    """The calls as a rollout makes them: prompts are written, forked for their responses,
    verified drafts are accepted, windows release their pages, the pool is compacted; after
    each the attention over what is there agrees with the definition in 64 bits."""
    D = lib()
    Hkv, G, d, P, T = 2, 4, 64, 16, 6
    rng = np.random.default_rng(5)
    g = torch.Generator().manual_seed(5 + dt)
    pool = D.Pool(200, P, 2, seed=7)
    X = wl.chunk_elems(dt)
    shapes = ((200, Hkv, d // X, P, X), (200, Hkv, d, P))
    if dt == 0:
        k, v = (torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") for s in shapes)
        ks = vs = None
    else:
        k, v = (torch.full(s, 0x7F, dtype=torch.uint8, device="cuda") for s in shapes)
        ks, vs = (torch.full((200,), float("nan"), device="cuda") for _ in range(2))
    kw = dict(num_kv_heads=Hkv, page_size=P, kv_dtype=dt, k_scales=ks, v_scales=vs)
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731

    def append(ids, x, y, counts, path=None):
        table, lens, _ = pool.block_table(ids)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        D.dora_kv_append_path(x, y, gpu(table), gpu(lens), k, v, counts=gpu(np.asarray(counts, np.int32)),
                              path=None if path is None else gpu(np.asarray(path, np.int32)), dev_status=status, **kw)
        assert int(status.item()) == 0

    def copy(src, dst):
        D.dora_kv_page_copy(k, v, gpu(src), gpu(dst), head_dim=d, **kw)

    def view(ids):
        """What is in the pool now, as the 64-bit reference reads it."""
        c = object.__new__(Cache)
        c.bt, c.lens, _ = pool.block_table(ids)
        c.Hkv, c.d, c.P, c.dt = Hkv, d, P, dt
        c.k, c.v = k.cpu(), v.cpu()
        c.ks, c.vs = (None if x is None else x.cpu() for x in (ks, vs))
        return c

    rand = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
    # two prompts, written in one call
    prompts = [pool.add_seq(1, 50), pool.add_seq(1, 200)]
    append(prompts, rand(2, 200, Hkv, d).cuda(), rand(2, 200, Hkv, d).cuda(), [50, 200])
    # three responses each; a fork from the middle of a prompt too
    ids, moves = [], []
    for p in prompts:
        for n in (None, None, 33):
            sid, src, dst = pool.fork_seq(p, n)
            ids.append(sid)
            moves.append((src, dst))
    copy(np.concatenate([m[0] for m in moves]), np.concatenate([m[1] for m in moves]))
    used, _ = pool.stats(1)
    assert used == 4 + 13 + 6  # the prompts' pages, and a last page for each fork
    for sid in prompts:
        pool.free_seq(sid)
    for step in range(4):
        table, lens, vers = pool.block_table(ids)
        B = len(ids)
        counts = rng.integers(1, T + 1, B).astype(np.int32)
        mask = random_trees(rng, counts, T)
        q, kd, vd = rand(B, T, Hkv * G, d), rand(B, T, Hkv, d), rand(B, T, Hkv, d)
        out = torch.zeros_like(q)
        c = view(ids)
        want, spread = tree_reference(c, q, kd, vd, mask, counts, out)
        owner = gpu(pool.page_owner())
        got = D.dora_decode_attn_tree(q.cuda(), kd.cuda(), vd.cuda(), gpu(mask.view(np.int64)), k, v, gpu(table), gpu(lens),
                                      gpu(vers), out.cuda(), node_counts=gpu(counts), page_owner=owner,
                                      flags=D.DORA_FLAG_VALIDATE, **kw)
        check(got, want, spread, f"step {step}")
        # accept the path from a root to the last node
        paths, taken = np.zeros((B, T), np.int32), np.zeros(B, np.int32)
        for b in range(B):
            nodes = [j for j in range(int(counts[b])) if (int(mask[b, counts[b] - 1]) >> j) & 1]
            paths[b, :len(nodes)], taken[b] = nodes, len(nodes)
        for b, sid in enumerate(ids):
            pool.extend_seq(sid, int(lens[b]) + int(taken[b]))
        append(ids, kd.cuda(), vd.cuda(), taken, paths)
    window, sinks = 40, 3
    released = sum(pool.release_window(sid, window, sinks) for sid in ids)
    assert released > 0
    for _ in range(2):
        table, lens, vers = pool.block_table(ids)
        q = rand(len(ids), Hkv * G, d)
        want, spread = window_reference(view(ids), q, window, sinks)
        got = D.dora_decode_attn_window(q.cuda(), k, v, gpu(table), gpu(lens), gpu(vers), torch.empty_like(q).cuda(),
                                        window=window, sinks=sinks, page_owner=gpu(pool.page_owner()),
                                        flags=D.DORA_FLAG_VALIDATE, **kw)
        check(got, want, spread, "window")
        src, dst = pool.compact()
        copy(src, dst)
        used, _ = pool.stats()
        assert np.all(pool.page_owner()[:used] >= 0) and np.all(pool.page_owner()[used:] < 0)

"""CPU checks of the entry points around the cache (tree and window attention, path append,
page copies): refusals before any launch, workspace sizes; the pool's forks, releases and
compaction against a plain model."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def d():
    from paper_2604_26256_amd import build as B
    if not os.path.exists(B.LIB):
        B.build()
    from paper_2604_26256_amd import dora
    return dora


def _desc(d, **kw):
    base = dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, block_table_stride=64,
                num_pages=1024)
    base.update(kw)
    return d.make_decode_desc(**base)


BAD = [("null", None, 1), ("heads", dict(num_q_heads=9), 1), ("negative", dict(num_seqs=-1), 1), ("d", dict(head_dim=96), 2),
       ("page", dict(page_size=8), 2), ("group", dict(num_q_heads=34), 2), ("dtype", dict(kv_dtype=2), 2),
       ("scale", dict(sm_scale=float("nan")), 1), ("flags", dict(flags=2), 1)]
PTR = 1 << 20  # an aligned address that is never read: every call here ends before a launch


def _tree(d, desc, nodes=4, q=PTR, kd=PTR, vd=PTR, mask=PTR, counts=None, k=PTR, v=PTR, bt=PTR, lens=PTR, vers=None, out=PTR, ws=PTR,
          size=0):
    return d.library().dora_decode_attn_tree(None if desc is None else ctypes.byref(desc), nodes, q, kd, vd, mask, counts, k, v, bt, lens,
                                             vers, out, ws, size, None)


def _window(d, desc, window=10, sinks=2, q=PTR, k=PTR, v=PTR, bt=PTR, lens=PTR, vers=None, out=PTR, ws=PTR, size=0):
    return d.library().dora_decode_attn_window(None if desc is None else ctypes.byref(desc), window, sinks, q, k, v, bt, lens, vers, out, ws,
                                               size, None)


def _path(d, desc, T=4, k_new=PTR, v_new=PTR, path=None, counts=None, bt=PTR, lens=PTR, vers=None, k=PTR, v=PTR, ks=None, vs=None):
    return d.library().dora_kv_append_path(None if desc is None else ctypes.byref(desc), T, k_new, v_new, path, counts, bt, lens, vers, k, v,
                                           ks, vs, None, None)


@pytest.mark.parametrize("call", [_tree, _window, _path])
def test_bad_descriptors(d, call):
    for name, kw, status in BAD:
        assert call(d, None if kw is None else _desc(d, **kw)) == status, name
    assert call(d, _desc(d, num_seqs=0)) == d.DORA_OK


def test_tree_refusals(d):
    big = 1 << 40
    for nodes in (0, -1, 65):
        assert _tree(d, _desc(d), nodes, size=big) == d.DORA_ERR_INVALID_ARG
        assert d.dora_decode_tree_workspace_bytes(_desc(d), nodes) == 0
    for name in ("q", "kd", "vd", "mask", "k", "v", "bt", "lens", "out", "ws"):
        assert _tree(d, _desc(d), size=big, **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("q", "kd", "vd", "k", "v", "out", "ws"):
        assert _tree(d, _desc(d), size=big, **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG, name
    assert _tree(d, _desc(d, kv_dtype=1), size=big) == d.DORA_ERR_INVALID_ARG  # no scales
    need = d.dora_decode_tree_workspace_bytes(_desc(d), 4)
    assert need > 0 and _tree(d, _desc(d), size=need - 1) == d.DORA_ERR_WORKSPACE_TOO_SMALL
    owned = _desc(d, flags=d.DORA_FLAG_VALIDATE)
    owned.page_owner = PTR
    assert _tree(d, owned, size=big) == d.DORA_ERR_INVALID_ARG  # owners without versions


def test_window_refusals(d):
    big = 1 << 40
    for window, sinks in ((0, 0), (-1, 0), (5, -1)):
        assert _window(d, _desc(d), window, sinks, size=big) == d.DORA_ERR_INVALID_ARG
        assert d.dora_decode_window_workspace_bytes(_desc(d), window, sinks) == 0
    for name in ("q", "k", "v", "bt", "lens", "out", "ws"):
        assert _window(d, _desc(d), size=big, **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("q", "k", "v", "out", "ws"):
        assert _window(d, _desc(d), size=big, **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG, name
    assert _window(d, _desc(d, kv_dtype=1), size=big) == d.DORA_ERR_INVALID_ARG
    need = d.dora_decode_window_workspace_bytes(_desc(d), 10, 2)
    assert need > 0 and _window(d, _desc(d), size=need - 1) == d.DORA_ERR_WORKSPACE_TOO_SMALL
    most = 2 ** 31 - 1  # no overflow at the ends of the range
    assert d.dora_decode_window_workspace_bytes(_desc(d), most, most) > 0
    # what a sequence can show bounds the workspace, not its length
    short, long = (_desc(d, num_seqs=2, block_table_stride=s) for s in (4096, 400000))
    assert d.dora_decode_window_workspace_bytes(short, 4000, 4) == d.dora_decode_window_workspace_bytes(long, 4000, 4)


def test_path_refusals(d):
    for T in (0, -3, (1 << 19) + 1):
        assert _path(d, _desc(d), T) == d.DORA_ERR_INVALID_ARG
    for name in ("k_new", "v_new", "bt", "lens", "k", "v"):
        assert _path(d, _desc(d), **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("k_new", "v_new", "k", "v"):
        assert _path(d, _desc(d), **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG, name
    assert _path(d, _desc(d, kv_dtype=1), ks=PTR) == d.DORA_ERR_INVALID_ARG
    owned = _desc(d, flags=d.DORA_FLAG_VALIDATE)
    owned.page_owner = PTR
    assert _path(d, owned) == d.DORA_ERR_INVALID_ARG


def test_page_copy_refusals(d):
    def call(desc, n=3, k=PTR, v=PTR, ks=None, vs=None, src=PTR, dst=PTR):
        return d.library().dora_kv_page_copy(None if desc is None else ctypes.byref(desc), k, v, ks, vs, src, dst, n, None, None)

    def pack(**kw):
        base = dict(kv_dtype=0, page_size=16, num_kv_heads=2, head_dim=128, num_pages=100, policy_version=0)
        return d.make_pack_desc(**{**base, **kw})

    assert call(None) == d.DORA_ERR_INVALID_ARG
    assert call(pack(num_pages=0)) == d.DORA_ERR_INVALID_ARG
    assert call(pack(kv_dtype=5)) == d.DORA_ERR_UNSUPPORTED
    assert call(pack(num_kv_heads=1, head_dim=3, page_size=1)) == d.DORA_ERR_UNSUPPORTED
    assert call(pack(), n=-1) == d.DORA_ERR_INVALID_ARG
    assert call(pack(), n=1 << 31) == d.DORA_ERR_INVALID_ARG
    for name in ("k", "v", "src", "dst"):
        assert call(pack(), **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("k", "v"):
        assert call(pack(), **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG, name
    assert call(pack(kv_dtype=1), ks=PTR) == d.DORA_ERR_INVALID_ARG
    assert call(pack(), n=0, k=None, v=None, src=None, dst=None) == d.DORA_OK


# ---------------------------------------------------------------------------
# pool
# ---------------------------------------------------------------------------

def test_fork_shares_full_pages_and_copies_the_last(d):
    pool = d.Pool(40, 16, 2, seed=3)
    a = pool.add_seq(1, 50)
    pages = pool.seq_pages(a)
    b, src, dst = pool.fork_seq(a)
    assert pool.seq_info(b) == (50, 1, 4) and src.tolist() == [pages[3]]
    assert pool.seq_pages(b).tolist() == pages[:3].tolist() + dst.tolist() and dst[0] not in pages
    c, src, dst = pool.fork_seq(a, 32)  # whole pages: nothing to copy
    assert len(src) == len(dst) == 0 and pool.seq_pages(c).tolist() == pages[:2].tolist()
    e, src, dst = pool.fork_seq(b, 0)
    assert len(src) == 0 and pool.seq_info(e) == (0, 1, 0)
    assert pool.stats(1) == (5, 35) and pool.stats() == (5, 35)
    pool.extend_seq(c, 33)  # grows into a page of its own
    assert pool.seq_pages(c)[2] not in pages and pool.stats(1)[0] == 6
    pool.free_seq(a)
    assert pool.stats(1)[0] == 5 and pool.page_owner()[pages[3]] == -1 and np.all(pool.page_owner()[pages[:3]] == 1)
    for s in (b, c, e):
        pool.free_seq(s)
    assert pool.stats() == (0, 40) and np.all(pool.page_owner() == -1)


def test_fork_refusals_leave_the_pool_as_it_was(d):
    pool = d.Pool(4, 16, 1)
    a = pool.add_seq(0, 60)
    for args, status in (((a,), d.DORA_ERR_POOL_EXHAUSTED), ((a, 61), d.DORA_ERR_INVALID_ARG), ((a, -1), d.DORA_ERR_INVALID_ARG),
                         ((99, 1), d.DORA_ERR_NOT_FOUND)):
        with pytest.raises(d.DoraError) as e:
            pool.fork_seq(*args)
        assert e.value.status == status
        assert pool.stats() == (4, 0)
    b, _, _ = pool.fork_seq(a, 48)
    pool.free_seq(a)
    assert pool.stats() == (3, 1) and pool.seq_info(b) == (48, 0, 3)
    assert d.library().dora_pool_fork_seq(pool.handle, b, 1, None, None, None, None) == d.DORA_ERR_INVALID_ARG


def test_release_frees_what_no_later_window_reads(d):
    pool = d.Pool(100, 16, 1)
    a = pool.add_seq(0, 1000)
    pages = pool.seq_pages(a).copy()
    assert pool.release_window(a, 5000, 4) == 0
    # the window starts at token 900, in page 56; the sinks fill two pages and a part of the third
    assert pool.release_window(a, 100, 33) == 56 - 3
    left = pool.seq_pages(a)
    assert left[:3].tolist() == pages[:3].tolist() and np.all(left[3:56] == -1) and left[56:].tolist() == pages[56:].tolist()
    assert pool.release_window(a, 100, 33) == 0 and pool.stats()[0] == 63 - 53
    table, lens, _ = pool.block_table([a])
    assert lens[0] == 1000 and np.all(table[0, 3:56] == 0)
    # forks of all its tokens keep the holes, shorter ones are refused
    b, src, dst = pool.fork_seq(a)
    assert np.all(pool.seq_pages(b)[3:56] == -1) and src.tolist() == [pages[62]]
    with pytest.raises(d.DoraError):
        pool.fork_seq(a, 990)
    # migration moves the live pages alone
    other = d.Pool(20, 16, 1)
    m, src, dst = pool.migrate_seq(a, other, 0)
    assert src.tolist() == pages[:3].tolist() + pages[56:].tolist() and other.stats()[0] == 10 == len(dst)
    moved = other.seq_pages(m)
    assert np.all(moved[3:56] == -1) and moved[moved >= 0].tolist() == dst.tolist()
    pool.extend_seq(a, 1017)
    assert pool.seq_info(a)[2] == 64
    pool.free_seq(a)
    pool.free_seq(b)
    assert pool.stats() == (0, 100)
    for window, sinks in ((0, 0), (1, -1)):
        s = pool.add_seq(0, 5)
        with pytest.raises(d.DoraError):
            pool.release_window(s, window, sinks)
    with pytest.raises(d.DoraError) as e:
        pool.release_window(10 ** 6, 1, 0)
    assert e.value.status == d.DORA_ERR_NOT_FOUND


def test_compact_with_too_little_room_changes_nothing(d):
    pool = d.Pool(10, 16, 1)
    a, b = pool.add_seq(0, 48), pool.add_seq(0, 48)
    pool.free_seq(a)
    n = ctypes.c_int32()
    one = np.zeros(1, np.int32)
    p = one.ctypes.data_as(ctypes.c_void_p)
    assert d.library().dora_pool_compact(pool.handle, p, p, 1, ctypes.byref(n)) == d.DORA_ERR_WORKSPACE_TOO_SMALL and n.value == 3
    assert pool.seq_pages(b).tolist() == [3, 4, 5]
    src, dst = pool.compact()
    assert src.tolist() == [3, 4, 5] and dst.tolist() == [0, 1, 2] and pool.seq_pages(b).tolist() == [0, 1, 2]
    assert [len(x) for x in pool.compact()] == [0, 0]
    assert pool.seq_pages(pool.add_seq(0, 20)).tolist() == [3, 4]


@pytest.mark.parametrize("seed", range(6))
def test_random_histories_keep_their_contents(d, seed):
    """A pool beside a model that keeps each sequence's tokens: adds, extensions, forks,
    releases, compactions and frees; what the pages hold follows the copies they ask for."""
    rng = np.random.default_rng(seed)
    P, n = 4, 60
    pool = d.Pool(n, P, 3, seed=seed)
    memory = np.full((n, P), -1, np.int64)
    model, stamp = {}, 0  # id -> [version, tokens, released pages]

    def write(sid, first):
        nonlocal stamp
        pages = pool.seq_pages(sid)
        for t in range(first, len(model[sid][1])):
            model[sid][1][t] = stamp
            memory[pages[t // P], t % P] = stamp
            stamp += 1

    for _ in range(300):
        op = rng.integers(0, 6)
        ids = list(model)
        try:
            if op == 0 or not ids:
                tokens = int(rng.integers(0, 20))
                v = int(rng.integers(0, 3))
                sid = pool.add_seq(v, tokens)
                model[sid] = [v, [None] * tokens, set()]
                write(sid, 0)
            elif op == 1:
                sid = ids[rng.integers(len(ids))]
                old = len(model[sid][1])
                new = old + int(rng.integers(0, 9))
                pool.extend_seq(sid, new)
                model[sid][1] += [None] * (new - old)
                write(sid, old)
            elif op == 2:
                sid = ids[rng.integers(len(ids))]
                v, tokens, gone = model[sid]
                k = len(tokens) if gone else int(rng.integers(0, len(tokens) + 1))
                new, src, dst = pool.fork_seq(sid, k)
                memory[dst] = memory[src]
                model[new] = [v, tokens[:k], set(gone)]
            elif op == 3:
                sid = ids[rng.integers(len(ids))]
                window, sinks = int(rng.integers(1, 12)), int(rng.integers(0, 6))
                pool.release_window(sid, window, sinks)
                L = len(model[sid][1])
                model[sid][2] |= {j for j in range(L // P) if j * P >= sinks and (j + 1) * P <= L - window}
            elif op == 4:
                src, dst = pool.compact()
                assert not set(src) & set(dst)
                memory[dst] = memory[src]
                memory[src] = -1
            else:
                sid = ids[rng.integers(len(ids))]
                pool.free_seq(sid)
                del model[sid]
        except d.DoraError as e:
            assert e.status == d.DORA_ERR_POOL_EXHAUSTED
        held = {}
        for sid, (v, tokens, gone) in model.items():
            pages = pool.seq_pages(sid)
            assert len(pages) == -(-len(tokens) // P)
            for j, pg in enumerate(pages):
                assert (pg == -1) == (j in gone)
                if pg >= 0:
                    held[pg] = v
                    part = tokens[j * P:(j + 1) * P]
                    assert memory[pg, :len(part)].tolist() == part
        owner = pool.page_owner()
        assert {int(p): int(owner[p]) for p in np.nonzero(owner >= 0)[0]} == {int(p): v for p, v in held.items()}
        assert pool.stats() == (len(held), n - len(held))
        for v in range(3):
            assert pool.stats(v)[0] == sum(x == v for x in held.values())

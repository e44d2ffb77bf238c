"""CPU checks of the operators that read less of the cache (4-bit pages, page bounds, page selection, attention
over listed pages, reads of the cache): refusals before any launch, sizes, what the binding hands on."""
import ctypes
import os

import numpy as np
import pytest
import torch

from fp4_util import bf16_of, bf16_value, dec4, enc4, get_keys, get_values, key_codes, put_keys, put_values, tile_bytes, value_codes


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


PTR, BIG = 1 << 20, 1 << 40  # an aligned address that is never read: every call here ends before a launch
BAD = [("null", None, 1), ("heads", dict(num_q_heads=9), 1), ("negative", dict(num_seqs=-1), 1), ("d", dict(head_dim=96), 2),
       ("page", dict(page_size=8), 2), ("group", dict(num_q_heads=34), 2), ("dtype", dict(kv_dtype=3), 2),
       ("scale", dict(sm_scale=float("nan")), 1), ("flags", dict(flags=2), 1)]


def _ref(desc):
    return None if desc is None else ctypes.byref(desc)


def _pages(d, desc, width=8, q=PTR, lists=PTR, counts=PTR, k=PTR, v=PTR, bt=PTR, lens=PTR, vers=None, out=PTR, ws=PTR, size=0):
    return d.library().dora_decode_attn_pages(_ref(desc), width, q, lists, counts, k, v, bt, lens, vers, out, ws, size, None)


def _select(d, desc, budget=8, sinks=1, recent=1, q=PTR, bounds=PTR, bt=PTR, lens=PTR, vers=None, lists=PTR, counts=PTR, scores=None, ws=PTR,
            size=0):
    return d.library().dora_page_select(_ref(desc), budget, sinks, recent, q, bounds, bt, lens, vers, lists, counts, scores, ws, size, None)


def _bounds(d, desc, T=4, counts=None, k=PTR, bt=PTR, lens=PTR, vers=None, bounds=PTR):
    return d.library().dora_kv_page_bounds(_ref(desc), T, counts, k, bt, lens, vers, bounds, None, None)


def _read(d, desc, T=4, counts=None, k=PTR, v=PTR, bt=PTR, lens=PTR, vers=None, ko=PTR, vo=PTR):
    return d.library().dora_kv_read(_ref(desc), T, counts, k, v, bt, lens, vers, ko, vo, None, None)


@pytest.mark.parametrize("call", [_pages, _select, _bounds, _read])
def test_bad_descriptors(d, call):
    for name, kw, status in BAD:
        assert call(d, None if kw is None else _desc(d, **kw)) == status, name
    for dt in (d.DORA_KV_BF16, d.DORA_KV_FP4):
        assert call(d, _desc(d, num_seqs=0, kv_dtype=dt)) == d.DORA_OK


def test_pages_refusals(d):
    for width in (0, -1, 1 << 19):
        assert _pages(d, _desc(d), width, size=BIG) == d.DORA_ERR_INVALID_ARG
        assert d.dora_decode_pages_workspace_bytes(_desc(d), width) == 0
    for name in ("q", "lists", "counts", "k", "v", "bt", "lens", "out", "ws"):
        assert _pages(d, _desc(d), size=BIG, **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("q", "k", "v", "out", "ws"):
        assert _pages(d, _desc(d), size=BIG, **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG, name
    assert _pages(d, _desc(d, kv_dtype=1), size=BIG) == d.DORA_ERR_INVALID_ARG  # fp8 without scales
    for dt in (0, d.DORA_KV_FP4):
        for width in (1, 8, 100, 5000, (1 << 19) - 1):
            need = d.dora_decode_pages_workspace_bytes(_desc(d, kv_dtype=dt), width)
            assert need >= 256
            assert _pages(d, _desc(d, kv_dtype=dt), width, size=need - 1) == d.DORA_ERR_WORKSPACE_TOO_SMALL


def test_select_refusals(d):
    for budget, sinks, recent in ((0, 0, 0), (-1, 0, 0), (1 << 19, 1, 1), (3, 2, 2), (3, -1, 1), (3, 1, -1), (5, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert _select(d, _desc(d), budget, sinks, recent, size=BIG) == d.DORA_ERR_INVALID_ARG, (budget, sinks, recent)
    for name in ("q", "bounds", "bt", "lens", "lists", "counts", "ws"):
        assert _select(d, _desc(d), size=BIG, **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    for name in ("q", "bounds", "ws"):
        assert _select(d, _desc(d), size=BIG, **{name: PTR + 4}) == d.DORA_ERR_INVALID_ARG, name
    need = d.dora_page_select_workspace_bytes(_desc(d))
    assert need >= 256 + 4 * 2 * 64 * 4
    assert _select(d, _desc(d), size=need - 1) == d.DORA_ERR_WORKSPACE_TOO_SMALL
    assert _select(d, _desc(d), scores=PTR, size=255) == d.DORA_ERR_WORKSPACE_TOO_SMALL


def test_bounds_and_read_refusals(d):
    for call in (_bounds, _read):
        for T in (0, -1, (1 << 19) + 1):
            assert call(d, _desc(d), T) == d.DORA_ERR_INVALID_ARG
        assert call(d, _desc(d, kv_dtype=1)) == d.DORA_ERR_INVALID_ARG  # fp8 without scales
        owner = torch.zeros(1024, dtype=torch.int16)
        assert call(d, _desc(d, flags=1, page_owner=owner)) == d.DORA_ERR_INVALID_ARG  # owners without versions
        for name in ("k", "bt", "lens"):
            assert call(d, _desc(d), **{name: None}) == d.DORA_ERR_INVALID_ARG, name
    assert _bounds(d, _desc(d), bounds=None) == d.DORA_ERR_INVALID_ARG
    assert _bounds(d, _desc(d), bounds=PTR + 8) == d.DORA_ERR_INVALID_ARG
    for name in ("v", "ko", "vo"):
        assert _read(d, _desc(d), **{name: None}) == d.DORA_ERR_INVALID_ARG
        assert _read(d, _desc(d), **{name: PTR + 8}) == d.DORA_ERR_INVALID_ARG


def test_calls_that_are_not_built_for_4_bit_pages(d):
    L, desc = d.library(), _desc(d, kv_dtype=d.DORA_KV_FP4)
    ref = ctypes.byref(desc)
    assert L.dora_decode_attn_tree(ref, 4, PTR, PTR, PTR, PTR, None, PTR, PTR, PTR, PTR, None, PTR, PTR, BIG, None) == d.DORA_ERR_UNSUPPORTED
    assert L.dora_decode_attn_window(ref, 10, 1, PTR, PTR, PTR, PTR, PTR, None, PTR, PTR, BIG, None) == d.DORA_ERR_UNSUPPORTED
    assert L.dora_decode_attn_grouped(ref, PTR, PTR, PTR, PTR, PTR, None, PTR, 2, None, PTR, BIG, None) == d.DORA_ERR_UNSUPPORTED
    assert d.dora_decode_tree_workspace_bytes(desc, 4) == 0
    assert d.dora_decode_window_workspace_bytes(desc, 10, 1) == 0
    assert d.dora_decode_grouped_workspace_bytes(desc, 2) == 0


def test_sizes(d):
    for heads, dim in ((1, 64), (3, 128), (8, 128), (127, 64)):
        used = heads * (2 * dim + 4)
        assert used <= d.dora_page_bounds_bytes(heads, dim) < used + 16 and d.dora_page_bounds_bytes(heads, dim) % 16 == 0
    assert d.dora_page_bounds_bytes(0, 64) == d.dora_page_bounds_bytes(128, 64) == d.dora_page_bounds_bytes(4, 96) == 0
    pack = lambda **kw: d.make_pack_desc(**{**dict(kv_dtype=d.DORA_KV_FP4, page_size=16, num_kv_heads=3, head_dim=64, num_pages=9, policy_version=0), **kw})  # noqa: E731
    assert d.dora_kv_packed_bytes(pack(), 5) == 256 + 2 * 5 * 3 * 544
    assert d.dora_kv_packed_bytes(pack(page_size=32, head_dim=128), 5) == 256 + 2 * 5 * 3 * 2176
    for kw in (dict(page_size=24), dict(head_dim=96)):  # no whole blocks of scales
        assert d.dora_kv_packed_bytes(pack(**kw), 5) == 0
    # the work of 4-bit pages is counted in steps of 64 tokens
    desc = _desc(d, kv_dtype=d.DORA_KV_FP4, block_table_stride=8)
    assert d.dora_decode_num_waves(desc) == 4 * 2 * 2 // 4
    assert d.dora_decode_workspace_bytes(desc) > 0
    assert d.dora_decode_num_waves(_desc(d, kv_dtype=d.DORA_KV_FP4, num_waves=77)) == 77


def test_what_the_binding_refuses(d):
    k4 = torch.zeros(9, 2, 1088, dtype=torch.uint8)
    bt, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    kw = dict(num_kv_heads=2, page_size=16, kv_dtype=d.DORA_KV_FP4)
    lists, counts = torch.zeros(3, 2, 5, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32)
    pages = lambda k=k4, v=k4, lists=lists, **more: d.dora_decode_attn_pages(q, lists, counts, k, v, bt, lens, None, q, **{**kw, **more})  # noqa: E731
    for bad in (k4[:, :, :1087], k4[:, :1], k4.view(9, 2, 1088, 1)):
        with pytest.raises(ValueError):
            pages(k=bad, v=bad)
    with pytest.raises(ValueError):
        pages(v=k4[:8])
    with pytest.raises(ValueError):
        pages(lists=lists[0])
    with pytest.raises(ValueError):
        pages(page_size=24)
    with pytest.raises(ValueError, match="GPU"):
        pages()
    with pytest.raises(ValueError, match="k_scales"):
        d.dora_decode_attn_pages(q, lists, counts, torch.zeros(9, 2, 8, 16, 16, dtype=torch.uint8), torch.zeros(9, 2, 128, 16, dtype=torch.uint8), bt,
                                 lens, None, q, num_kv_heads=2, page_size=16, kv_dtype=1)
    rows = torch.zeros(3, 6, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        d.dora_kv_read(k4, k4, bt, lens, rows[:, :, :1], rows, **kw)
    with pytest.raises(ValueError):
        d.dora_kv_read(k4, k4, bt[:2], lens, rows, rows, **kw)
    with pytest.raises(ValueError):
        d.dora_kv_page_bounds(k4, bt, lens, k4, num_tokens=1 << 31, head_dim=128, **kw)
    with pytest.raises(ValueError):
        d.dora_page_select(q, k4, bt, lens, lists[0], counts, num_kv_heads=2, page_size=16)
    with pytest.raises(ValueError):
        d.dora_page_select(q, k4, bt, lens, lists, counts, num_kv_heads=2, page_size=16, sink_pages=1 << 32)
    # nothing to do is done without a GPU
    none = lambda t: t[:0]  # noqa: E731
    assert d.dora_decode_attn_pages(none(q), none(lists), none(counts), k4, k4, none(bt), none(lens), None, none(q), **kw).shape[0] == 0
    d.dora_kv_read(k4, k4, none(bt), none(lens), none(rows), none(rows), **kw)
    d.dora_kv_page_bounds(k4, none(bt), none(lens), k4, num_tokens=1, head_dim=128, **kw)
    d.dora_page_select(none(q), k4, none(bt), none(lens), none(lists), none(counts), num_kv_heads=2, page_size=16)


def test_the_written_down_pages():
    """The definition that the GPU tests compare with, against brute force: every bf16 number as a block's largest, all
    ties, and what a tile gives back."""
    y = np.linspace(-8, 8, 2 ** 12 + 1)
    err = np.abs(dec4(enc4(y)) - y)
    every = np.array([dec4(np.uint8(c)) for c in range(16)])
    assert (err == np.abs(np.clip(y, -6, 6)[:, None] - every).min(1) + np.maximum(np.abs(y) - 6, 0)).all()
    for tie, even in ((0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5, 6)):
        assert enc4(np.array([tie])) == even and enc4(np.array([-tie])) == even + 8
    top = np.arange(1, 0x7F80, dtype=np.uint16)  # every positive finite bf16 number
    rows = np.zeros((len(top), 64), np.uint16)
    rows[:, 5] = top
    codes, e = key_codes(rows[:, :32])
    x = bf16_value(top).astype(np.float64)
    scale = np.exp2(e[:, 0].astype(np.float64) - 127)
    normal = (top >= 0x0180) & (top < 0x7F00)
    assert (np.abs(dec4(codes[:, 5]) * scale - x)[normal] <= scale[normal]).all()  # half a step of the largest codes, 4 to 6, is 1
    assert (x[normal] / scale[normal] >= 3.5).all() and (x[normal] / scale[normal] < 7).all()
    codes, s = value_codes(rows)
    steps = normal & (top >= 0x01C0)  # 6 * 2^-126: below, the scale is the smallest there is
    assert (codes[steps, 5] == 7).all()  # the largest is 6 steps
    rng = np.random.default_rng(0)
    for dim, P in ((64, 16), (128, 32)):
        tile, slot = np.zeros((2, tile_bytes(dim, P)), np.uint8), rng.permutation(P)[:11]
        x = bf16_of(rng.standard_normal((11, dim)))
        put_keys(tile[0], slot, *key_codes(x))
        put_values(tile[1], slot, *value_codes(x))
        codes, e = key_codes(x)
        assert np.array_equal(get_keys(tile[0], slot, dim), dec4(codes) * np.repeat(np.exp2(e - 127.0), 32, axis=1))
        codes, s = value_codes(x)
        assert np.array_equal(get_values(tile[1], slot, dim), dec4(codes) * np.repeat(bf16_value(s).astype(np.float64), 64, axis=1))

"""CPU checks of what the binding of the operators that read less of the cache refuses by itself."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def d():
    from paper_2604_26256_amd import build as B
    if not os.path.exists(B.LIB):
        B.build()
    from paper_2604_26256_amd import dora
    return dora


def _calls(d):
    """Each call as (function, its tensors by name, its other arguments)."""
    def i32(*shape):
        return torch.zeros(*shape, dtype=torch.int32)

    pool = dict(k_pages=torch.zeros(9, 2, 16 * 128 * 17 // 32, dtype=torch.uint8), v_pages=torch.zeros(9, 2, 16 * 128 * 17 // 32, dtype=torch.uint8))
    rows = dict(block_table=i32(3, 4), seq_lens=i32(3))
    lists = dict(page_lists=i32(3, 2, 5), page_counts=i32(3, 2))
    q, out = (torch.zeros(3, 8, 128, dtype=torch.bfloat16) for _ in range(2))
    k_out, v_out = (torch.zeros(3, 6, 2, 128, dtype=torch.bfloat16) for _ in range(2))
    bounds = torch.zeros(9, d.dora_page_bounds_bytes(2, 128), dtype=torch.uint8)
    kw = dict(num_kv_heads=2, page_size=16)
    kw4 = dict(kw, kv_dtype=d.DORA_KV_FP4)
    return [(d.dora_kv_read, dict(**pool, **rows, k_out=k_out, v_out=v_out), kw4),
            (d.dora_kv_page_bounds, dict(k_pages=pool["k_pages"], **rows, bounds=bounds), dict(kw4, num_tokens=1, head_dim=128)),
            (d.dora_page_select, dict(q=q, bounds=bounds, **rows, **lists), kw),
            (d.dora_decode_attn_pages, dict(q=q, **lists, **pool, **rows, out=out), dict(kw4, version_ids=None))]


def test_a_missing_tensor_is_named(d):
    for call, tensors, kw in _calls(d):
        with pytest.raises(ValueError, match="GPU"):  # all there: the first that is not on a GPU is named
            call(**tensors, **kw)
        for name in tensors:
            with pytest.raises(ValueError, match=f"{name} is required"):
                call(**{**tensors, name: None}, **kw)


@pytest.mark.parametrize("shape", [(), (3, 1), (2,)])
def test_lengths_of_another_shape_are_refused(d, shape):
    for call, tensors, kw in _calls(d):
        with pytest.raises(ValueError):
            call(**{**tensors, "seq_lens": torch.zeros(shape, dtype=torch.int32)}, **kw)


def test_bounds_of_another_shape_are_refused(d):
    for call, tensors, kw in _calls(d)[1:3]:
        for shape in ((), (9,), (9, 5), (9, 1, 528)):
            with pytest.raises(ValueError):
                call(**{**tensors, "bounds": torch.zeros(shape, dtype=torch.uint8)}, **kw)

"""CPU checks of what the binding hands on for the operators around the cache."""
import os

import pytest


@pytest.fixture(scope="module")
def d():
    from paper_2604_26256_amd import build as B
    if not os.path.exists(B.LIB):
        B.build()
    from paper_2604_26256_amd import dora
    return dora


@pytest.mark.parametrize("more", [1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 32) + 5, 1 << 40])
def test_counts_past_32_bits_are_refused(d, more):
    """2^32 + 5 is no window of 5: its pages would be gone."""
    pool = d.Pool(40, 16, 1)
    a = pool.add_seq(0, 300)
    for call in (lambda: pool.release_window(a, more), lambda: pool.release_window(a, 5, more), lambda: pool.fork_seq(a, more)):
        with pytest.raises(ValueError):
            call()
    assert pool.stats() == (19, 21) and (pool.seq_pages(a) >= 0).all()
    desc = d.make_decode_desc(num_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, block_table_stride=64, num_pages=99)
    for call in (lambda: d.dora_decode_tree_workspace_bytes(desc, more), lambda: d.dora_decode_window_workspace_bytes(desc, more, 1),
                 lambda: d.dora_decode_window_workspace_bytes(desc, 1, more)):
        with pytest.raises(ValueError):
            call()
    assert pool.release_window(a, (1 << 31) - 1, 0) == 0
    assert pool.release_window(a, 5, (1 << 31) - 1) == 0

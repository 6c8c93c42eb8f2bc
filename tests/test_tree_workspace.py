"""What attn_tree's workspace has to hold never shrinks with the step: one made for an engine's largest step serves every smaller one."""
import ctypes

import pytest

from paper_2512_22560_amd import binding as B

KINDS = [(B.F32, B.F32), (B.BF16, B.BF16), (B.BF16, B.FP8_E4M3), (B.BF16, B.FP8_E4M3_HEAD), (B.BF16, B.INT8_HEAD)]


def size(q, kv, heads, d, total, most, batch=64, pages=1024):
    desc = B.Desc(batch=batch, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d, page_size=16, max_pages_per_seq=pages, num_pages=5,
                  q_dtype=q, kv_dtype=kv, sm_scale=0.1, k_scale=0x1000, v_scale=0x1000)
    got = B.lib().rollattn_tree_workspace_bytes(ctypes.byref(desc), total, most)
    assert got > 0
    return got


def never_less(sizes):
    sizes = list(sizes)
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("heads", [(2, 2), (8, 4), (32, 8), (64, 4), (24, 8), (40, 1), (256, 1)])
@pytest.mark.parametrize("q,kv", KINDS)
def test_more_rows_need_no_less(q, kv, heads):
    for d in (64, 128):
        for pages in (1, 64, 65, 1024):
            never_less(size(q, kv, heads, d, 4096, most, pages=pages) for most in range(0, 200))
            for most in (1, 7, 72, 199):
                never_less(size(q, kv, heads, d, total, most, pages=pages) for total in (*range(0, 200), 1000, 4096))


@pytest.mark.parametrize("q,kv", KINDS)
def test_more_trajectories_and_wider_tables_need_no_less(q, kv):
    for most in (1, 4, 8, 16, 72):
        never_less(size(q, kv, (64, 4), 128, 4096, most, batch=batch) for batch in range(0, 700))
        never_less(size(q, kv, (64, 4), 128, 4096, most, pages=pages) for pages in (1, 63, 64, 65, 66, 1000, 4000))

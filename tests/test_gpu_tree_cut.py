"""Attention of drafts under tables with more pages than any trajectory has: such a table's rows are cut over workgroups and joined, where
narrow ones are not, so what holds of the small drafts of test_gpu_tree is asked again.  Tolerances are that file's: a joined row is a sum of
float32 sums."""
import numpy as np
import pytest
import torch

from tests import test_gpu_tree as narrow
from tests.tree_common import KINDS, any_masks, drafts, tree_masks

pytestmark = pytest.mark.gpu
PAGES = 200


def widened(*args, **kw):
    b = drafts(*args, **kw)
    more = PAGES - b.page_table.shape[1]
    if more > 0:
        b.page_table = torch.cat([b.page_table, torch.full((len(b.page_table), more), -1, dtype=torch.int32, device=b.page_table.device)], 1).contiguous()
    return b


@pytest.fixture(autouse=True)
def wide_tables(monkeypatch):
    monkeypatch.setattr(narrow, "drafts", widened)


@pytest.mark.parametrize("masks", [tree_masks, any_masks])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS[1:])
def test_drafts_of_all_kinds_of_lengths(src, kv, d, masks):
    narrow.test_drafts_of_all_kinds_of_lengths(src, kv, d, masks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS[1:])
def test_query_rows_around_tiles(src, kv, d):
    """4 heads to a KV head: 32, 64, 128 and 256 query rows are whole tiles of one, two, four and eight waves."""
    for most in (7, 8, 9, 16, 17, 32, 33, 64, 65, 130):
        b = widened((8, 2), d, src, kv, ("uniform", 0, 700), ("uniform", 0, most), most, batch=5)
        if b.total_q:
            narrow.check(b, any_masks(b, most), f"{most}")


@pytest.mark.parametrize("src,kv", KINDS[1:])
def test_rows_that_see_nothing(src, kv):
    narrow.test_rows_that_see_nothing(src, kv)


@pytest.mark.parametrize("edge", [0, 1, 16, 31, 32, 33, 65])
def test_prefixes_around_pages_and_blocks(edge):
    narrow.test_prefixes_around_pages_and_blocks(edge)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "int8_head"])
def test_many_trajectories(kv):
    narrow.test_many_trajectories(kv)


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS[1:4])
def test_undefined_values_of_nodes_that_a_row_does_not_see(src, kv, d, kind):
    narrow.test_undefined_values_of_nodes_that_a_row_does_not_see(src, kv, d, kind)


def test_infinite_values_reach_the_rows_that_see_them():
    narrow.test_infinite_values_reach_the_rows_that_see_them("bf16")


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3_head"])
def test_rows_behind_the_last_draft_stay(kv):
    narrow.test_rows_behind_the_last_draft_stay(kv)


def test_negative_and_zero_scales_of_the_softmax():
    narrow.test_negative_and_zero_scales_of_the_softmax()


@pytest.mark.parametrize("src,kv", KINDS[1:])
def test_understated_longest_draft(src, kv):
    """Nodes past max_q_len are answered wrongly or not at all; the others as ever, and nothing else is written."""
    for heads, most, said in (((8, 2), 20, 8), ((8, 2), 40, 16), ((8, 1), 60, 20), ((4, 4), 90, 33)):
        for make in (drafts, widened):
            b = make(heads, 64, src, kv, ("uniform", 0, 300), ("uniform", 1, most), 7)
            mask = any_masks(b, 3)
            want = narrow.call(b, mask)
            lens = b.q_lens_host.copy()
            out = torch.full_like(want, 5.0)
            lse = torch.full((b.total_q, heads[0]), 5.0, device=want.device)
            narrow.B.attn_tree(b.q, b.q_lens, b.q_offsets, narrow.on_device(mask), b.k_pages, b.v_pages, b.page_table, b.ctx_lens,
                               sm_scale=b.workload.sm_scale, max_q_len=said, k_scale=b.k_scale, v_scale=b.v_scale, out=out, lse=lse)
            first = np.concatenate([np.arange(n) < said for n in lens])
            keep = torch.from_numpy(first).to(want.device)
            assert (out[keep].float() - want[keep].float()).abs().max() <= 2 ** -6 * want.float().abs().max()

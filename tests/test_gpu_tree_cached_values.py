"""Values of cached tokens that are no numbers, under drafts: every row sees those tokens, so every row's output is no number where theirs
are, wherever the prefix ends in a page, a block of 32 tokens or a worker's run; the other dims and the denominators stay as they are, bit for
bit (what a dim comes to is a sum over its own values alone)."""
import numpy as np
import pytest
import torch

from oracle import tree as T
from paper_2512_22560_amd import workloads as W
from tests.helpers import oracle_args
from tests.test_gpu_tree import call
from tests.test_gpu_tree_cut import widened
from tests.tree_common import KINDS, any_masks, drafts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# heads and nodes of a draft: 12, 48, 96 and 160 query rows to a KV head, which are one, two, four and eight waves', and two tiles of eight
SHAPES = [((8, 2), 3), ((8, 2), 12), ((8, 2), 24), ((8, 2), 40), ((16, 1), 20)]
PREFIXES = (1, 16, 31, 32, 33, 97, 112, 127)
TABLES = {"narrow": drafts, "wide": widened}


def values_at(b, row, token):
    """V of one cached token of a trajectory, [Hkv, D]."""
    return b.v_pages[int(b.page_table[row, token // 16]), :, token % 16]


def strange(kv):
    """What goes into the first dims of a value, and what a row that sees it has there."""
    if kv.startswith("fp8"):
        return (0x7F, 0xFF), (float("nan"), float("nan"))
    inf = float("inf")
    return (float("nan"), inf, -inf), (float("nan"), inf, -inf)


@pytest.mark.parametrize("table", TABLES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS[:4])
def test_values_of_cached_tokens_reach_every_row(src, kv, d, table):
    bits, want = strange(kv)
    for heads, new in SHAPES:
        for prefix in PREFIXES:
            b = TABLES[table](heads, d, src, kv, ("const", prefix), ("const", new), 7 * prefix + new, batch=3)
            mask = any_masks(b, prefix)
            lse = [torch.zeros((b.total_q, heads[0]), device=DEV) for _ in range(2)]
            before = call(b, mask, lse=lse[0]).float()
            for token in {prefix - 1, (prefix - 1) // 32 * 32}:                   # the last, and the first of its block
                kept = [values_at(b, t, token).clone() for t in range(3)]
                for t in range(3):
                    for dim, x in enumerate(bits):
                        values_at(b, t, token)[:, dim] = x
                got = call(b, mask, lse=lse[1]).float()
                what = f"{heads} {new} nodes behind {prefix}, token {token}"
                for dim, x in enumerate(want):
                    there = got[:, :, dim]
                    assert (torch.isnan(there) if x != x else there == x).all(), f"{what}: dim {dim} has {there[~(torch.isnan(there) if x != x else there == x)][:3].tolist()}"
                assert torch.equal(got[:, :, len(want):], before[:, :, len(want):]) and torch.equal(*lse), what
                for t in range(3):
                    values_at(b, t, token)[:] = kept[t]


@pytest.mark.parametrize("table", TABLES)
@pytest.mark.parametrize("src,kv", [("bf16", "bf16"), ("bf16", "fp8_e4m3_head")])
def test_values_of_cached_tokens_and_of_nodes(src, kv, table):
    """Both at once, in neighbouring places: numbers and what is none stand where the definition has them."""
    bits, _ = strange(kv)
    for heads, new in SHAPES:
        b = TABLES[table](heads, 64, src, kv, ("uniform", 3, 70), ("const", new), new, batch=5)
        mask = any_masks(b, new)
        for t in range(5):
            prefix = int(b.ctx_lens_host[t]) - new
            for dim, x in enumerate(bits):
                values_at(b, t, prefix - 1 - dim)[:, 4 * dim] = x       # of a cached token, a dim of its own each
                values_at(b, t, prefix + dim)[:, 4 * dim + 1] = x       # of a node
        with np.errstate(invalid="ignore"):
            ref, _, most = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **oracle_args(b))
        got = call(b, mask).double().cpu().numpy()
        finite = np.isfinite(ref)
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]), heads
        # (values of a standard normal: below 6 where they are numbers)
        assert np.abs(got[finite] - ref[finite]).max() <= (2.0 ** -7 + 1e-4) * 6, heads

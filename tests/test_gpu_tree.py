"""Attention of drafts on the GPU against its definition in float64.

Tolerances, from what is rounded.  A row's output is sum w v / sum w.  16-bit queries: weights are rounded to bf16 (or, with scales per
head, to f16) for the second product, off by at most half a step, 2^-8 of themselves, so the sum is off by 2^-8 of sum w |v| / sum w at
most, that is of the largest |v| that the row sees; the result is rounded to bf16, another 2^-8 of itself.  Together 2^-7 of the
largest |v|.  Sums and exponentials in float32 add less than 1e-4 of it (scores below 64, 2^-24 a step).  float32 queries have the
latter alone.  The denominator's log2 takes unrounded weights: 1e-4."""
import numpy as np
import pytest
import torch

from oracle import tree as T
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.helpers import oracle_args
from tests.tree_common import KINDS, any_masks, drafts, on_device, tree_masks, words_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def call(b, mask, **kw):
    return B.attn_tree(b.q, b.q_lens, b.q_offsets, on_device(mask) if isinstance(mask, np.ndarray) else mask, b.k_pages, b.v_pages, b.page_table, b.ctx_lens,
                       sm_scale=b.workload.sm_scale, max_q_len=int(max(1, b.q_lens_host.max(initial=1))), k_scale=b.k_scale, v_scale=b.v_scale, **kw)


def close(got, lse, b, mask, what=""):
    ref, ref_lse, most = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **oracle_args(b))
    got = got.detach().double().cpu().numpy()
    tol = ((0.0 if b.workload.q_dtype == "f32" else 2.0 ** -7) + 1e-4) * most[:, :, None]
    assert np.isfinite(got).all(), what
    bad = np.argwhere(np.abs(got - ref) > tol)
    assert bad.size == 0, f"{what}: {len(bad)} of {got.size} off, first {bad[0].tolist()}: {got[tuple(bad[0])]} for {ref[tuple(bad[0])]}"
    if lse is not None:
        l = lse.double().cpu().numpy()
        seen = np.isfinite(ref_lse)
        assert np.array_equal(seen, np.isfinite(l)) and (l[~seen] == -np.inf).all(), what
        assert np.abs(l[seen] - ref_lse[seen]).max(initial=0.0) <= 1e-4, what


def check(b, mask, what="", with_lse=True):
    lse = torch.full((b.total_q, b.workload.num_q_heads), 7.0, device=DEV) if with_lse else None
    out = call(b, mask, lse=lse)
    torch.cuda.synchronize()
    close(out, lse, b, mask, what)


@pytest.mark.parametrize("masks", [tree_masks, any_masks])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS)
def test_drafts_of_all_kinds_of_lengths(src, kv, d, masks):
    for heads, prefix, new, seed in (((4, 2), ("uniform", 0, 40), ("uniform", 0, 9), 1), ((8, 1), ("uniform", 30, 200), ("uniform", 1, 17), 2),
                                     ((2, 2), ("uniform", 0, 3), ("uniform", 20, 90), 3), ((20, 4), ("uniform", 500, 900), ("const", 1), 4)):
        b = drafts(heads, d, src, kv, prefix, new, seed)
        check(b, masks(b, seed), f"{heads} {prefix} {new}")


@pytest.mark.parametrize("src,kv", KINDS)
def test_one_token_after_another(src, kv):
    """A chain's mask is the causal one: what attn_append gives."""
    b = drafts((8, 2), 128, src, kv, ("uniform", 0, 300), ("uniform", 1, 30), 11)
    parents = np.concatenate([np.arange(n) - 1 for n in b.q_lens_host])
    mask, _ = T.tree_mask(parents, b.q_lens_host, b.ctx_lens_host, words_of(b))
    check(b, mask)


@pytest.mark.parametrize("src,kv", KINDS)
def test_rows_that_see_nothing(src, kv):
    """No cached tokens and no bits: zero, and -inf; the tokens it does not see are there."""
    b = drafts((6, 2), 64, src, kv, ("const", 0), ("uniform", 1, 40), 5)
    mask = np.zeros((b.total_q, 1), dtype=np.uint64)
    lse = torch.zeros((b.total_q, 6), device=DEV)
    out = call(b, mask, lse=lse)
    assert (out == 0).all() and (lse == -np.inf).all()
    mask[::2] = 1
    check(b, mask)


@pytest.mark.parametrize("edge", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65])
def test_prefixes_around_pages_and_blocks(edge):
    for n in (1, 2, 15, 16, 17, 33, 64, 65):
        b = drafts((4, 1), 128, "bf16", "bf16", ("const", edge), ("const", n), 100 * edge + n, batch=2)
        check(b, any_masks(b, n), f"{edge} {n}")


@pytest.mark.parametrize("src,kv", KINDS)
def test_long_contexts(src, kv):
    for heads, new, batch in (((8, 2), ("uniform", 1, 9), 3), ((16, 2), ("uniform", 30, 70), 2)):
        b = drafts(heads, 128, src, kv, ("uniform", 3000, 9000), new, 21, batch=batch)
        check(b, tree_masks(b, 1), f"{heads}")


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "int8_head"])
def test_many_trajectories(kv):
    b = drafts((8, 2), 64, "bf16", kv, ("uniform", 0, 80), ("uniform", 0, 6), 31, batch=300)
    check(b, any_masks(b, 3))


@pytest.mark.parametrize("src,kv", KINDS)
def test_large_drafts_of_several_words(src, kv):
    b = drafts((4, 4), 64, src, kv, ("uniform", 10, 100), ("uniform", 130, 300), 41, batch=2)
    check(b, tree_masks(b, 1), "tree")
    check(b, any_masks(b, 2), "any")
    # fewer words than nodes: the nodes past them are seen by nobody
    narrow = any_masks(b, 3)[:, :1].copy()
    check(b, narrow, "narrow")


def spoil(b, token, kind):
    """Token `token` of every trajectory's draft: keys and values that are no numbers, in every head."""
    for pool in (b.k_pages, b.v_pages):
        for t in range(len(b.q_lens_host)):
            if b.q_lens_host[t] <= token:
                continue
            at = int(b.ctx_lens_host[t] - b.q_lens_host[t]) + token
            row = pool[int(b.page_table[t, at // 16]), :, at % 16]
            if b.workload.kv_dtype.startswith("fp8"):
                row[:, ::3] = 0x7F if kind != 1 else 0xFF
            else:
                row[:, ::3] = (float("nan"), float("inf"), -float("inf"))[kind]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS[:4])
def test_undefined_values_of_nodes_that_a_row_does_not_see(src, kv, d, kind):
    for heads, new in (((4, 1), 13), ((8, 2), 40)):
        b = drafts(heads, d, src, kv, ("uniform", 0, 100), ("const", new), 51, batch=5)
        mask = any_masks(b, 7)
        node = np.uint64(1) << np.uint64(9)
        mask &= ~node
        whole, ref_lse = call(b, mask), None
        spoil(b, 9, kind)
        lse = torch.zeros((b.total_q, heads[0]), device=DEV)
        got = call(b, mask, lse=lse)
        assert torch.isfinite(got.float()).all() and torch.equal(got, whole)
        # a row that sees it has what the formula has: its keys are no numbers either
        mask[::5] |= node
        got = call(b, mask).float()
        sees = torch.zeros(b.total_q, dtype=torch.bool)
        sees[::5] = True
        assert torch.isnan(got[sees.to(DEV)]).all(dim=2).all() if kind == 0 else not torch.isfinite(got[sees.to(DEV)]).all()
        rest = ~sees.to(DEV)
        assert torch.equal(got[rest], whole.float()[rest])


@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_infinite_values_reach_the_rows_that_see_them(src):
    b = drafts((4, 2), 64, src, src, ("uniform", 5, 60), ("const", 6), 61, batch=3)
    mask = tree_masks(b, 1) & ~np.uint64(4)
    mask[::6] |= np.uint64(4)
    before = call(b, mask).float()
    for t in range(3):
        at = int(b.ctx_lens_host[t]) - 6 + 2
        row = b.v_pages[int(b.page_table[t, at // 16]), :, at % 16]
        row[:, 0], row[:, 1] = float("inf"), -float("inf")
    got = call(b, mask).float()
    sees = torch.zeros(b.total_q, dtype=torch.bool, device=DEV)
    sees[::6] = True
    assert (got[sees][:, :, 0] == float("inf")).all() and (got[sees][:, :, 1] == -float("inf")).all()
    assert torch.equal(got[sees][:, :, 2:], before[sees][:, :, 2:]) and torch.equal(got[~sees], before[~sees])


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3_head"])
def test_rows_behind_the_last_draft_stay(kv):
    b = drafts((8, 2), 128, "bf16", kv, ("uniform", 0, 200), ("uniform", 1, 12), 71)
    mask = any_masks(b, 1)
    more = 5
    q = torch.cat([b.q, torch.full((more,) + tuple(b.q.shape[1:]), float("nan"), dtype=b.q.dtype, device=DEV)])
    out, lse = torch.full_like(q, 3.0), torch.full((len(q), 8), 3.0, device=DEV)
    wide = np.concatenate([mask, np.full((more, mask.shape[1]), 2 ** 64 - 1, dtype=np.uint64)])
    B.attn_tree(q, b.q_lens, b.q_offsets, on_device(wide), b.k_pages, b.v_pages, b.page_table, b.ctx_lens, sm_scale=b.workload.sm_scale,
                max_q_len=int(b.q_lens_host.max()) + 3, k_scale=b.k_scale, v_scale=b.v_scale, out=out, lse=lse)
    assert (out[-more:] == 3).all() and (lse[-more:] == 3).all()
    close(out[:-more], lse[:-more], b, mask)


def test_negative_and_zero_scales_of_the_softmax():
    for scale in (-0.3, 0.0, 2.0):
        for src, kv in KINDS:
            b = drafts((4, 2), 64, src, kv, ("uniform", 0, 90), ("uniform", 1, 10), 81)
            mask = any_masks(b, 5)
            out = B.attn_tree(b.q, b.q_lens, b.q_offsets, on_device(mask), b.k_pages, b.v_pages, b.page_table, b.ctx_lens, sm_scale=scale,
                              max_q_len=int(b.q_lens_host.max()), k_scale=b.k_scale, v_scale=b.v_scale)
            ref, _, most = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **dict(oracle_args(b), sm_scale=scale))
            tol = ((0.0 if src == "f32" else 2.0 ** -7) + 1e-4) * most[:, :, None]
            assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all(), (scale, kv)


def test_pages_far_behind_in_a_large_pool():
    """Offsets past 32 bits, in bytes and in elements."""
    b = drafts((8, 8), 128, "bf16", "bf16", ("uniform", 100, 200), ("uniform", 1, 12), 91, batch=3)
    mask = any_masks(b, 1)
    want = call(b, mask)
    n, room = b.k_pages.shape[0], 300000
    for name in ("k_pages", "v_pages"):
        pool = torch.empty((room,) + tuple(b.k_pages.shape[1:]), dtype=torch.bfloat16, device=DEV)
        pool[room - n:] = getattr(b, name)
        setattr(b, name, pool)
    b.page_table += room - n
    assert torch.equal(call(b, mask), want)


def test_the_same_bits_again_and_any_placement_of_pages():
    b = drafts((16, 2), 128, "bf16", "int8_head", ("uniform", 0, 3000), ("uniform", 1, 9), 101, batch=20)
    mask = on_device(any_masks(b, 1))
    want = call(b, mask)
    assert torch.equal(call(b, mask), want)
    perm = torch.randperm(b.k_pages.shape[0], generator=torch.Generator().manual_seed(1)).to(DEV)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        t = getattr(b, name)
        moved = torch.empty_like(t)
        moved[perm] = t
        setattr(b, name, moved)
    b.page_table = torch.where(b.page_table >= 0, perm[b.page_table.clamp_min(0).long()].to(torch.int32), -1).contiguous()
    assert torch.equal(call(b, mask), want)

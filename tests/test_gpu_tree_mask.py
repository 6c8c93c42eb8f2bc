"""Masks and positions of drafts on the GPU: whole numbers, equal to the definition's."""
import numpy as np
import pytest
import torch

from oracle import tree as T
from paper_2512_22560_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)


def check(parents, lens, ctx, words=None, max_q_len=None, behind=0):
    lens, ctx = np.asarray(lens), np.asarray(ctx)
    words = words or max(1, -(-int(lens.max(initial=1)) // 64))
    total = int(lens.sum())
    mask = torch.full((total + behind, words), -7, dtype=torch.int64, device=DEV)
    positions = torch.full((total + behind,), -7, dtype=torch.int32, device=DEV)
    given = np.concatenate([np.asarray(parents), np.full(behind, 3)])
    got = B.attn_tree_mask(ints(given), ints(lens), ints(np.concatenate([[0], np.cumsum(lens)])), ints(ctx), max_q_len=max_q_len or int(lens.max(initial=1)),
                           tree_mask=mask, positions=positions)
    assert got[0] is mask and got[1] is positions
    want, places = T.tree_mask(parents, lens, ctx, words)
    assert np.array_equal(mask[:total].cpu().numpy().view(np.uint64), want)
    assert np.array_equal(positions[:total].cpu().numpy(), places)
    assert (mask[total:] == -7).all() and (positions[total:] == -7).all()


def parents_of(lens, kind, seed=0):
    rng, out = np.random.default_rng(seed), []
    for n in lens:
        i = np.arange(n)
        out.append({"chain": i - 1, "star": np.where(i > 0, 0, -1), "roots": np.full(n, -1), "binary": (i + 1) // 2 - 1,
                    "any": np.array([rng.integers(-1, max(1, j)) if j else -1 for j in i], dtype=np.int64)}[kind])
    return np.concatenate(out or [np.zeros(0, np.int64)])


@pytest.mark.parametrize("kind", ["chain", "star", "roots", "binary", "any"])
def test_trees_of_all_sizes(kind):
    for lens in ([1], [0, 3, 0], [1, 2, 15, 16, 17, 31, 32, 33], [63, 64], [65], [64, 128, 129, 7], [500, 1], [1024]):
        check(parents_of(lens, kind), lens, np.asarray(lens) + 100 * np.arange(len(lens)))


def test_many_small_trees():
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 20, 3000)
    check(parents_of(lens, "any", 5), lens, lens + rng.integers(0, 9, 3000), behind=3)


@pytest.mark.parametrize("lens", [[20, 3], [100, 70, 200]])
def test_more_and_fewer_words_than_nodes(lens):
    for words in (1, 2, 5, 16):
        check(parents_of(lens, "any", 2), lens, np.asarray(lens) + 7, words=words, behind=2)


def test_parents_that_are_none():
    """Nodes of no lower number, and numbers below -1, are no parents."""
    lens = [9, 80]
    parents = parents_of(lens, "any", 3)
    parents[2], parents[4], parents[5], parents[9 + 70], parents[9 + 40] = 2, 8, -5, 79, 1 << 30
    check(parents, lens, [50, 90])


def test_a_longest_draft_that_is_over_and_understated():
    check(parents_of([5, 20], "any", 4), [5, 20], [8, 30], max_q_len=500)
    for most in (1, 17):
        check(parents_of([5, 90, 200], "any", 4), [5, 90, 200], [8, 95, 300], max_q_len=most)


def test_allocated_outputs():
    mask, positions = B.attn_tree_mask(ints([-1, 0, 0, 2]), ints([4]), ints([0, 4]), ints([10]), max_q_len=4)
    assert mask.tolist() == [[1], [3], [5], [13]] and positions.tolist() == [6, 7, 7, 8]

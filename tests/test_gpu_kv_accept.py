"""The move of accepted rows on the GPU against its definition, bit for bit: pools and scales."""
import numpy as np
import pytest
import torch

from oracle import tree as T
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.tree_common import KINDS, drafts, parents_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)


def some(b, seed, share=0.5):
    """Nodes at random of every draft, ascending; now and then none or all."""
    rng, rows, lens = np.random.default_rng(seed), [], []
    for t, n in enumerate(b.q_lens_host.tolist()):
        keep = rng.random(n) < (share if t % 4 else rng.choice([0.0, 1.0]))
        nodes = np.nonzero(keep)[0]
        rows.append(np.concatenate([nodes, np.full(n - len(nodes), 99999)]))
        lens.append(len(nodes))
    return np.concatenate(rows).astype(np.int64), np.array(lens)


def paths(b, seed):
    parents, rng, rows, lens, at = parents_of(b, seed), np.random.default_rng(seed), [], [], 0
    for n in b.q_lens_host.tolist():
        i, path = int(rng.integers(0, n)) if n else -1, []
        while i >= 0:
            path.append(i)
            i = int(parents[at + i])
        rows.append(np.array(path[::-1] + [-1] * (n - len(path)), dtype=np.int64))
        lens.append(len(path))
        at += n
    return np.concatenate(rows), np.array(lens)


def check(b, accepted, lens, what="", max_q=None):
    pools = [b.k_pages.clone(), b.v_pages.clone()]
    scales = [None if s is None else s.clone() for s in (b.k_scale, b.v_scale)]
    B.kv_accept(ints(accepted), ints(lens), b.q_lens, b.q_offsets, *pools, b.page_table, b.ctx_lens, max_q_len=max_q or int(max(1, b.q_lens_host.max(initial=1))),
                k_scale=scales[0], v_scale=scales[1])
    want = T.accept(accepted, lens, b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table), W.raw_numpy(b.k_pages), W.raw_numpy(b.v_pages),
                    kv_dtype=b.workload.kv_dtype, k_scale=W.raw_numpy(b.k_scale), v_scale=W.raw_numpy(b.v_scale))
    bits = lambda x: x.view(np.uint32) if x.dtype == np.float32 else x
    for name, g, r in zip(("k", "v", "k_scale", "v_scale"), pools + scales, want):
        if r is None:
            assert g is None
            continue
        bad = np.argwhere(bits(W.raw_numpy(g)) != bits(np.ascontiguousarray(r)))
        assert bad.size == 0, f"{what}: {name} differs at {bad[:4].tolist()} ({len(bad)} elements)"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS)
def test_paths_and_any_nodes(src, kv, d):
    for heads, prefix, new, seed in (((4, 2), ("uniform", 0, 40), ("uniform", 0, 9), 1), ((1, 1), ("uniform", 0, 40), ("uniform", 1, 30), 2),
                                     ((8, 8), ("uniform", 0, 17), ("uniform", 20, 120), 3), ((24, 24), ("const", 15), ("uniform", 2, 40), 4),
                                     ((72, 72), ("uniform", 0, 20), ("uniform", 1, 20), 5)):
        b = drafts(heads, d, src, kv, prefix, new, seed)
        check(b, *paths(b, seed), f"path {heads}")
        check(b, *some(b, seed), f"any {heads}")
        check(b, *some(b, seed, 0.9), f"most {heads}")


@pytest.mark.parametrize("src,kv", KINDS)
def test_large_drafts(src, kv):
    b = drafts((2, 2), 64, src, kv, ("uniform", 0, 20), ("uniform", 200, 500), 11, batch=3)
    check(b, *some(b, 1), "any")
    check(b, *some(b, 1, 0.1), "few")
    check(b, *some(b, 2), "understated", max_q=8)


@pytest.mark.parametrize("kv", ["fp8_e4m3", "fp8_e4m3_head", "int8_head"])
def test_loud_and_faint_pages(kv):
    """Scales of neighbouring pages a hundred and a million apart: rows arrive from louder and from fainter pages."""
    b = drafts((4, 4), 64, "bf16", kv, ("uniform", 0, 40), ("uniform", 20, 90), 21)
    gen = torch.Generator().manual_seed(3)
    for s in (b.k_scale, b.v_scale):
        s *= torch.exp(torch.randn(s.shape, generator=gen) * 5).to(DEV)
    for seed in range(3):
        check(b, *some(b, seed), f"{seed}")


@pytest.mark.parametrize("src,kv", KINDS)
def test_nothing_is_accepted_or_all_of_it(src, kv):
    b = drafts((4, 2), 128, src, kv, ("uniform", 0, 40), ("uniform", 1, 30), 31)
    accepted = np.concatenate([np.arange(n) for n in b.q_lens_host])
    pools = [b.k_pages.clone(), b.v_pages.clone()]
    for lens in (np.zeros(7, dtype=np.int64), b.q_lens_host):
        B.kv_accept(ints(accepted), ints(lens), b.q_lens, b.q_offsets, b.k_pages, b.v_pages, b.page_table, b.ctx_lens, max_q_len=30, k_scale=b.k_scale, v_scale=b.v_scale)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(pools, (b.k_pages, b.v_pages)))   # (as bytes: dead places hold undefined values)


def test_many_trajectories():
    b = drafts((2, 2), 64, "bf16", "int8_head", ("uniform", 0, 40), ("uniform", 0, 12), 41, batch=600)
    check(b, *paths(b, 1))


def test_pages_far_behind_in_a_large_pool():
    b = drafts((8, 8), 128, "bf16", "bf16", ("uniform", 0, 40), ("uniform", 10, 40), 51)
    accepted, lens = some(b, 1)
    want = [b.k_pages.clone(), b.v_pages.clone()]
    B.kv_accept(ints(accepted), ints(lens), b.q_lens, b.q_offsets, *want, b.page_table, b.ctx_lens, max_q_len=40)
    n, room = b.k_pages.shape[0], 300000
    got = []
    for t in (b.k_pages, b.v_pages):
        pool = torch.empty((room,) + tuple(t.shape[1:]), dtype=t.dtype, device=DEV)
        pool[room - n:] = t
        got.append(pool)
    B.kv_accept(ints(accepted), ints(lens), b.q_lens, b.q_offsets, *got, b.page_table + (room - n), b.ctx_lens, max_q_len=40)
    assert all(np.array_equal(W.raw_numpy(g[room - n:]), W.raw_numpy(w)) for g, w in zip(got, want))

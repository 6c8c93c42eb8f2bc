"""Drafts for the tests of the calls around them."""
from __future__ import annotations

import numpy as np
import torch

from oracle import tree as T
from paper_2512_22560_amd import workloads as W

KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8_e4m3"), ("bf16", "fp8_e4m3_head"), ("bf16", "int8_head")]


def drafts(heads, d, src, kv, prefix, new, seed, batch=7, device="cuda:0"):
    """Pools, tables and queries of a batch whose last `new` tokens are drafts (places that no token has hold undefined values)."""
    return W.build(W.Workload("t", batch, heads[0], heads[1], d, src, kv, prefix, qlen=new, seed=seed, ctx_is_prefix=True), device)


def words_of(b):
    return max(1, -(-int(b.q_lens_host.max(initial=1)) // 64))


def parents_of(b, seed, chain=False):
    rng, out = np.random.default_rng(seed), []
    for n in b.q_lens_host.tolist():
        i = np.arange(n)
        out.append(i - 1 if chain else np.maximum(i - 1 - rng.exponential(2.0, n).astype(np.int64), -1))
    return np.concatenate(out or [np.zeros(0)]).astype(np.int32)


def tree_masks(b, seed):
    return T.tree_mask(parents_of(b, seed), b.q_lens_host, b.ctx_lens_host, words_of(b))[0]


def any_masks(b, seed):
    """Bits at random, of places past the draft too; some rows with none."""
    rng = np.random.default_rng(seed)
    bits = rng.integers(0, 1 << 63, (b.total_q, words_of(b)), dtype=np.uint64) * np.uint64(2) + rng.integers(0, 2, (b.total_q, words_of(b)), dtype=np.uint64)
    bits[rng.random(b.total_q) < 0.3] = 0
    return bits


def on_device(mask, device="cuda:0"):
    return torch.from_numpy(mask.view(np.int64).copy()).to(device)

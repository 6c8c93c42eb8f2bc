"""Multi-turn rollouts over an 8-bit cache: observations and tokens of one attention layer, from the projection to its output.

    python examples/rollout_8bit.py            (on a machine with an MI355X)

Every turn, the new tokens of all trajectories go through the layer's projection, whose output holds q, k and v of a token side
by side.  `kv_write_rope` reads it as it is: it rotates queries and keys to their positions, quantises keys and values with a scale
for each page and KV head, and puts them into the pages.  `attn_append` (an observation arrived) or `attn_decode` (one token each)
attends over the cache.  Images among the observations have positions in time, height and width; text counts along on all three.
The result is compared with attention in float32 over the unquantised history.
"""
from __future__ import annotations

import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_22560_amd import binding as ra  # noqa: E402

PAGE = 16


class Cache:
    """Pools of one layer, and the pages of every trajectory."""

    def __init__(self, batch, hkv, d, max_tokens, dtype, device):
        per_seq = -(-max_tokens // PAGE)
        shape = (batch * per_seq, hkv, PAGE, d)
        self.k, self.v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        self.k_scale, self.v_scale = (torch.ones(shape[:2], device=device) for _ in range(2))
        self.free = np.random.default_rng(0).permutation(shape[0]).tolist()
        self.table = np.full((batch, per_seq), -1, dtype=np.int32)
        self.lens = np.zeros(batch, dtype=np.int64)

    def extend(self, new):
        """Room for `new` more tokens of every trajectory."""
        for b, n in enumerate(new):
            for p in range(-(-int(self.lens[b]) // PAGE), -(-int(self.lens[b] + n) // PAGE)):
                self.table[b, p] = self.free.pop()
        self.lens += new


def rotary_table(positions, rot_dim, base=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def rollout(dtype=torch.int8, turns=((37, 5, 130, 0), (1, 1, 1, 1), (1, 1, 1, 1), (20, 64, 3, 1)), heads=(16, 4, 128), seed=0, device="cuda:0"):
    """The turns' new tokens per trajectory; returns the largest error of an output, relative to the rms of all."""
    hq, hkv, d = heads
    batch, width = len(turns[0]), 256
    gen = torch.Generator(device=device).manual_seed(seed)
    weight = (torch.randn((width, (hq + 2 * hkv) * d), generator=gen, device=device) / math.sqrt(width)).to(torch.bfloat16)
    cache = Cache(batch, hkv, d, sum(max(t) for t in turns), dtype, device)
    cos_sin = rotary_table(1024, d).to(device)
    pair_axes = [0] * (d // 2 - 2 * (3 * d // 16)) + [1] * (3 * d // 16) + [2] * (3 * d // 16)
    history = [[] for _ in range(batch)]
    ints = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).to(device)
    worst, scale = 0.0, 1.0 / math.sqrt(d)
    for new in turns:
        new = np.asarray(new)
        start = cache.lens.copy()
        cache.extend(new)
        at = np.concatenate([np.arange(s, s + n) for s, n in zip(start, new)])
        image = (at // 16) % 2 == 1                        # every other 16 tokens are a 4 x 4 image
        positions = np.stack([np.where(image, at - at % 16, at), np.where(image, at - at % 16 + at % 16 // 4, at), np.where(image, at - at % 16 + at % 4, at)])
        offsets = np.concatenate([[0], np.cumsum(new)])
        hidden = torch.randn((int(new.sum()), width), generator=gen, device=device).to(torch.bfloat16)
        q, k, v = (hidden @ weight).view(-1, hq + 2 * hkv, d).split([hq, hkv, hkv], dim=1)
        lens = (ints(new), ints(offsets))
        where = (ints(cache.table), ints(cache.lens))
        scales = dict(k_scale=cache.k_scale, v_scale=cache.v_scale)
        most = int(new.max())
        q = ra.kv_write_rope(q, k, v, *lens, cache.k, cache.v, *where, cos_sin=cos_sin, positions=ints(positions), pair_axes=pair_axes,
                             max_q_len=most, **scales)
        if (new == 1).all():
            out = ra.attn_decode(q, cache.k, cache.v, *where, sm_scale=scale, **scales)
        else:
            out = ra.attn_append(q, *lens, cache.k, cache.v, *where, sm_scale=scale, max_q_len=most, **scales)
        # the same in float32, nothing quantised
        turn = torch.from_numpy(positions).to(device)[torch.tensor(pair_axes, device=device)].T
        pair = torch.arange(d // 2, device=device)
        c, s = cos_sin[turn, pair][:, None], cos_sin[turn, pair + d // 2][:, None]
        lo, hi = k.float().split(d // 2, dim=2)
        turned = torch.cat([lo * c - hi * s, hi * c + lo * s], dim=2)
        plain = torch.zeros_like(out, dtype=torch.float32)
        for b in range(batch):
            rows = slice(int(offsets[b]), int(offsets[b + 1]))
            history[b].append((turned[rows], v[rows].float()))
            keys, values = (torch.cat([h[i] for h in history[b]]).repeat_interleave(hq // hkv, dim=1) for i in range(2))
            for i in range(int(new[b])):
                seen = int(start[b]) + i + 1
                p = torch.softmax((keys[:seen] * q[offsets[b] + i].float()).sum(-1) * scale, dim=0)
                plain[offsets[b] + i] = (p[:, :, None] * values[:seen]).sum(0)
        worst = max(worst, float((out.float() - plain).abs().max() / plain.square().mean().sqrt()))
    return worst


if __name__ == "__main__":
    for dtype in (torch.int8, torch.uint8):
        print(f"{'int8' if dtype == torch.int8 else 'E4M3'} cache: largest error of an output {rollout(dtype):.3f} of their rms")

"""Plain definitions of what a step with drafted tokens does: visibility of trees, attention under it, the norm in front of the
rotation, the move of the accepted rows.

TEST INFRASTRUCTURE ONLY -- see the package docstring.  numpy only; loops over trajectories, nodes, heads and pages, nothing blocked
or fused.

A draft is n_b nodes behind the L_b - n_b cached tokens of trajectory b; L_b counts them.
  tree_mask   node i sees itself and, as long as a parent in [0, i) is given, its ancestors; its position is L_b - n_b plus the
              number of its ancestors
  attn_tree   row i sees the cached tokens and node j of its draft where bit j % 64 of its word j / 64 is set; softmax over what it
              sees, in float64; a row that sees nothing is zero, its denominator's log2 -inf.  What a row does not see takes no part.
  normalise   (x * r) * weight, r = 1 / sqrt(mean(x^2) + eps), every product, quotient and root one float32 operation; squares in
              float32, four neighbours' (a + b) + (c + d) in float32, these in float64, the mean rounded to float32 once
  accept      rows accepted[0] < accepted[1] < .. of a draft move to its places 0, 1, ..  8-bit pools, per page that a row moves into
              (and KV head where scales are per head): need = largest |code * scale of its page| among the rows that come from other
              pages / 448 or / 127; now = max(scale, need); the page's rows up to the last accepted one: enc(code * scale of its page /
              now), each product and quotient one float32 operation, or the codes as they are where the scale of their page is now
              already (products with a subnormal scale would not come back as they went)
The published method of scoring drafts as a tree and the root-mean-square norm; the paper this library serves prints nothing to check
against.
"""
from __future__ import annotations

import numpy as np

from .attention import decode_storage, gather_tokens
from .kv_write import E4M3_MAX, PAGE, _e4m3fn_to_float32, float32_to_e4m3fn
from .kv_write_rope import _int8

__all__ = ["tree_mask", "attn_tree", "normalise", "accept"]


def tree_mask(parents, q_lens, ctx_lens, words):
    masks, positions, at = [], [], 0
    for n, length in zip(q_lens, ctx_lens):
        for i in range(int(n)):
            bits, depth, j = 0, 0, i
            while True:
                bits |= 1 << j
                p = int(parents[at + j])
                if not 0 <= p < j:
                    break
                j, depth = p, depth + 1
            masks.append([(bits >> (64 * w)) & (2 ** 64 - 1) for w in range(words)])
            positions.append(int(length) - int(n) + depth)
        at += int(n)
    return np.array(masks, dtype=np.uint64).reshape(-1, words), np.array(positions, dtype=np.int32)


def attn_tree(q, q_lens, mask, k_pages, v_pages, page_table, ctx_lens, *, sm_scale, q_dtype, kv_dtype, k_scale=None, v_scale=None):
    """(out float64 [total_q, Hq, D], lse [total_q, Hq] in log2 units, the largest |v| that a row's KV head holds for it, same shape)."""
    q = decode_storage(q, q_dtype)
    total, hq, d = q.shape
    hkv = k_pages.shape[1]
    group = hq // hkv
    out, lse, most = np.zeros((total, hq, d)), np.full((total, hq), -np.inf), np.zeros((total, hq))
    scale, row = np.float64(np.float32(sm_scale)), 0
    mask = np.asarray(mask).astype(np.uint64)
    for b in range(len(q_lens)):
        n, length = int(q_lens[b]), int(ctx_lens[b])
        for g in range(hkv if n else 0):
            k = gather_tokens(k_pages, page_table, b, g, length, kv_dtype, k_scale)
            v = gather_tokens(v_pages, page_table, b, g, length, kv_dtype, v_scale)
            for i in range(n):
                sees = np.arange(length) < length - n
                for j in range(min(n, 64 * mask.shape[1])):
                    sees[length - n + j] = (int(mask[row + i, j // 64]) >> (j % 64)) & 1
                if not sees.any():
                    continue
                for h in range(g * group, (g + 1) * group):
                    z = scale * (k[sees] @ q[row + i, h])
                    top = z.max()
                    w = np.exp(z - top)
                    out[row + i, h] = (w @ v[sees]) / w.sum()
                    lse[row + i, h] = (top + np.log(w.sum())) / np.log(2.0)
                    most[row + i, h] = np.abs(v[sees]).max()
        row += n
    return out, lse, most


def normalise(x, weight, eps):
    """x [..., D] float32."""
    x = np.asarray(x, dtype=np.float32)
    s = (x * x).astype(np.float32).reshape(x.shape[:-1] + (-1, 4))
    fours = ((s[..., 0] + s[..., 1]).astype(np.float32) + (s[..., 2] + s[..., 3]).astype(np.float32)).astype(np.float32)
    mean = (fours.astype(np.float64).sum(axis=-1) / x.shape[-1]).astype(np.float32)
    r = (np.float32(1.0) / np.sqrt((mean + np.float32(eps)).astype(np.float32))).astype(np.float32)
    return ((x * r[..., None]).astype(np.float32) * np.asarray(weight, dtype=np.float32)).astype(np.float32)


def accept(accepted, accept_lens, q_lens, ctx_lens, page_table, k_pages, v_pages, *, kv_dtype, k_scale=None, v_scale=None):
    """Returns (k_pages, v_pages, k_scale, v_scale); inputs are not modified.  accepted packed like the drafts."""
    codes, int8, per_head = kv_dtype not in ("f32", "bf16"), kv_dtype == "int8_head", kv_dtype in ("fp8_e4m3_head", "int8_head")
    enc = _int8 if int8 else float32_to_e4m3fn
    dec = (lambda c: c.astype(np.float32)) if int8 else _e4m3fn_to_float32
    qmax = np.float32(127.0) if int8 else E4M3_MAX
    pools, scales = [np.array(p, copy=True) for p in (k_pages, v_pages)], [None if s is None else np.array(s, dtype=np.float32, copy=True) for s in (k_scale, v_scale)]
    offs = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int64)
    for b in range(len(q_lens)):
        first, m = int(ctx_lens[b]) - int(q_lens[b]), int(accept_lens[b])
        nodes = [int(x) for x in accepted[offs[b]:offs[b] + m]]
        assert all(x < y for x, y in zip(nodes, nodes[1:])) and (not nodes or nodes[-1] < q_lens[b])
        moves = {}
        for i, node in enumerate(nodes):
            moves.setdefault((first + i) // PAGE, []).append((first + i, first + node))
        for page_i, rows in moves.items():
            if all(d == s for d, s in rows):
                continue
            page, s0 = int(page_table[b, page_i]), rows[0][0] % PAGE
            came = [(d % PAGE, int(page_table[b, s // PAGE]), s % PAGE) for d, s in rows]
            for pool, scale in zip(pools, scales):
                src = [pool[p, :, s].copy() for _, p, s in came]                 # [Hkv, D] each
                if not codes:
                    for (d, _, _), x in zip(came, src):
                        pool[page, :, d] = x
                    continue
                hkv = pool.shape[1]
                for h in (range(hkv) if per_head else [slice(None)]):
                    at = (lambda p: (p, h)) if per_head else (lambda p: p)
                    x = [(dec(c[h]) * scale[at(p)]).astype(np.float32) for (_, p, _), c in zip(came, src)]
                    amax = max([np.float32(np.max(np.abs(y))) for y, (_, p, _) in zip(x, came) if p != page], default=np.float32(0))
                    old, froms = scale[at(page)], {p: scale[at(p)] for _, p, _ in came}
                    now = max(old, np.float32(amax / qmax))
                    if now > old:
                        pool[page, h, :s0] = enc(((dec(pool[page, h, :s0]) * old).astype(np.float32) / now).astype(np.float32))
                    for (d, p, _), c, y in zip(came, src, x):
                        pool[page, h, d] = c[h] if froms[p] == now else enc((y / now).astype(np.float32))
                    scale[at(page)] = now
    return pools[0], pools[1], scales[0], scales[1]

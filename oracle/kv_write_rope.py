"""Plain definition of the KV write with the position rotation on the way.

TEST INFRASTRUCTURE ONLY -- see the package docstring.  numpy only; loops over trajectories, pages and heads, nothing blocked
or fused.

What it defines.  Of the first rot_dim dimensions of a head, pair j of rot_dim / 2 is (j, j + rot_dim / 2), or (2 j, 2 j + 1)
where interleaved; a token at position p turns it to
    lo' = lo * c - hi * s,   hi' = hi * c + lo * s,   c = cos_sin[p, j], s = cos_sin[p, rot_dim / 2 + j]
with every product and sum one float32 operation, in that order; the other dimensions stay.  p is the token's place in its
context, L_b - n_b + i for new row i of trajectory b, or positions[axis of the pair, row]; outside the table it is the table's
last row.  Queries are rounded once to their type.  Rotated keys, and values as they are, go to the places that kv_write states:
rounded once into pools of the source type, quantised into the others.  Pools with one scale for a page follow kv_write's rule;
in those with a scale for each page and head ("fp8_e4m3_head", "int8_head"), per page that receives rows in slots [s0, s1) and per
head:
    need = max(amax / qmax, 2**-64), amax over the head's new rows of the page, qmax 448 or 127
    fresh page (s0 == 0): scale = need;  else scale = max(old, need), and where that exceeds the old scale the codes in slots
    [0, s0) become enc(dec(code) * old / scale)
    new rows: code = enc(x / scale), int8 codes nearest even and clamped to [-127, 127]
Rotary positions are the published method; the paper this library serves prints nothing to check against.
"""
from __future__ import annotations

import numpy as np

from .kv_write import E4M3_MAX, PAGE, _e4m3fn_to_float32, _to_float32, float32_to_e4m3fn

__all__ = ["float32_to_bf16", "rotate", "kv_write_rope"]

LEAST = np.float32(2.0 ** -64)


def float32_to_bf16(x) -> np.ndarray:
    """Round finite float32 values to bf16 bit patterns, nearest, ties to even."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def _int8(x) -> np.ndarray:
    return np.clip(np.rint(x), -127, 127).astype(np.int8)


def rotate(x, rows, cos_sin, interleaved=False) -> np.ndarray:
    """x [T, heads, D] float32; rows [T, pairs]: the table's row for each pair of each token."""
    x, t = np.asarray(x, dtype=np.float32), np.asarray(cos_sin, dtype=np.float32)
    half = t.shape[1] // 2
    rows = np.asarray(rows, dtype=np.int64)
    rows = np.where((rows < 0) | (rows >= t.shape[0]), t.shape[0] - 1, rows)
    c, s = t[rows, np.arange(half)][:, None, :], t[rows, half + np.arange(half)][:, None, :]
    first = 2 * np.arange(half) if interleaved else np.arange(half)
    second = first + (1 if interleaved else half)
    lo, hi = x[..., first], x[..., second]
    y = x.copy()
    y[..., first] = (lo * c).astype(np.float32) - (hi * s).astype(np.float32)
    y[..., second] = (hi * c).astype(np.float32) + (lo * s).astype(np.float32)
    return y


def kv_write_rope(q, k_new, v_new, q_lens, ctx_lens, page_table, k_pages, v_pages, *, src_dtype, kv_dtype, cos_sin=None,
                  positions=None, pair_axes=None, interleaved=False, k_scale=None, v_scale=None):
    """Returns (q_out, k_pages, v_pages, k_scale, v_scale); inputs are not modified.  cos_sin None: no rotation (q may be None)."""
    q_lens, ctx_lens = np.asarray(q_lens, dtype=np.int64), np.asarray(ctx_lens, dtype=np.int64)
    back = (lambda y: y) if src_dtype == "f32" else float32_to_bf16
    k, v = _to_float32(k_new, src_dtype), _to_float32(v_new, src_dtype)
    q_out = q
    if cos_sin is not None:
        half = np.shape(cos_sin)[1] // 2
        place = np.concatenate([np.arange(l - n, l) for l, n in zip(ctx_lens, q_lens)] or [np.zeros(0, np.int64)])
        axes = np.zeros(half, dtype=np.int64) if pair_axes is None else np.asarray(list(pair_axes), dtype=np.int64)
        rows = np.repeat(place[:, None], half, axis=1) if positions is None else np.atleast_2d(positions)[axes].T
        k = rotate(k, rows, cos_sin, interleaved)
        if q is not None:
            q_out = back(rotate(_to_float32(q, src_dtype), rows, cos_sin, interleaved))
    k_pages, v_pages = np.array(k_pages, copy=True), np.array(v_pages, copy=True)
    codes = kv_dtype not in ("f32", "bf16")
    int8, per_head = kv_dtype == "int8_head", kv_dtype in ("fp8_e4m3_head", "int8_head")
    if codes:
        k_scale, v_scale = np.array(k_scale, dtype=np.float32, copy=True), np.array(v_scale, dtype=np.float32, copy=True)
    enc = _int8 if int8 else float32_to_e4m3fn
    dec = (lambda c: c.astype(np.float32)) if int8 else _e4m3fn_to_float32
    qmax = np.float32(127.0) if int8 else E4M3_MAX
    row = 0
    for b in range(len(q_lens)):
        pos, end = int(ctx_lens[b] - q_lens[b]), int(ctx_lens[b])
        while pos < end:
            page, s0 = int(page_table[b, pos // PAGE]), pos % PAGE
            count = min(PAGE - s0, end - pos)
            for x, pool, scale in ((k, k_pages, k_scale), (v, v_pages, v_scale)):
                new = np.swapaxes(x[row:row + count], 0, 1)                       # [Hkv, slots, D]
                if not codes:
                    pool[page, :, s0:s0 + count] = back(new)
                    continue
                heads = [slice(h, h + 1) for h in range(new.shape[0])] if per_head else [slice(None)]
                for i, h in enumerate(heads):
                    at = (page, i) if per_head else page
                    need = np.float32(np.float32(np.max(np.abs(new[h]))) / qmax)
                    if per_head:
                        need = max(need, LEAST)
                    elif s0 == 0 and need == 0:
                        need = np.float32(1.0)
                    old = scale[at] if s0 else need
                    now = max(old, need)
                    if now > old:
                        kept = (dec(pool[page, h, :s0]) * old).astype(np.float32)
                        pool[page, h, :s0] = enc((kept / now).astype(np.float32))
                    pool[page, h, s0:s0 + count] = enc((new[h] / now).astype(np.float32))
                    scale[at] = now
            pos, row = pos + count, row + count
    return q_out, k_pages, v_pages, k_scale, v_scale

"""The operators of a step with drafted tokens over a paged cache as callable cases.

A draft is a tree of guessed tokens behind a trajectory's cached tokens.  One step of an engine that works so makes the tree's
visibility and positions from its nodes' parents, writes the nodes' keys (normalised and rotated to their positions) and values
into the pages, attends from every node to the cached tokens and its own ancestors, and afterwards moves the rows of the path that
was accepted to where the trajectory goes on.  Every case is one call of one operator with the buffers an engine keeps made
beforehand.  Lengths and trees belong to the case (drawn from its `lengths` seed), values, placement of the pages and, where they
are the operator's input, parents to the seed that `prepare` is given.  Head shapes, batch sizes and lengths are those of the
workloads that the repository states, and smaller ones of the same kind.

Kinds of case:
  draft    attn_tree_mask: parents to visibility bits and positions
  write    kv_write_norm_rope: q and k of the new tokens, as one projection leaves them, are normalised by head and rotated, q is
           handed back, k and v go into the pages
  tree     attn_tree: a draft attends to its context
  accept   kv_accept: the accepted rows move together

With `own` false the operators are computed in elementary torch operations in 32 bits, else by the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
ITEM = {"bf16": 2, "fp8": 1, "int8": 1}
QMAX = {"fp8": 448.0, "int8": 127.0}
TINY = 2.0 ** -64            # the least scale of a page and head
BASE = 10000.0               # of the rotation's frequencies
EPS = 1e-6                   # of the norms


def _case(kind, batch, heads, kv, prefix, new, lengths, name=None, tree=True):
    """prefix, new: least and most cached and new tokens of a trajectory; tree: the new ones are a draft, else they follow each other."""
    c = {"kind": kind, "batch": batch, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "kv": kv, "prefix_lo": prefix[0],
         "prefix_hi": prefix[1], "new_lo": new[0], "new_hi": new[1], "lengths": lengths, "tree": tree}
    return c if name is None else dict(c, name=name)


def listed():
    a, b, tiny = (32, 8, 128), (64, 4, 128), (8, 2, 64)
    return [
        # the last few trajectories of a rollout draft: launches and latency
        _case("draft", 5, a, "bf16", (2048, 32767), (5, 24), 1, name="draft_few"),
        # a whole batch with large drafts, several words of bits to a node
        _case("draft", 512, a, "bf16", (64, 8191), (32, 200), 2, name="draft_b512"),
        # the drafts of a handful of trajectories go into the cache
        _case("write", 5, a, "bf16", (7, 64), (5, 24), 3, name="write_norm_bf16_few"),
        # those of a whole batch, E4M3 pages
        _case("write", 256, b, "fp8", (0, 63), (3, 17), 4, name="write_norm_fp8_b256"),
        # observations of a whole batch, int8 pages: the largest write
        _case("write", 64, a, "int8", (0, 40), (64, 1024), 5, name="write_norm_int8_chunks_b64", tree=False),
        # the last few long trajectories draft
        _case("tree", 3, a, "bf16", (2048, 32767), (5, 16), 6, name="tree_bf16_few"),
        # short histories with small heads, some of them not begun yet
        _case("tree", 37, tiny, "fp8", (0, 300), (1, 9), 7, name="tree_fp8_short_d64"),
        # an ordinary step of a batch
        _case("tree", 64, a, "bf16", (512, 8191), (6, 16), 8, name="tree_bf16_b64"),
        # a large batch, many query heads to a KV head, short drafts: the most bytes
        _case("tree", 160, b, "int8", (1024, 16383), (2, 4), 9, name="tree_int8_b160"),
        # wide drafts, many query heads to a KV head: the most operations
        _case("tree", 24, b, "bf16", (1024, 8191), (24, 72), 10, name="tree_bf16_wide_b24"),
        # a handful of trajectories goes on
        _case("accept", 5, a, "bf16", (2048, 8191), (5, 24), 11, name="accept_bf16_few"),
        # a whole batch, int8 pages
        _case("accept", 512, b, "int8", (64, 512), (16, 64), 12, name="accept_int8_b512"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; none has more bytes or operations than the largest listed ones."""
    while True:
        kind = rng.choice(["draft", "write", "tree", "tree", "accept"])
        heads = rng.choice([(32, 8, 128), (64, 4, 128), (64, 8, 128), (8, 2, 64)])
        kv = rng.choice(["bf16", "fp8", "int8"])
        batch = _log_int(rng, 1, 512)
        seed = rng.randrange(1 << 30)
        lo, hi = sorted((_log_int(rng, 1, 200), _log_int(rng, 1, 200)))
        p, q = sorted((_log_int(rng, 1, 32768) - 1, _log_int(rng, 1, 32768) - 1))
        if kind == "write" and rng.random() < 0.4:
            c = _case(kind, batch, heads, kv, (0, rng.randrange(8, 64)), (lo, 5 * hi), seed, tree=False)
        elif kind in ("write", "accept"):
            c = _case(kind, batch, heads, kv, (min(p, 256), min(q, 512)), (lo, hi), seed)
        else:
            c = _case(kind, batch, heads, kv, (p, q), (lo, hi), seed)
        w = work(c)
        ctx, new = _lengths(c)
        padded = len(ctx) * int(ctx.max())
        if kind == "draft" or (w["bytes"] <= 1.1e9 and w["flops"] <= 2.5e11 and padded * heads[1] * heads[2] <= 4.4e9 and
                               (kind != "tree" or padded * heads[0] * int(new.max()) <= 7e9)):
            return c


def _lengths(c):
    """Tokens in the cache, the new ones among them, and new tokens, of every trajectory."""
    rng = np.random.default_rng(c["lengths"])
    n = c["batch"]
    new = np.exp(rng.uniform(math.log(c["new_lo"]), math.log(c["new_hi"] + 1), n)).astype(np.int64).clip(c["new_lo"], c["new_hi"])
    if c["prefix_hi"] - c["prefix_lo"] < 1000:
        prefix = rng.integers(c["prefix_lo"], c["prefix_hi"] + 1, n)
    else:                                         # long histories: many short ones, few long ones
        lo, hi = c["prefix_lo"] + 1, c["prefix_hi"] + 1
        prefix = np.exp(rng.uniform(math.log(lo), math.log(hi), n)).astype(np.int64).clip(lo, hi) - 1
    return prefix + new, new


def _parents(new, seed):
    """Of every node: a node shortly before it, mostly; now and then none, as the first of every draft."""
    rng = np.random.default_rng(seed)
    i = np.concatenate([np.arange(n) for n in new.tolist()])
    back = 1 + rng.exponential(2.0, len(i)).astype(np.int64)
    return np.maximum(i - back, np.where(rng.random(len(i)) < 0.02, -1, np.minimum(i - 1, 0)))


def _depths(new, parents):
    """How many ancestors every node has."""
    depth, at = np.zeros(len(parents), dtype=np.int64), 0
    for n in new.tolist():
        for i in range(n):
            depth[at + i] = 0 if parents[at + i] < 0 else depth[at + parents[at + i]] + 1
        at += n
    return depth


def _accepted(c, new):
    """The path to one node of every draft: [total] nodes, packed like the drafts, and how many there are."""
    parents, rng = _parents(new, c["lengths"] + 1), np.random.default_rng(c["lengths"] + 2)
    rows, lens, at = np.zeros(len(parents), dtype=np.int64), np.zeros(len(new), dtype=np.int64), 0
    for b, n in enumerate(new.tolist()):
        i, path = int(rng.integers(0, n)), []
        while i >= 0:
            path.append(i)
            i = int(parents[at + i])
        rows[at:at + len(path)], lens[b] = path[::-1], len(path)
        at += n
    return rows, lens


def _quantised(x, kv):
    """Pages as codes and a scale for each page and head."""
    scale = (x.abs().amax(dim=(2, 3)) / torch.full((), QMAX[kv], device=x.device)).clamp_min(TINY)
    return _encode(x / scale[:, :, None, None], kv), scale


def _encode(x, kv):
    if kv == "int8":
        return x.round().clamp(-127, 127).to(torch.int8)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _seen_bits(new, parents, words):
    """Visibility as an engine keeps it: [total, words] of 64 bits, bit j of a node's for node j of its draft."""
    bits, at = np.zeros((len(parents), words), dtype=np.uint64), 0
    for n in new.tolist():
        for i in range(n):
            if parents[at + i] >= 0:
                bits[at + i] = bits[at + parents[at + i]]
            bits[at + i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
        at += n
    return bits.view(np.int64)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    ctx, new = _lengths(case)
    hq, hkv, d, kv, kind = case["q_heads"], case["kv_heads"], case["head_dim"], case["kv"], case["kind"]

    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(np.asarray(x).astype(np.int32))).to(dev)

    total, words = int(new.sum()), (int(new.max()) + 63) // 64
    s = {"kind": kind, "kv": kv, "max_q": int(new.max()), "scale": 1.0 / math.sqrt(d), "k_scale": None, "v_scale": None, "words": words,
         "ctx": ints(ctx), "new": ints(new), "off": ints(np.concatenate([[0], np.cumsum(new)]))}
    if kind == "draft":
        s["parents"] = ints(_parents(new, seed))
        return s
    pages = (ctx + PAGE - 1) // PAGE
    used = int(pages.sum())
    place = torch.randperm(used, generator=gen, device=dev).to(torch.int32)
    table = np.full((len(ctx), max(1, int(pages.max()))), -1, dtype=np.int64)
    first = np.concatenate([[0], np.cumsum(pages)])
    for b, n in enumerate(pages.tolist()):
        table[b, :n] = np.arange(first[b], first[b] + n)
    logical = torch.from_numpy(table).to(dev)
    s["table"] = torch.where(logical >= 0, place[logical.clamp_min(0)], -1).to(torch.int32).contiguous()

    def values(n, heads, loud):
        """Heads are not equally loud, and neither are a head's channels: keys more than values."""
        x = torch.randn((n, heads, d), generator=gen, device=dev)
        return x.mul_(torch.exp(loud * torch.randn((heads, 1), generator=gen, device=dev) + loud * torch.randn((heads, d), generator=gen, device=dev)))

    for name, loud in (("k", 0.3), ("v", 0.1)):
        shape = (used, hkv, PAGE, d)
        if kv == "bf16":
            s[name] = torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16)
            continue
        s[name] = torch.empty(shape, device=dev, dtype=torch.int8 if kv == "int8" else torch.float8_e4m3fn)
        s[name + "_scale"] = torch.empty((used, hkv), device=dev)
        for p in range(0, used, 16384):            # (a slab at a time: in 32 bits the pool would be four times as large)
            n = min(16384, used - p)
            x = values(n * PAGE, hkv, loud).view(n, PAGE, hkv, d).transpose(1, 2)
            s[name][p:p + n], s[name + "_scale"][p:p + n] = _quantised(x, kv)
    if kv == "fp8":
        s["k"], s["v"] = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
    if kind == "accept":
        rows, lens = _accepted(case, new)
        s["rows"], s["lens"] = ints(rows), ints(lens)
        return s
    parents = _parents(new, case["lengths"] + 1)
    if kind == "tree":
        s["q"] = torch.randn((total, hq, d), generator=gen, device=dev).to(torch.bfloat16)
        s["mask"] = torch.from_numpy(_seen_bits(new, parents, words)).to(dev)
        return s
    # what the projection leaves: q, k and v of a token side by side
    rows = torch.cat([values(total, h, loud) for h, loud in ((hq, 0.1), (hkv, 0.3), (hkv, 0.1))], dim=1).to(torch.bfloat16)
    s["q"], s["k_new"], s["v_new"] = rows.split([hq, hkv, hkv], dim=1)
    s["q_weight"], s["k_weight"] = (1.0 + 0.2 * torch.randn((2, d), generator=gen, device=dev)).unbind(0)
    half = d // 2
    angle = torch.arange(int(ctx.max()) + 64, device=dev, dtype=torch.float64)[:, None] * BASE ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32)
    s["positions"] = ints(np.repeat(ctx - new, new) + _depths(new, parents)) if case["tree"] else None
    return s


def _flat(s):
    """Trajectory of every new token, and its number among that trajectory's."""
    n = s["new"].long()
    total = s["k_new"].shape[0] if "k_new" in s else next(s[x].shape[0] for x in ("q", "parents", "rows") if x in s)
    b = torch.repeat_interleave(torch.arange(len(n), device=n.device), n, output_size=total)
    return b, torch.arange(total, device=n.device) - s["off"].long()[b]


def _plain_draft(s):
    b, i = _flat(s)
    n_b, most, parents = len(s["new"]), s["max_q"], s["parents"].long()
    reach = torch.eye(most, device=b.device).expand(n_b, -1, -1).clone()
    has = parents >= 0
    reach[b, i, parents.clamp_min(0)] += has.float()
    reach[b, i, i] = 1.0
    for _ in range(max(1, (most - 1).bit_length())):               # ancestors of 1, 2, 4, ... steps
        reach = torch.matmul(reach, reach).clamp_max(1.0)
    seen = torch.zeros((len(b), s["words"] * 64), dtype=torch.int64, device=b.device)
    seen[:, :most] = reach[b, i].long()
    mask = (seen.view(len(b), -1, 64) << torch.arange(64, device=b.device)).sum(dim=-1)
    return {"mask": mask, "positions": (s["ctx"].long()[b] - s["new"].long()[b] + seen.sum(dim=1) - 1).to(torch.int32)}


def _normed(x, weight):
    """By the mean square of each head's row: squares in 32 bits, four neighbours' at a time, the rest of the sum in 64."""
    x = x.float()
    y = (x * x).unflatten(-1, (-1, 4))
    sums = ((y[..., 0] + y[..., 1]) + (y[..., 2] + y[..., 3])).double().sum(dim=-1)
    t = torch.sqrt((sums / x.shape[-1]).float() + torch.full((), EPS, device=x.device))
    return (x * (torch.ones_like(t) / t)[..., None]) * weight


def _rotated(x, cos, sin):
    half = cos.shape[-1]
    c, w = cos[:, None, :], sin[:, None, :]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * w, hi * c + lo * w], dim=-1)


def _put(s, name, x, page, slot):
    """Rows x of the new tokens into the pages of one pool, in place."""
    pool, kv = s[name], s["kv"]
    if kv == "bf16":
        pool[page, :, slot] = x.to(torch.bfloat16)
        return
    touched, where = torch.unique(page, return_inverse=True)
    index = where[:, None].expand(-1, x.shape[1])
    amax = torch.zeros((len(touched), x.shape[1]), device=x.device).scatter_reduce(0, index, x.abs().amax(dim=2), "amax")
    begins = torch.full((len(touched),), PAGE, device=x.device).scatter_reduce(0, where, slot, "amin")
    need = (amax / torch.full((), QMAX[kv], device=x.device)).clamp_min(TINY)
    old = s[name + "_scale"][touched]
    _recode(s, name, touched, begins, old, torch.where((begins == 0)[:, None], need, torch.maximum(old, need)))
    pool.view(torch.uint8)[page, :, slot] = _encode(x / s[name + "_scale"][page][:, :, None], kv).view(torch.uint8)


def _recode(s, name, touched, begins, old, scale_new):
    """New scales for pages, and the codes of their first `begins` slots once more where a scale grew."""
    kv, pool = s["kv"], s[name]
    before = pool.view(torch.float8_e4m3fn if kv == "fp8" else torch.int8)[touched]
    again = _encode(before.float() * old[:, :, None, None] / scale_new[:, :, None, None], kv)
    kept = torch.arange(PAGE, device=old.device)[None, :] < begins[:, None]
    grown = (kept[:, None, :] & (scale_new > old)[:, :, None])[..., None]
    pool.view(torch.uint8)[touched] = torch.where(grown, again.view(torch.uint8), before.view(torch.uint8))
    s[name + "_scale"][touched] = scale_new


def _plain_write(s):
    b, i = _flat(s)
    pos = s["ctx"].long()[b] - s["new"].long()[b] + i
    page, slot = s["table"].long()[b, pos // PAGE], pos % PAGE
    half = s["cos_sin"].shape[1] // 2
    row = s["cos_sin"][pos if s["positions"] is None else s["positions"].long()]
    cos, sin = row[:, :half], row[:, half:]
    _put(s, "k", _rotated(_normed(s["k_new"], s["k_weight"]), cos, sin), page, slot)
    _put(s, "v", s["v_new"].float(), page, slot)
    return _rotated(_normed(s["q"], s["q_weight"]), cos, sin).to(torch.bfloat16)


def _plain_accept(s):
    b, i = _flat(s)
    kept = i < s["lens"].long()[b]
    b, i, node = b[kept], i[kept], s["rows"].long()[kept]
    start = s["ctx"].long()[b] - s["new"].long()[b]
    src, dst = start + node, start + i
    from_page, from_slot = s["table"].long()[b, src // PAGE], src % PAGE
    page, slot = s["table"].long()[b, dst // PAGE], dst % PAGE
    for name in ("k", "v"):
        pool, kv = s[name], s["kv"]
        if kv == "bf16":
            pool[page, :, slot] = pool[from_page, :, from_slot]
            continue
        scales = s[name + "_scale"]
        x = pool.view(torch.float8_e4m3fn if kv == "fp8" else torch.int8)[from_page, :, from_slot].float() * scales[from_page][:, :, None]
        touched, where = torch.unique(page, return_inverse=True)
        index = where[:, None].expand(-1, x.shape[1])
        comes = torch.where((page != from_page)[:, None], x.abs().amax(dim=2), torch.zeros((), device=x.device))
        amax = torch.zeros((len(touched), x.shape[1]), device=x.device).scatter_reduce(0, index, comes, "amax")
        begins = torch.full((len(touched),), PAGE, device=x.device).scatter_reduce(0, where, slot, "amin")
        old = scales[touched]
        _recode(s, name, touched, begins, old, torch.maximum(old, amax / torch.full((), QMAX[kv], device=x.device)))
        pool.view(torch.uint8)[page, :, slot] = _encode(x / scales[page][:, :, None], kv).view(torch.uint8)


def _context(s, name):
    """Keys or values of every trajectory, padded, in 32 bits: [B, Hkv, tokens, D]."""
    pool = s[name].view(torch.float8_e4m3fn) if s["kv"] == "fp8" else s[name]
    at = s["table"].long().clamp_min(0)
    x = pool[at].float()
    if s["k_scale"] is not None:
        x.mul_(s[name + "_scale"][at][..., None, None])                         # [B, pages, Hkv, 16, D]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_tree(s):
    total, hq, d = s["q"].shape
    n_b, hkv, most = len(s["ctx"]), s["k"].shape[1], s["max_q"]
    b, i = _flat(s)
    prefix = (s["ctx"] - s["new"]).long()
    q = torch.zeros((n_b, most, hq, d), device=b.device)
    q[b, i] = s["q"].float()
    q = q.view(n_b, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_b, hkv, -1, d)
    k = _context(s, "k")
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(n_b, hkv, hq // hkv, most, -1)
    del k
    rel = torch.arange(x.shape[-1], device=b.device)[None, :] - prefix[:, None]                   # [B, tokens]
    masks = torch.zeros((n_b, most, s["words"]), dtype=torch.int64, device=b.device)
    masks[b, i] = s["mask"]
    word = (rel.clamp(0, 64 * s["words"] - 1) // 64)[:, None, :].expand(-1, most, -1)
    drafted = (torch.gather(masks, 2, word) >> (rel.clamp_min(0) % 64)[:, None, :]) & 1
    seen = (rel < 0)[:, None, :] | ((rel >= 0) & (rel < s["new"].long()[:, None]))[:, None, :] & (drafted > 0)
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    p = x.sub_(top.masked_fill(top == float("-inf"), 0.0)).exp_()
    sums = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(n_b, hkv, -1, p.shape[-1]), _context(s, "v")).view(n_b, hkv, hq // hkv, most, d)
    o = (o / sums.masked_fill(sums == 0, 1.0)).permute(0, 3, 1, 2, 4).reshape(n_b, most, hq, d)
    return o[b, i].to(torch.bfloat16)


def _pools(s, **more):
    """The pools as the values that they hold, and the scales."""
    out = {name: s[name].view(torch.float8_e4m3fn) if s["kv"] == "fp8" else s[name] for name in ("k", "v")}
    return dict(out, **more) if s["k_scale"] is None else dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"], **more)


def _run_own(s):
    from paper_2512_22560_amd import binding as B

    chunk = (s["new"], s["off"])
    if s["kind"] == "draft":
        if "mask" not in s:                        # a program keeps its outputs and workspace from step to step
            s["mask"] = torch.empty((len(s["parents"]), s["words"]), dtype=torch.int64, device=s["parents"].device)
            s["positions"] = torch.empty_like(s["parents"])
        B.attn_tree_mask(s["parents"], *chunk, s["ctx"], max_q_len=s["max_q"], tree_mask=s["mask"], positions=s["positions"])
        return {"mask": s["mask"], "positions": s["positions"]}
    pools, where, scales = (s["k"], s["v"]), (s["table"], s["ctx"]), {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if s["kind"] == "write":
        s["q_out"] = B.kv_write_norm_rope(s["q"], s["k_new"], s["v_new"], *chunk, *pools, *where, q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                          cos_sin=s["cos_sin"], max_q_len=s["max_q"], positions=s["positions"], q_out=s.get("q_out"), **scales)
        return _pools(s, q=s["q_out"])
    if s["kind"] == "accept":
        B.kv_accept(s["rows"], s["lens"], *chunk, *pools, *where, max_q_len=s["max_q"], **scales)
        return _pools(s)
    if "workspace" not in s:
        s["workspace"] = B.alloc_tree_workspace(s["q"], *pools, *where, max_q_len=s["max_q"], **scales)
        s["out"] = torch.empty_like(s["q"])
    return B.attn_tree(s["q"], *chunk, s["mask"], *pools, *where, sm_scale=s["scale"], max_q_len=s["max_q"], out=s["out"], workspace=s["workspace"], **scales)


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "draft":
        return _plain_draft(s)
    if s["kind"] == "write":
        return _pools(s, q=_plain_write(s))
    if s["kind"] == "accept":
        _plain_accept(s)
        return _pools(s)
    return _plain_tree(s)


def work(case):
    ctx, new = _lengths(case)
    hq, hkv, d, item, t = case["q_heads"], case["kv_heads"], case["head_dim"], ITEM[case["kv"]], int(new.sum())
    if case["kind"] == "draft":
        words = (int(new.max()) + 63) // 64
        return {"bytes": t * (4 + 8 * words + 4) + 12 * len(new), "flops": 0}
    scale = 0 if case["kv"] == "bf16" else 8 * hkv                # K's and V's scales of a page
    pages = (ctx + PAGE - 1) // PAGE
    if case["kind"] == "accept":
        rows, lens = _accepted(case, new)
        first = np.concatenate([[0], np.cumsum(new)])[:-1]
        moved = sum(int((rows[f:f + m] != np.arange(m)).sum()) for f, m in zip(first.tolist(), lens.tolist()))
        touched = int(((ctx - new + lens + PAGE - 1) // PAGE - (ctx - new) // PAGE).sum())
        return {"bytes": moved * 4 * hkv * d * item + touched * (4 + 2 * scale) + 4 * int(lens.sum()) + 16 * len(new), "flops": 0}
    if case["kind"] == "write":
        touched = int((pages - (ctx - new) // PAGE).sum())
        at = np.repeat(ctx - new, new)
        at = np.unique(at + (_depths(new, _parents(new, case["lengths"] + 1)) if case["tree"] else np.concatenate([np.arange(n) for n in new.tolist()])))
        n = t * (2 * hq * d * 2 + 2 * hkv * d * (2 + item)) + touched * (4 + 2 * scale) + len(at) * d * 4 + 8 * d
        return {"bytes": n + (4 * t if case["tree"] else 0), "flops": 7 * t * d * (hq + hkv)}
    depth = _depths(new, _parents(new, case["lengths"] + 1))
    pairs = int((new * (ctx - new)).sum() + (depth + 1).sum())
    words = (int(new.max()) + 63) // 64
    return {"bytes": int(ctx.sum()) * 2 * hkv * d * item + int(pages.sum()) * (4 + scale) + 4 * t * hq * d + 8 * words * t, "flops": 4 * hq * d * pairs}


# What run() returns, from the definition, one trajectory (or one page) after the other in 64 bits.

def _e4m3(x):
    """The nearest value of E4M3 (three bits behind the point, least exponent -6), ties to even, at most 448."""
    exponent = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp(-6, 8)
    step = torch.exp2(exponent - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _int8(x):
    return torch.round(x).clamp(-127, 127)


def _held(s, name):
    return s[name].view(torch.float8_e4m3fn).double() if s["kv"] == "fp8" else s[name].double()


def _exact_pages(case, s, rows_of):
    """Pools and scales after rows_of(name) = [(trajectory, first position, rows [n, Hkv, D], which of them come from elsewhere)] went in."""
    kv, table, out = case["kv"], s["table"].cpu().numpy(), {}
    grid = _e4m3 if kv == "fp8" else _int8
    for name in ("k", "v"):
        held, scale = _held(s, name), None if kv == "bf16" else s[name + "_scale"].double()
        for b, at, rows, comes in rows_of(name):
            lo, end, fresh = at, at + len(rows), case["kind"] == "write"
            while lo < end:
                page, s0, k = int(table[b, lo // PAGE]), lo % PAGE, min(end - lo, PAGE - lo % PAGE)
                x = rows[lo - at:lo - at + k].transpose(0, 1)                   # [Hkv, k, D]
                if kv != "bf16":
                    need = (x * comes[lo - at:lo - at + k][None, :, None]).abs().amax(dim=(1, 2)) / QMAX[kv]
                    need = need.clamp_min(TINY) if fresh and s0 == 0 else torch.maximum(need, scale[page])
                    changed = (need > scale[page])[:, None, None]
                    held[page, :, :s0] = torch.where(changed, grid(held[page, :, :s0] * (scale[page] / need)[:, None, None]), held[page, :, :s0])
                    x, scale[page] = grid(x / need[:, None, None]), need
                held[page, :, s0:s0 + k] = x
                lo += k
        out[name] = held if kv != "int8" else None           # (whole numbers: no value to be near to)
        if kv != "bf16":
            out[name + "_scale"] = scale
    return out


def _exact_write(case, s):
    ctx, new = _lengths(case)
    d = case["head_dim"]
    at = np.concatenate([np.arange(l - n, l) for l, n in zip(ctx.tolist(), new.tolist())])
    where = torch.from_numpy(at).to(s["q"].device) if s["positions"] is None else s["positions"].long()
    cos, sin = (s["cos_sin"].double()[where][:, None, h * d // 2:(h + 1) * d // 2] for h in (0, 1))

    def made(x, weight):
        x = x.double()
        x = x / torch.sqrt((x ** 2).mean(dim=-1, keepdim=True) + EPS) * weight.double()
        return torch.cat([x[..., :d // 2] * cos - x[..., d // 2:] * sin, x[..., d // 2:] * cos + x[..., :d // 2] * sin], dim=-1)

    new_rows = {"k": made(s["k_new"], s["k_weight"]), "v": s["v_new"].double()}

    def rows_of(name):
        first = np.concatenate([[0], np.cumsum(new)]).tolist()
        for b, (l, n) in enumerate(zip(ctx.tolist(), new.tolist())):
            yield b, l - n, new_rows[name][first[b]:first[b] + n], torch.ones(n, dtype=torch.float64, device=where.device)

    return dict(_exact_pages(case, s, rows_of), q=made(s["q"], s["q_weight"]))


def _exact_accept(case, s):
    ctx, new = _lengths(case)
    nodes, lens = _accepted(case, new)
    table = s["table"].long()

    def rows_of(name):
        held, first, moves = _held(s, name), 0, []
        for b, (l, n, m) in enumerate(zip(ctx.tolist(), new.tolist(), lens.tolist())):
            src = torch.from_numpy(nodes[first:first + m]).to(table.device) + (l - n)
            page = table[b, src // PAGE]
            x = held[page, :, src % PAGE]
            if case["kv"] != "bf16":
                x = x * s[name + "_scale"].double()[page][:, :, None]
            dst = torch.arange(l - n, l - n + m, device=table.device)
            moves.append((b, l - n, x, (src // PAGE != dst // PAGE).double()))
            first += n
        return moves

    return _exact_pages(case, s, rows_of)


def _exact_tree(case, s):
    ctx, new = _lengths(case)
    parents = _parents(new, case["lengths"] + 1)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    out, row = torch.zeros((int(new.sum()), hq, d), dtype=torch.float64, device=s["q"].device), 0
    for b, (l, n) in enumerate(zip(ctx.tolist(), new.tolist())):
        pages = s["table"][b, :(l + PAGE - 1) // PAGE].long()
        both = []
        for name in ("k", "v"):
            x = _held({"kv": s["kv"], name: s[name][pages]}, name)
            x = x if case["kv"] == "bf16" else x * s[name + "_scale"][pages].double()[..., None, None]
            both.append(x.transpose(0, 1).reshape(hkv, -1, d)[:, :l])
        seen = np.zeros((n, l), dtype=bool)
        seen[:, :l - n] = True
        for i in range(n):
            j = i
            while j >= 0:
                seen[i, l - n + j] = True
                j = int(parents[row + j])
        hidden = torch.from_numpy(~seen).to(out.device)
        q = s["q"][row:row + n].double()
        for h in range(hq):
            x = (q[:, h] @ both[0][h // (hq // hkv)].T.contiguous() / math.sqrt(d)).masked_fill(hidden, float("-inf"))
            out[row:row + n, h] = torch.softmax(x, dim=1) @ both[1][h // (hq // hkv)]
        row += n
    return out


def exact(case, seed):
    ctx, new = _lengths(case)
    if case["kind"] == "draft" or (case["kind"] != "tree" and int((new // PAGE + 2).sum()) > 12000):
        return None                                # (whole numbers; page after page it would take too long)
    s = prepare(case, seed)
    return {"write": _exact_write, "accept": _exact_accept, "tree": _exact_tree}[case["kind"]](case, s)

"""The operators of a rotated, 8-bit paged KV cache as callable cases: the write that fills it and the attention that reads it.

A trajectory's keys are rotated to their positions, scaled to 8 bits for each page of 16 tokens and KV head, written into
the pages, and read by decode and append attention.  Every case is one call of one operator with the buffers an engine
keeps (pools, tables, scales) made beforehand.  Lengths belong to the case (drawn from its `lengths` seed), values and the
physical placement of the pages to the seed that `prepare` is given.  Head shapes, batch sizes and lengths are those of the
workloads that the repository states, and smaller ones of the same kind.

Kinds of case:
  write    kv_write_rope: q, k and v of the new tokens, as one projection leaves them side by side, are rotated; q is
           handed back, k and v go into the pages
  decode   attn_decode over a cache in 8 bits with a scale for each page and KV head
  append   attn_append over such a cache: a chunk per trajectory behind its cached prefix

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


def _case(kind, batch, heads, kv, prefix, new=(1, 1), lengths=0, name=None, rot=0, axes=1, adjacent=False):
    """prefix, new: least and most cached and new tokens of a trajectory; rot: rotated dims of a head; axes: of the positions."""
    c = {"kind": kind, "batch": batch, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "kv": kv,
         "prefix_lo": prefix[0], "prefix_hi": prefix[1], "new_lo": new[0], "new_hi": new[1], "lengths": lengths,
         "rot": rot, "axes": axes, "adjacent": adjacent}
    return c if name is None else dict(c, name=name)


def listed():
    a, b, tiny = (32, 8, 128), (64, 4, 128), (8, 2, 64)
    return [
        # the tail of a rollout: a handful of trajectories, one token each; launches and latency
        _case("write", 5, a, "bf16", (7, 64), lengths=1, rot=128, name="write_bf16_few"),
        # one token per trajectory of a whole batch, into int8 pages that are partly filled
        _case("write", 512, b, "int8", (0, 63), lengths=2, rot=128, name="write_int8_tokens_b512"),
        # observations with images: positions in time, height and width, E4M3 pages
        _case("write", 128, b, "fp8", (0, 40), new=(32, 512), lengths=3, rot=128, axes=3, name="write_fp8_axes_b128"),
        # observations of a whole batch, half of each head rotated in adjacent pairs, int8 pages: the largest write
        _case("write", 64, a, "int8", (0, 40), new=(64, 1024), lengths=4, rot=64, adjacent=True, name="write_int8_chunks_b64"),
        # the last few long trajectories still generate
        _case("decode", 3, a, "int8", (2048, 32767), lengths=5, name="decode_int8_few"),
        # short histories with small heads, some of them not begun yet
        _case("decode", 37, tiny, "fp8", (-1, 300), lengths=6, name="decode_fp8_short_d64"),
        # an ordinary decode step
        _case("decode", 64, a, "int8", (512, 8191), lengths=7, name="decode_int8_b64"),
        # a large decode step, many query heads to a KV head: the most bytes
        _case("decode", 256, b, "int8", (1024, 32767), lengths=8, name="decode_int8_b256"),
        # environments answer one by one: three observations
        _case("append", 3, a, "int8", (2048, 16384), new=(16, 512), lengths=9, name="append_int8_few"),
        # terse observations of a medium batch
        _case("append", 33, b, "fp8", (256, 8192), new=(3, 96), lengths=10, name="append_fp8_short"),
        # observations behind long prefixes: the most operations
        _case("append", 24, a, "int8", (2048, 8192), new=(64, 512), lengths=11, name="append_int8_b24"),
        # after a weight update histories are prefilled again
        _case("append", 12, a, "fp8", (0, 0), new=(512, 4096), lengths=12, name="append_fp8_again"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; none has more bytes or operations than the largest listed ones."""
    while True:
        kind = rng.choice(["write", "decode", "append"])
        heads = rng.choice([(32, 8, 128), (64, 4, 128), (64, 8, 128), (8, 2, 64)])
        kv = rng.choice(["int8", "fp8"])
        batch = _log_int(rng, 1, 512)
        seed = rng.randrange(1 << 30)
        if kind == "write":
            lo, hi = sorted((_log_int(rng, 1, 1024), _log_int(rng, 1, 1024)))
            if rng.random() < 0.4:
                lo = hi = 1
            c = _case(kind, batch, heads, rng.choice([kv, kv, "bf16"]), (0, rng.randrange(8, 64)), (lo, hi), seed,
                      rot=heads[2] // rng.choice([1, 1, 2]), axes=rng.choice([1, 1, 3]), adjacent=rng.random() < 0.3)
        elif kind == "decode":
            lo, hi = sorted((_log_int(rng, 1, 32768), _log_int(rng, 1, 32768)))
            c = _case(kind, batch, heads, kv, (lo - 1, hi - 1), (1, 1), seed)
        else:
            lo, hi = sorted((_log_int(rng, 2, 1024), _log_int(rng, 2, 1024)))
            p, q = sorted((_log_int(rng, 64, 16384), _log_int(rng, 64, 16384)))
            if rng.random() < 0.25:
                p, q, lo, hi = 0, 0, lo, 4 * hi
            c = _case(kind, batch, heads, kv, (p, q), (lo, hi), seed)
        w = work(c)
        ctx, new = _lengths(c)
        padded = len(ctx) * int(ctx.max())
        if (w["bytes"] <= 2.4e9 and w["flops"] <= 6e11 and padded * heads[1] * heads[2] <= 4.4e9 and
                (kind == "write" or padded * heads[0] * int(new.max()) <= 6.5e9)):
            return c


def _lengths(c):
    """Tokens in the cache, the new ones among them, and new tokens, of every trajectory."""
    rng = np.random.default_rng(c["lengths"])
    n = c["batch"]
    new = np.exp(rng.uniform(math.log(c["new_lo"]), math.log(c["new_hi"] + 1), n)).astype(np.int64).clip(c["new_lo"], c["new_hi"])
    if c["kind"] == "write" or c["prefix_hi"] - c["prefix_lo"] < 1000:
        prefix = rng.integers(c["prefix_lo"], c["prefix_hi"] + 1, n)
    else:                                         # long histories: many short ones, few long ones
        lo, hi = c["prefix_lo"] + 1, c["prefix_hi"] + 1
        prefix = np.exp(rng.uniform(math.log(lo), math.log(hi), n)).astype(np.int64).clip(lo, hi) - 1
    return prefix + new, new


def _pair_axes(c):
    """Which axis of the positions turns each pair of a head's rotated dims: time first, then height, then width."""
    pairs = c["rot"] // 2
    side = pairs * 3 // 8
    return [0] * pairs if c["axes"] == 1 else [0] * (pairs - 2 * side) + [1] * side + [2] * side


def _positions(c, gen, dev, ctx, new):
    """Of every new token on every axis: text counts along, an image stands still in time and counts rows and columns."""
    at = np.concatenate([np.arange(l - n, l) for l, n in zip(ctx.tolist(), new.tolist())])
    at = torch.from_numpy(at.astype(np.int32)).to(dev)
    start = at - at % 64
    image = torch.randint(0, 2, (1024,), generator=gen, device=dev, dtype=torch.int32)[(start // 64) % 1024]
    return torch.stack([torch.where(image > 0, x, at) for x in (start, start + (at - start) // 8, start + (at - start) % 8)]).to(torch.int32)


def _quantised(x, kv):
    """Pages as codes and a scale for each page and head."""
    scale = (x.abs().amax(dim=(2, 3)) / torch.full((), QMAX[kv], device=x.device)).clamp_min(TINY)
    return _encode(x / scale[:, :, None, None], kv), scale


def _encode(x, kv):
    if kv == "int8":
        return x.round().clamp(-127, 127).to(torch.int8)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    ctx, new = _lengths(case)
    hq, hkv, d, kv = case["q_heads"], case["kv_heads"], case["head_dim"], case["kv"]
    pages = (ctx + PAGE - 1) // PAGE
    used = int(pages.sum())
    place = torch.randperm(used, generator=gen, device=dev).to(torch.int32)
    table = np.full((len(ctx), max(1, int(pages.max()))), -1, dtype=np.int64)
    first = np.concatenate([[0], np.cumsum(pages)])
    for b, n in enumerate(pages.tolist()):
        table[b, :n] = np.arange(first[b], first[b] + n)
    logical = torch.from_numpy(table).to(dev)

    def ints(x):
        return torch.from_numpy(np.asarray(x).astype(np.int32)).to(dev)

    total = int(new.sum())
    s = {"kind": case["kind"], "kv": kv, "max_q": int(new.max()), "scale": 1.0 / math.sqrt(d), "k_scale": None, "v_scale": None,
         "table": torch.where(logical >= 0, place[logical.clamp_min(0)], -1).to(torch.int32).contiguous(),
         "ctx": ints(ctx), "new": ints(new), "off": ints(np.concatenate([[0], np.cumsum(new)]))}

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
    if case["kind"] != "write":
        s["q"] = torch.randn((total, hq, d), generator=gen, device=dev).to(torch.bfloat16)
        return s
    # what the projection leaves: q, k and v of a token side by side
    rows = torch.cat([values(total, h, loud) for h, loud in ((hq, 0.1), (hkv, 0.3), (hkv, 0.1))], dim=1).to(torch.bfloat16)
    s["q"], s["k_new"], s["v_new"] = rows.split([hq, hkv, hkv], dim=1)
    most = int(ctx.max()) + 64
    half = case["rot"] // 2
    angle = torch.arange(most, device=dev, dtype=torch.float64)[:, None] * BASE ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32)
    s["positions"] = _positions(case, gen, dev, ctx, new) if case["axes"] > 1 else None
    s["pair_axes"] = _pair_axes(case) if case["axes"] > 1 else None
    s["adjacent"] = case["adjacent"]
    return s


def _flat(s):
    """Trajectory and position of every new token."""
    b = torch.repeat_interleave(torch.arange(len(s["new"]), device=s["new"].device), s["new"].long(), output_size=s["q"].shape[0])
    i = torch.arange(s["q"].shape[0], device=b.device) - s["off"].long()[b]
    return b, s["ctx"].long()[b] - s["new"].long()[b] + i


def _rotated(x, cos, sin, adjacent):
    x = x.float()
    r = 2 * cos.shape[-1]
    c, w = cos[:, None, :], sin[:, None, :]
    lo, hi = (x[..., 0:r:2], x[..., 1:r:2]) if adjacent else (x[..., :r // 2], x[..., r // 2:r])
    lo, hi = lo * c - hi * w, hi * c + lo * w
    turned = torch.stack([lo, hi], dim=-1).flatten(-2) if adjacent else torch.cat([lo, hi], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _put(s, name, x, page, slot):
    """Rows x of the new tokens into the pages of one pool, in place."""
    pool, kv = s[name], s["kv"]
    if kv == "bf16":
        pool[page, :, slot] = x.to(torch.bfloat16)
        return
    codes, scale = (pool.view(torch.float8_e4m3fn) if kv == "fp8" else pool), s[name + "_scale"]
    touched, where = torch.unique(page, return_inverse=True)
    index = where[:, None].expand(-1, x.shape[1])
    amax = torch.zeros((len(touched), x.shape[1]), device=x.device).scatter_reduce(0, index, x.abs().amax(dim=2), "amax")
    begins = torch.full((len(touched),), PAGE, device=x.device).scatter_reduce(0, where, slot, "amin")
    need = (amax / torch.full((), QMAX[kv], device=x.device)).clamp_min(TINY)
    old = scale[touched]
    scale_new = torch.where((begins == 0)[:, None], need, torch.maximum(old, need))
    before = codes[touched]
    again = _encode(before.float() * old[:, :, None, None] / scale_new[:, :, None, None], kv)
    kept = torch.arange(PAGE, device=x.device)[None, :] < begins[:, None]
    grown = (kept[:, None, :] & (scale_new > old)[:, :, None])[..., None]
    raw = torch.where(grown, again.view(torch.uint8), before.view(torch.uint8))
    pool.view(torch.uint8)[touched] = raw
    pool.view(torch.uint8)[page, :, slot] = _encode(x / scale_new[where][:, :, None], kv).view(torch.uint8)
    scale[touched] = scale_new


def _plain_write(s):
    b, pos = _flat(s)
    page, slot = s["table"].long()[b, pos // PAGE], pos % PAGE
    half = s["cos_sin"].shape[1] // 2
    if s["positions"] is None:
        cos, sin = s["cos_sin"][pos, :half], s["cos_sin"][pos, half:]
    else:
        axis = torch.tensor(s["pair_axes"], device=pos.device)
        row = s["positions"].long()[axis].T                                    # [tokens, pairs]
        pair = torch.arange(half, device=pos.device)
        cos, sin = s["cos_sin"][row, pair], s["cos_sin"][row, pair + half]
    _put(s, "k", _rotated(s["k_new"], cos, sin, s["adjacent"]), page, slot)
    _put(s, "v", s["v_new"].float(), page, slot)
    return _rotated(s["q"], cos, sin, s["adjacent"]).to(torch.bfloat16)


def _context(s, name):
    """Keys or values of every trajectory, padded, in 32 bits: [B, Hkv, tokens, D]."""
    pool = s[name].view(torch.float8_e4m3fn) if s["kv"] == "fp8" else s[name]
    at = s["table"].long().clamp_min(0)
    x = pool[at].float().mul_(s[name + "_scale"][at][..., None, None])          # [B, pages, Hkv, 16, D]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attention(s):
    total, hq, d = s["q"].shape
    n_b, hkv, most = len(s["ctx"]), s["k"].shape[1], s["max_q"]
    b, pos = _flat(s)
    i = pos - (s["ctx"].long() - s["new"].long())[b]
    q = torch.zeros((n_b, most, hq, d), device=b.device)
    q[b, i] = s["q"].float()
    q = q.view(n_b, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_b, hkv, -1, d)
    k = _context(s, "k")
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(n_b, hkv, hq // hkv, most, -1)
    del k
    last = (s["ctx"].long() - s["new"].long())[:, None] + torch.arange(most, device=b.device)[None, :]
    hidden = torch.arange(x.shape[-1], device=b.device)[None, None, :] > torch.minimum(last, s["ctx"].long()[:, None] - 1)[:, :, None]
    x.masked_fill_(hidden[:, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    p = x.sub_(top.masked_fill(top == float("-inf"), 0.0)).exp_()
    sums = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(n_b, hkv, -1, p.shape[-1]), _context(s, "v")).view(n_b, hkv, hq // hkv, most, d)
    o = (o / sums.masked_fill(sums == 0, 1.0)).permute(0, 3, 1, 2, 4).reshape(n_b, most, hq, d)
    return o[b, i].to(torch.bfloat16)


def _pools(s, q):
    """A write's outputs: the rotated queries, the pools as the values that they hold, the scales."""
    out = {"q": q, "k": s["k"].view(torch.float8_e4m3fn) if s["kv"] == "fp8" else s["k"], "v": s["v"].view(torch.float8_e4m3fn) if s["kv"] == "fp8" else s["v"]}
    return out if s["k_scale"] is None else dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"])


def _run_own(s):
    from paper_2512_22560_amd import binding as B

    pools, where, scales = (s["k"], s["v"]), (s["table"], s["ctx"]), {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if s["kind"] == "write":
        s["q_out"] = B.kv_write_rope(s["q"], s["k_new"], s["v_new"], s["new"], s["off"], *pools, *where, cos_sin=s["cos_sin"],
                                     max_q_len=s["max_q"], positions=s["positions"], pair_axes=s["pair_axes"], interleaved=s["adjacent"],
                                     q_out=s.get("q_out"), **scales)
        return _pools(s, s["q_out"])
    if "workspace" not in s:                       # a program keeps its workspace and output from step to step
        s["workspace"] = B.alloc_workspace(B.make_desc(s["q"], s["k"], s["table"], sm_scale=s["scale"], **scales), s["q"].shape[0], s["q"].device)
        s["out"] = torch.empty_like(s["q"])
    kept = {"sm_scale": s["scale"], "out": s["out"], "workspace": s["workspace"], **scales}
    if s["kind"] == "decode":
        return B.attn_decode(s["q"], *pools, *where, **kept)
    return B.attn_append(s["q"], s["new"], s["off"], *pools, *where, max_q_len=s["max_q"], **kept)


def run(s):
    if own:
        return _run_own(s)
    return _pools(s, _plain_write(s)) if s["kind"] == "write" else _plain_attention(s)


def work(case):
    ctx, new = _lengths(case)
    hq, hkv, d, item, t = case["q_heads"], case["kv_heads"], case["head_dim"], ITEM[case["kv"]], int(new.sum())
    scale = 0 if case["kv"] == "bf16" else 8 * hkv                # K's and V's scales of a page
    pages = (ctx + PAGE - 1) // PAGE
    if case["kind"] == "write":
        touched = int((pages - (ctx - new) // PAGE)[new > 0].sum())
        at = np.unique(np.concatenate([np.arange(l - n, l) for l, n in zip(ctx.tolist(), new.tolist())]))
        n = t * (2 * hq * d * 2 + 2 * hkv * d * (2 + item)) + touched * (4 + 2 * scale) + len(at) * case["rot"] * 4
        return {"bytes": n + (4 * case["axes"] * t if case["axes"] > 1 else 0), "flops": 3 * t * case["rot"] * (hq + hkv)}
    pairs = int((new * (ctx - new) + new * (new + 1) // 2).sum())
    return {"bytes": int(ctx.sum()) * 2 * hkv * d * item + int(pages.sum()) * (4 + scale) + 4 * t * hq * d, "flops": 4 * hq * d * pairs}


# What run() returns, from the definition, one trajectory (or one page) after the other in 64 bits.

def _e4m3(x):
    """The nearest value of E4M3 (three bits behind the point, least exponent -6), ties to even, at most 448."""
    exponent = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp(-6, 8)
    step = torch.exp2(exponent - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_write(case, s):
    ctx, new = _lengths(case)
    hkv, kv = case["kv_heads"], case["kv"]
    half = case["rot"] // 2
    table, dev = s["table"].cpu().numpy(), s["q"].device
    at = np.concatenate([np.arange(l - n, l) for l, n in zip(ctx.tolist(), new.tolist())])
    axes = torch.tensor(_pair_axes(case), device=dev)
    where = torch.from_numpy(at).to(dev)[None].expand(3, -1) if s["positions"] is None else s["positions"].long()
    cos, sin = torch.zeros((2, len(at), 1, half), dtype=torch.float64, device=dev)
    for j in range(half):                          # (the table is an input: its values, not its formula)
        cos[:, 0, j], sin[:, 0, j] = s["cos_sin"][where[axes[j]], j].double(), s["cos_sin"][where[axes[j]], half + j].double()
    first = torch.arange(half, device=dev) * 2 if case["adjacent"] else torch.arange(half, device=dev)
    second = first + (1 if case["adjacent"] else half)

    def turn(x):
        x = x.double()
        y = x.clone()
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        return y

    out = {"q": turn(s["q"])}
    for name, rows in (("k", turn(s["k_new"])), ("v", s["v_new"].double())):
        held = s[name].view(torch.float8_e4m3fn).double() if kv == "fp8" else s[name].double()
        scale = None if kv == "bf16" else s[name + "_scale"].double()
        row = 0
        for b, (l, n) in enumerate(zip(ctx.tolist(), new.tolist())):
            lo = l - n
            while lo < l:
                page, s0, k = int(table[b, lo // PAGE]), lo % PAGE, min(l - lo, PAGE - lo % PAGE)
                x = rows[row:row + k].transpose(0, 1)                           # [Hkv, k, D]
                if kv != "bf16":
                    need = (x.abs().amax(dim=(1, 2)) / QMAX[kv]).clamp_min(TINY)
                    grid = _e4m3 if kv == "fp8" else lambda v: torch.round(v).clamp(-127, 127)
                    if s0:
                        need = torch.maximum(need, scale[page])
                        changed = (need > scale[page])[:, None, None]
                        held[page, :, :s0] = torch.where(changed, grid(held[page, :, :s0] * (scale[page] / need)[:, None, None]), held[page, :, :s0])
                    x, scale[page] = grid(x / need[:, None, None]), need
                held[page, :, s0:s0 + k] = x
                lo, row = lo + k, row + k
        out[name] = held if kv != "int8" else None           # (whole numbers: no value to be near to)
        if kv != "bf16":
            out[name + "_scale"] = scale
    return out


def exact(case, seed):
    ctx, new = _lengths(case)
    if case["kind"] == "write" and int((ctx // PAGE + 1).sum()) > 12000:
        return None                                # (page after page it would take too long)
    s = prepare(case, seed)
    if case["kind"] == "write":
        return _exact_write(case, s)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    out, row = torch.zeros((int(new.sum()), hq, d), dtype=torch.float64, device=s["q"].device), 0
    for b, (l, n) in enumerate(zip(ctx.tolist(), new.tolist())):
        if n == 0 or l == 0:
            row += n
            continue
        pages = s["table"][b, :(l + PAGE - 1) // PAGE].long()
        both = []
        for name in ("k", "v"):
            x = s[name][pages].view(torch.float8_e4m3fn).double() if case["kv"] == "fp8" else s[name][pages].double()
            both.append((x * s[name + "_scale"][pages].double()[..., None, None]).transpose(0, 1).reshape(hkv, -1, d)[:, :l])
        q = s["q"][row:row + n].double()
        seen = torch.arange(l, device=q.device)[None, :] <= torch.arange(l - n, l, device=q.device)[:, None]
        for h in range(hq):
            x = (q[:, h] @ both[0][h // (hq // hkv)].T.contiguous() / math.sqrt(d)).masked_fill(~seen, float("-inf"))
            out[row:row + n, h] = torch.softmax(x, dim=1) @ both[1][h // (hq // hkv)]
        row += n
    return out

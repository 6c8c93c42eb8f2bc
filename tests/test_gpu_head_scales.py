"""Attention over 8-bit pools with a scale for each page and KV head, against the oracle in 64 bits on the same stored bytes.

The bound on an output element is derived from what the kernels round, and nothing else: the output once to bf16 (8 bits: 2^-8 of itself),
each weight once to f16 (2^-11 of it, so of the weighted sum of |v|), and scores and sums in float32, for which 2^-12 of that sum
is allowed: a score of 64 in log2 units is off by 64 * 2^-24 * a few.  Queries and codes are exact in f16."""
import numpy as np
import pytest
import torch

from oracle import attention as O
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.helpers import oracle_args

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KV = ["int8_head", "fp8_e4m3_head"]
SCORE_ROOM = 2.0 ** -12


def build(kv, heads, d, ctx, qlen=("const", 1), batch=7, seed=3, prefix=False, append_rows=None):
    w = W.Workload("t", batch, heads[0], heads[1], d, "bf16", kv, ctx, qlen=qlen, seed=seed, ctx_is_prefix=prefix, append_rows=append_rows)
    return W.build(w, DEV)


def lengths(b, ctx, new=None):
    """The batch with other lengths, all within the pages that its table has."""
    ctx = np.asarray(ctx)
    new = np.ones(len(ctx), dtype=np.int64) if new is None else np.asarray(new)
    b.ctx_lens_host, b.q_lens_host = ctx, new
    b.ctx_lens, b.q_lens = (torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (ctx, new))
    b.q_offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    return b


def call(b, which="decode", **kw):
    args = dict(sm_scale=b.workload.sm_scale, k_scale=b.k_scale, v_scale=b.v_scale, **kw)
    pools = (b.k_pages, b.v_pages, b.page_table, b.ctx_lens)
    if which.startswith("decode"):
        return getattr(B, "attn_" + which)(b.q, *pools, **args)
    return getattr(B, "attn_" + which)(b.q, b.q_lens, b.q_offsets, *pools, max_q_len=int(max(1, b.q_lens_host.max(initial=1))), **args)


def oracle(b, which="decode", magnitudes=False):
    a = oracle_args(b)
    if magnitudes:                                        # the weighted sum of |v|
        v = a["v_pages"]
        a["v_pages"] = np.abs(np.maximum(v, -127)) if v.dtype == np.int8 else v & 0x7F
    q = W.raw_numpy(b.q)
    return O.attn_decode(q, **a) if which == "decode" else O.attn_append(q, b.q_lens_host, **a)


def check(got, b, which="decode", extra=0.0):
    ref, room = oracle(b, which), oracle(b, which, True)
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all()
    bound = (2.0 ** -8) * np.abs(ref) + (2.0 ** -11 + SCORE_ROOM + extra) * room + 1e-30
    worst = float((np.abs(g - ref) / bound).max(initial=0.0))
    assert worst <= 1.0, f"{worst:.2f} times the bound"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", KV)
def test_decode_at_every_edge_of_a_page_and_block(kv, d):
    edges = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 2047, 2048, 2049]
    b = lengths(build(kv, (8, 2), d, ("const", 2064), batch=len(edges)), edges)
    check(call(b), b)


@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (5, 1), (16, 1), (17, 1), (40, 2), (32, 8), (64, 4), (12, 3)])
@pytest.mark.parametrize("kv", KV)
def test_decode_head_counts(kv, heads):
    b = build(kv, heads, 128 if heads[0] % 2 == 0 else 64, ("uniform", 0, 700))
    check(call(b), b)


@pytest.mark.parametrize("workers", [1, 3, 50])
@pytest.mark.parametrize("kv", KV)
def test_decode_however_rows_are_cut(kv, workers):
    b = build(kv, (16, 4), 128, ("uniform", 0, 900), batch=9, seed=5)
    B.set_decode_workers(workers)
    try:
        check(call(b), b)
    finally:
        B.set_decode_workers(0)


@pytest.mark.parametrize("kv", KV)
def test_decode_of_many_rows(kv):
    """Planned by a launch of its own, rows cut and rows whole."""
    for ctx, batch in ((("uniform", 200, 400), 150), (("loguniform", 4, 3000), 90)):
        b = build(kv, (8, 4), 64, ctx, batch=batch, seed=6)
        check(call(b), b)
        out = torch.empty_like(b.q)
        assert torch.equal(call(b, "decode_static", out=out), call(b))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", KV)
def test_append_at_every_edge_of_a_page_and_block(kv, d):
    new = [1, 2, 15, 16, 17, 31, 33, 0, 63, 64, 65, 1, 100, 7]
    ctx = [1, 2, 15, 17, 48, 31, 33, 50, 64, 128, 130, 1000, 700, 1300]
    for heads in ((8, 2), (32, 8), (64, 1)):
        b = build(kv, heads, d, ("const", 1312), qlen=("const", 35), batch=len(new), seed=8)
        b = lengths(b, ctx, new)
        b.q = b.q[: int(np.sum(new))].contiguous()
        check(call(b, "append"), b, "append")


@pytest.mark.parametrize("heads,d,qlen,ctx", [((32, 8), 128, ("uniform", 1, 30), ("uniform", 0, 600)), ((64, 4), 128, ("uniform", 1, 8), ("uniform", 1000, 3000)),
                                              ((64, 4), 64, ("uniform", 1, 8), ("uniform", 1500, 2500)), ((3, 3), 64, ("uniform", 1, 200), ("uniform", 0, 300)),
                                              ((20, 1), 128, ("uniform", 1, 50), ("uniform", 0, 400)), ((32, 8), 128, ("uniform", 100, 300), ("const", 0))])
@pytest.mark.parametrize("kv", KV)
def test_append_tiles_of_either_size(kv, heads, d, qlen, ctx):
    b = build(kv, heads, d, ctx, qlen=qlen, batch=5, seed=9, prefix=True)
    check(call(b, "append"), b, "append")


@pytest.mark.parametrize("kv", KV)
def test_append_cut_into_pieces(kv):
    """Few tiles behind long contexts; the last rows of one see the whole of it."""
    for qlen in (("const", 4), ("const", 40)):
        b = build(kv, (32, 8), 128, ("uniform", 5000, 7000), qlen=qlen, batch=2, seed=10, prefix=True)
        check(call(b, "append"), b, "append")


@pytest.mark.parametrize("kv", KV)
def test_mixed_step_and_its_parts(kv):
    b = build(kv, (16, 4), 128, ("uniform", 1, 900), qlen=("uniform", 2, 60), batch=80, seed=11, prefix=True, append_rows=20)
    out = call(b, "step")
    check(out, b, "append")
    dec, app = b.select(b.decode_rows()), b.select(b.append_rows())
    row = lambda part: torch.from_numpy(np.concatenate([np.arange(o, o + n) for o, n in
                                        zip(np.cumsum(b.q_lens_host) - b.q_lens_host, b.q_lens_host) if (n == 1) == part])).to(DEV)
    assert torch.equal(out[row(True)], call(dec)) and torch.equal(out[row(False)], call(app, "append"))


@pytest.mark.parametrize("kv", KV)
def test_shared_prompts(kv):
    b = build(kv, (16, 2), 128, ("uniform", 520, 900), batch=24, seed=12)
    b = W.alias_shared_prefix(b, 8, np.array([512, 512, 100]))
    out = call(b, "decode_shared", group_size=8, shared_lens=torch.tensor([512, 512, 96], dtype=torch.int32, device=DEV))
    # (two more roundings to bf16 of the halves' rows)
    check(out, b, extra=2.0 ** -8)


@pytest.mark.parametrize("kv", KV)
def test_denominators_and_merge(kv):
    b = build(kv, (8, 2), 128, ("uniform", 0, 500), batch=12, seed=13)
    b = lengths(b, np.where(np.arange(12) % 5 == 0, 0, b.ctx_lens_host))
    out, lse = call(b, "decode_lse")
    assert torch.equal(out, call(b))
    a = oracle_args(b)
    want = O.attn_lse(W.raw_numpy(b.q), None, a["k_pages"], a["page_table"], a["ctx_lens"], sm_scale=a["sm_scale"], q_dtype="bf16", kv_dtype=kv, k_scale=a["k_scale"])
    seen = np.isfinite(want)
    got = lse.double().cpu().numpy()
    assert np.array_equal(seen, np.isfinite(got)) and np.abs(got[seen] - want[seen]).max() < 1e-4
    # the first 8 pages and the rest, as two calls
    cut = 128
    first = np.minimum(b.ctx_lens_host, cut)
    rest = b.ctx_lens_host - first
    ints = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)
    args = dict(sm_scale=b.workload.sm_scale, k_scale=b.k_scale, v_scale=b.v_scale)
    o1, l1 = B.attn_decode_lse(b.q, b.k_pages, b.v_pages, b.page_table, ints(first), **args)
    o2, l2 = B.attn_decode_lse(b.q, b.k_pages, b.v_pages, b.page_table[:, 8:].contiguous(), ints(rest), **args)
    merged, l = B.attn_merge(o1, l1, o2, l2)
    check(merged, b, extra=2.0 ** -8)
    assert np.abs(l.double().cpu().numpy()[seen] - want[seen]).max() < 1e-4
    c = build(kv, (8, 2), 64, ("uniform", 0, 200), qlen=("uniform", 1, 60), batch=6, seed=14, prefix=True)
    out, lse = call(c, "append_lse")
    a = oracle_args(c)
    want = O.attn_lse(W.raw_numpy(c.q), c.q_lens_host, a["k_pages"], a["page_table"], a["ctx_lens"], sm_scale=a["sm_scale"], q_dtype="bf16", kv_dtype=kv, k_scale=a["k_scale"])
    assert np.abs(lse.double().cpu().numpy() - want).max() < 1e-4


@pytest.mark.parametrize("which", ["decode", "append"])
@pytest.mark.parametrize("kv", KV)
def test_a_first_token_that_takes_nearly_all_the_weight(kv, which):
    """What is left for the others, 2^-18 each, is what the output is made of where the first token's value is zero."""
    b = build(kv, (4, 2), 128, ("const", 1500), qlen=("const", 1 if which == "decode" else 30), batch=3, seed=15, prefix=which == "append")
    # keys of the first tokens along the queries' sum; the other keys small
    table, first = b.page_table.long(), int(b.page_table[0, 0])
    b.k_scale.mul_(0.05)
    for i in range(3):
        p = int(table[i, 0])
        lo = int(b.q_offsets[i])
        for g in range(2):
            q = b.q[lo, 2 * g].float()
            code = (q / q.abs().max() * (127 if kv == "int8_head" else 448)).round()
            b.k_pages[p, g, 0] = code.to(torch.int8) if kv == "int8_head" else code.to(torch.float8_e4m3fn).view(torch.uint8)
            want = 18 / 1.4427 / b.workload.sm_scale / float((q * code).sum())    # its score: 18 in log2 units
            old = float(b.k_scale[p, g])
            b.k_scale[p, g] = want
            shrunk = W.raw_numpy(b.k_pages[p, g, 1:])
            dec = O.decode_storage(shrunk, kv) * old / want
            b.k_pages[p, g, 1:] = (torch.from_numpy(dec).round().clamp(-127, 127).to(torch.int8) if kv == "int8_head" else
                                   torch.from_numpy(dec).float().to(torch.float8_e4m3fn).view(torch.uint8)).to(DEV)
        b.v_pages[p, :, 0] = 0
    if which == "append":
        b.q.copy_(b.q.view(3, 30, 4, 128)[:, :1].expand(-1, 30, -1, -1).reshape(90, 4, 128))
    check(call(b, which), b, which)


@pytest.mark.parametrize("which", ["decode", "append"])
@pytest.mark.parametrize("kv", KV)
def test_scales_and_queries_far_from_one(kv, which):
    """Loud and faint pages and heads side by side, and queries that f16 could not hold."""
    rng = np.random.default_rng(16)
    for q_mag, k_mag in ((2.0 ** 100, 2.0 ** -100), (2.0 ** -60, 2.0 ** 60), (2.0 ** 20, 2.0 ** -20)):
        b = build(kv, (8, 2), 64, ("uniform", 100, 400), qlen=("const", 1 if which == "decode" else 20), batch=4, seed=17, prefix=which == "append")
        if k_mag == 2.0 ** -100:
            k_mag, q_mag = 2.0 ** -50, 2.0 ** 50
        b.q = (b.q.float() * q_mag * torch.exp2(torch.from_numpy(rng.integers(-3, 1, (b.q.shape[0], 8, 1))).to(DEV).float())).to(torch.bfloat16)
        b.k_scale.mul_(k_mag)
        b.v_scale.mul_(torch.from_numpy(np.exp2(rng.integers(-20, 20, b.v_scale.shape)).astype(np.float32)).to(DEV))
        check(call(b, which), b, which)


@pytest.mark.parametrize("which", ["decode", "append"])
@pytest.mark.parametrize("kv", KV)
def test_queries_that_are_undefined_or_zero_concern_their_rows_alone(kv, which):
    b = build(kv, (8, 2), 128, ("uniform", 100, 400), qlen=("const", 1 if which == "decode" else 40), batch=6, seed=25, prefix=which == "append")
    bad = torch.zeros(b.q.shape[:2], dtype=torch.bool)
    bad[::3, 5] = bad[1::4, 2] = True
    b.q[1::2, 0] = 0
    clean = b.q.clone()
    for value in (float("inf"), float("nan"), -float("inf")):
        b.q = clean.clone()
        b.q[bad.to(DEV), 17] = value
        out = call(b, which)
        assert not torch.isfinite(out[bad.to(DEV)]).all(dim=-1).any()
        b.q = clean
        out[bad.to(DEV)] = call(b, which)[bad.to(DEV)]
        check(out, b, which)


@pytest.mark.parametrize("which", ["decode", "append"])
@pytest.mark.parametrize("kv", KV)
def test_pages_of_zero_values(kv, which):
    """Their scale is the least there is; next to others, and alone."""
    b = build(kv, (8, 2), 128, ("uniform", 60, 300), qlen=("const", 1 if which == "decode" else 9), batch=4, seed=18, prefix=which == "append")
    t = b.page_table.long()
    for i in range(4):
        live = t[i][t[i] >= 0]
        some = live if i == 0 else live[::2]
        b.v_scale[some] = 2.0 ** -64
        b.v_pages[some] = torch.where(b.v_pages[some] == (-128 if kv == "int8_head" else 0x7F), b.v_pages[some], torch.zeros_like(b.v_pages[some]))
    out = call(b, which)
    check(out, b, which)
    rows = int(b.q_offsets[1])
    assert (out[:rows] == 0).all()


def test_pages_that_nobody_has_are_never_looked_at():
    """Scales and codes of every page that no live token is in may be anything, page 0 among them."""
    for kv in KV:
        for which, qlen in (("decode", 1), ("append", 11)):
            b = build(kv, (8, 2), 128, ("uniform", 1, 90), qlen=("const", qlen), batch=5, seed=19, prefix=True)
            want = call(b, which)
            n = b.k_pages.shape[0]
            grown = lambda t: torch.cat([t.new_full((1, *t.shape[1:]), float("nan") if t.dtype == torch.float32 else 127), t])
            b.page_table = torch.where(b.page_table >= 0, b.page_table + 1, b.page_table).contiguous()
            b.k_pages, b.v_pages, b.k_scale, b.v_scale = (grown(t) for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
            assert b.k_pages.shape[0] == n + 1 and torch.equal(call(b, which), want)


@pytest.mark.parametrize("which", ["decode", "append"])
def test_a_pool_past_four_gigabytes(which):
    small = build("int8_head", (32, 8), 128, ("uniform", 100, 300), qlen=("const", 1 if which == "decode" else 20), batch=3, seed=20, prefix=which == "append")
    want = call(small, which)
    pages, n = 270_000, small.k_pages.shape[0]
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        t = getattr(small, name)
        big = torch.empty((pages, *t.shape[1:]), dtype=t.dtype, device=DEV)
        big[pages - n:] = t
        setattr(small, name, big)
    small.page_table = torch.where(small.page_table >= 0, small.page_table + (pages - n), small.page_table).contiguous()
    assert torch.equal(call(small, which), want)


@pytest.mark.parametrize("kv", KV)
def test_replays_of_a_captured_turn(kv):
    """Write and attention captured together; tokens change between the replays."""
    b = build(kv, (16, 4), 128, ("uniform", 20, 600), batch=70, seed=21)
    gen = torch.Generator(device=DEV).manual_seed(1)
    new = lambda h: torch.randn((70, h, 128), generator=gen, device=DEV).to(torch.bfloat16)
    k, v = new(4), new(4)
    table = torch.cat([torch.ones(700, 64), torch.zeros(700, 64)], dim=1).to(DEV)
    def turn(pools, q_out, out, ws):
        q = B.kv_write_rope(b.q, k, v, b.q_lens, b.q_offsets, pools[0], pools[1], b.page_table, b.ctx_lens, cos_sin=table, max_q_len=1,
                            k_scale=pools[2], v_scale=pools[3], q_out=q_out)
        return B.attn_decode(q, pools[0], pools[1], b.page_table, b.ctx_lens, sm_scale=0.1, k_scale=pools[2], v_scale=pools[3], out=out, workspace=ws)
    pools = [t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    desc = B.make_desc(b.q, pools[0], b.page_table, sm_scale=0.1, k_scale=pools[2], v_scale=pools[3])
    ws, q_out, out = B.alloc_workspace(desc, 70, DEV), torch.empty_like(b.q), torch.empty_like(b.q)
    turn([t.clone() for t in pools], torch.empty_like(q_out), torch.empty_like(out), ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn(pools, q_out, out, ws)
    for _ in range(3):
        for t, h in ((b.q, 16), (k, 4), (v, 4)):
            t.copy_(new(h))
        eager = [t.clone() for t in pools]
        want = turn(eager, torch.empty_like(q_out), torch.empty_like(out), B.alloc_workspace(desc, 70, DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(pools, eager))


@pytest.mark.parametrize("kv", KV)
def test_a_long_context(kv):
    b = build(kv, (8, 1), 128, ("const", 60_001), batch=1, seed=22)
    check(call(b), b)
    c = build(kv, (8, 1), 128, ("const", 30_000), qlen=("const", 33), batch=1, seed=23, prefix=True)
    check(call(c, "append"), c, "append")


def test_gather_of_int8_pages():
    b = build("int8_head", (8, 2), 64, ("uniform", 1, 100), batch=3, seed=24)
    for i, n in enumerate(b.ctx_lens_host.tolist()):
        got = B.debug_gather(b.v_pages, b.page_table, b.ctx_lens, i, 1, n)
        assert np.array_equal(W.raw_numpy(got), O.gather_tokens(W.raw_numpy(b.v_pages), W.raw_numpy(b.page_table), i, 1, n, "int8_head", raw=True))


SHORT = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 161, 255, 256, 257, 479, 480, 481, 511, 512]


@pytest.mark.parametrize("heads,d", [((8, 2), 64), ((8, 2), 128), ((16, 1), 128), ((5, 1), 64), ((40, 2), 128), ((17, 1), 64)])
@pytest.mark.parametrize("kv", KV)
def test_rows_that_one_workgroup_takes(kv, heads, d):
    """Tables of 32 pages, few rows: every length around the ends of pages, blocks and the waves' shares; one launch, no plan."""
    b = lengths(build(kv, heads, d, ("const", 512), batch=len(SHORT), seed=21), SHORT)
    assert b.page_table.shape[1] == 32
    desc = B.make_desc(b.q, b.k_pages, b.page_table, sm_scale=1.0, k_scale=b.k_scale, v_scale=b.v_scale)
    ws = B.alloc_workspace(desc, len(SHORT), DEV).fill_(255)
    out, lse = call(b, "decode_lse", workspace=ws)
    check(out, b)
    assert B.read_plan(desc, ws)[1] == 0
    a = oracle_args(b)
    want = O.attn_lse(W.raw_numpy(b.q), None, a["k_pages"], a["page_table"], a["ctx_lens"], sm_scale=a["sm_scale"], q_dtype="bf16", kv_dtype=kv, k_scale=a["k_scale"])
    seen, got = np.isfinite(want), lse.double().cpu().numpy()
    assert np.array_equal(seen, np.isfinite(got)) and np.abs(got[seen] - want[seen]).max() < 1e-4
    static = torch.empty_like(b.q)
    call(b, "decode_static", out=static)
    assert torch.equal(static, out) and torch.equal(call(b, workspace=ws), out)
    # what comes out depends on the row alone
    for i in (1, 9, 20, 27):
        one = B.attn_decode(b.q[i:i + 1].contiguous(), b.k_pages, b.v_pages, b.page_table[i:i + 1].contiguous(), b.ctx_lens[i:i + 1].clone(), sm_scale=b.workload.sm_scale,
                            k_scale=b.k_scale, v_scale=b.v_scale)
        assert torch.equal(one[0], out[i])


@pytest.mark.parametrize("batch", [128, 129])
@pytest.mark.parametrize("kv", KV)
def test_either_side_of_what_workgroups_take(kv, batch):
    """512 rows are a workgroup's each, 516 a wave's; 65 pages are planned for few rows, 33 for many."""
    b = build(kv, (8, 4), 64, ("uniform", 0, 500), batch=batch, seed=22)
    check(call(b), b)
    for tokens, n in ((528, batch), (1024, 7), (1040, 7)):
        c = lengths(build(kv, (8, 4), 64, ("const", tokens), batch=n, seed=23), tokens - np.arange(n) * 4)
        desc = B.make_desc(c.q, c.k_pages, c.page_table, sm_scale=1.0, k_scale=c.k_scale, v_scale=c.v_scale)
        ws = B.alloc_workspace(desc, n, DEV).fill_(255)
        check(call(c, workspace=ws), c)
        assert (B.read_plan(desc, ws)[1] > 0) == (tokens == 1040 or n == 129)


@pytest.mark.parametrize("kv", KV)
def test_a_mixed_step_of_short_contexts(kv):
    b = build(kv, (16, 4), 128, ("uniform", 1, 300), qlen=("uniform", 2, 60), batch=80, seed=24, prefix=True, append_rows=20)
    assert b.page_table.shape[1] <= 32
    out = call(b, "step")
    check(out, b, "append")
    dec, app = b.select(b.decode_rows()), b.select(b.append_rows())
    row = lambda part: torch.from_numpy(np.concatenate([np.arange(o, o + n) for o, n in
                                        zip(np.cumsum(b.q_lens_host) - b.q_lens_host, b.q_lens_host) if (n == 1) == part])).to(DEV)
    assert torch.equal(out[row(True)], call(dec)) and torch.equal(out[row(False)], call(app, "append"))


@pytest.mark.parametrize("kv", KV)
def test_undefined_queries_of_short_contexts_concern_their_rows_alone(kv):
    b = lengths(build(kv, (8, 2), 64, ("const", 300), batch=6, seed=25), [300, 40, 1, 170, 33, 290])
    clean = call(b).clone()
    b.q[1, 3, 5], b.q[3, 0, 0], b.q[5, 7, 63] = float("nan"), float("inf"), -float("inf")
    out = call(b)
    hurt = torch.zeros(6, 8, dtype=torch.bool, device=DEV)
    hurt[1, 3] = hurt[3, 0] = hurt[5, 7] = True
    assert torch.equal(out[~hurt], clean[~hurt]) and not torch.isfinite(out[hurt]).any()


@pytest.mark.parametrize("heads,d", [((8, 2), 64), ((6, 2), 128), ((34, 2), 128), ((3, 3), 64)])
@pytest.mark.parametrize("kv", KV)
def test_rows_that_one_wave_takes(kv, heads, d):
    """Tables of 32 pages, more than 512 rows; the last workgroup is not full."""
    ctx = np.random.default_rng(26).permutation(np.tile(SHORT, 10))[:271]
    b = lengths(build(kv, heads, d, ("const", 512), batch=len(ctx), seed=26), ctx)
    out, lse = call(b, "decode_lse")
    check(out, b)
    a = oracle_args(b)
    want = O.attn_lse(W.raw_numpy(b.q), None, a["k_pages"], a["page_table"], a["ctx_lens"], sm_scale=a["sm_scale"], q_dtype="bf16", kv_dtype=kv, k_scale=a["k_scale"])
    seen, got = np.isfinite(want), lse.double().cpu().numpy()
    assert np.array_equal(seen, np.isfinite(got)) and np.abs(got[seen] - want[seen]).max() < 1e-4
    assert torch.equal(call(b), out)
    order = torch.randperm(len(ctx), generator=torch.Generator().manual_seed(1)).to(DEV)       # each row depends on itself alone
    again = B.attn_decode(b.q[order].contiguous(), b.k_pages, b.v_pages, b.page_table[order].contiguous(), b.ctx_lens[order].contiguous(), sm_scale=b.workload.sm_scale,
                          k_scale=b.k_scale, v_scale=b.v_scale)
    assert torch.equal(again, out[order])


@pytest.mark.parametrize("kv", KV)
def test_a_mixed_step_of_many_short_contexts(kv):
    b = build(kv, (16, 4), 128, ("uniform", 1, 300), qlen=("uniform", 2, 20), batch=200, seed=27, prefix=True, append_rows=40)
    out = call(b, "step")
    check(out, b, "append")
    row = torch.from_numpy(np.concatenate([np.arange(o, o + n) for o, n in zip(np.cumsum(b.q_lens_host) - b.q_lens_host, b.q_lens_host) if n == 1])).to(DEV)
    assert torch.equal(out[row], call(b.select(b.decode_rows())))

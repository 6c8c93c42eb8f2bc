"""The rotating KV write on the GPU against its oracle, bit for bit: rotated queries, pools, scales.  Every operation behind a
stored bit is one float32 operation in a stated order, so there is no tolerance."""
import numpy as np
import pytest
import torch

from oracle import kv_write as KW
from oracle import kv_write_rope as R
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SRC = {"f32": torch.float32, "bf16": torch.bfloat16}
KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8_e4m3"), ("bf16", "fp8_e4m3_head"), ("bf16", "int8_head")]


def table_of(rows, rot, base=1000.0):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32).to(DEV)


def rows_of(gen, total, heads, d, src, mag=None):
    x = torch.randn((total, heads, d), generator=gen) * torch.exp(0.7 * torch.randn((1, heads, 1), generator=gen))
    return (x if mag is None else x * mag).to(SRC[src]).to(DEV)


def batch_of(name, heads, d, src, kv, prefix, new, seed, batch=9):
    """A workload's pools and tables; new tokens are given by the tests."""
    w = W.Workload(name, batch, heads[0], heads[1], d, src, kv, prefix, qlen=new, seed=seed, ctx_is_prefix=True)
    return W.build(w, DEV)


def both(b, q, k, v, cos_sin, *, positions=None, pair_axes=None, interleaved=False, max_q=None, q_out=None, state=None):
    """One write on the GPU, on clones of the pools, and in the oracle."""
    w = b.workload
    kp, vp, ks, vs = state or tuple(None if t is None else t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
    before = [W.raw_numpy(t) for t in (kp, vp, ks, vs)]
    q_raw = W.raw_numpy(q)
    kw = dict(cos_sin=cos_sin, positions=positions, pair_axes=pair_axes, interleaved=interleaved)
    got = B.kv_write_rope(q, k, v, b.q_lens, b.q_offsets, kp, vp, b.page_table, b.ctx_lens, max_q_len=max_q or int(max(1, b.q_lens_host.max(initial=1))),
                          k_scale=ks, v_scale=vs, q_out=q_out, **kw)
    torch.cuda.synchronize()
    want = R.kv_write_rope(q_raw, W.raw_numpy(k), W.raw_numpy(v), b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table), before[0], before[1],
                           src_dtype=w.q_dtype, kv_dtype=w.kv_dtype, k_scale=before[2], v_scale=before[3],
                           **dict(kw, cos_sin=W.raw_numpy(cos_sin), positions=W.raw_numpy(positions)))
    return (got, kp, vp, ks, vs), want


def same(got, want, what=""):
    for name, g, r in zip(("q", "k_pages", "v_pages", "k_scale", "v_scale"), got, want):
        if r is None:
            assert g is None
            continue
        g = W.raw_numpy(g)
        if g.dtype == np.float32:
            g, r = g.view(np.uint32), np.ascontiguousarray(r, dtype=np.float32).view(np.uint32)
        bad = np.argwhere(g != r)
        assert bad.size == 0, f"{what}: {name} differs at {bad[:4].tolist()} ({len(bad)} elements)"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [1.0, 0.5, 24, 8])
@pytest.mark.parametrize("src,kv", KINDS)
def test_chunks_and_single_tokens(src, kv, rot, interleaved):
    d = 128 if rot == 1.0 else 64
    rot = int(rot * d) if rot <= 1 else rot
    for heads, prefix, new, seed in (((8, 2), ("uniform", 0, 40), ("uniform", 0, 50), 1), ((32, 8), ("uniform", 0, 90), ("const", 1), 2),
                                     ((6, 3), ("uniform", 0, 20), ("uniform", 1, 20), 3)):
        b = batch_of("t", heads, d, src, kv, prefix, new, seed)
        gen = torch.Generator().manual_seed(seed)
        q, k, v = (rows_of(gen, b.total_q, h, d, src) for h in (heads[0], heads[1], heads[1]))
        got, want = both(b, q, k, v, table_of(160, rot), interleaved=interleaved)
        same(got, want, f"{heads} {new}")


@pytest.mark.parametrize("heads", [(1, 1), (20, 1), (40, 40), (5, 5), (72, 24)])
@pytest.mark.parametrize("src,kv", KINDS)
def test_head_counts(src, kv, heads):
    """More heads than a workgroup holds at once, counts that fill no round, a lone head."""
    for d, new in ((128, ("uniform", 1, 40)), (64, ("const", 1)), (64, ("const", 3))):
        b = batch_of("t", heads, d, src, kv, ("uniform", 0, 33), new, 11, batch=4)
        gen = torch.Generator().manual_seed(5)
        q, k, v = (rows_of(gen, b.total_q, h, d, src) for h in (heads[0], heads[1], heads[1]))
        got, want = both(b, q, k, v, table_of(128, d))
        same(got, want, f"{d} {new}")


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_of_several_axes(axes, interleaved):
    b = batch_of("t", (12, 4), 128, "bf16", "int8_head", ("uniform", 0, 60), ("uniform", 0, 70), 21)
    rng = np.random.default_rng(axes)
    gen = torch.Generator().manual_seed(6)
    positions = rng.integers(0, 300, (axes, b.total_q)).astype(np.int32)
    positions[:, ::17] = 299 + positions[:, ::17] % 3         # on and past the table's last row
    positions[:, 5::31] = -1
    q, k, v = (rows_of(gen, b.total_q, h, 128, "bf16") for h in (12, 4, 4))
    for pair_axes in ([0] * 32 if axes == 1 else sorted(rng.integers(0, axes, 32).tolist()), rng.integers(0, axes, 32).tolist()):
        got, want = both(b, q, k, v, table_of(300, 64), positions=torch.from_numpy(positions).to(DEV), pair_axes=pair_axes, interleaved=interleaved)
        same(got, want)
    if axes == 1:
        got, want = both(b, q, k, v, table_of(300, 64), positions=torch.from_numpy(positions[0]).to(DEV), interleaved=interleaved)
        same(got, want)


@pytest.mark.parametrize("kv", ["bf16", "int8_head"])
def test_rows_of_one_projection_in_place_and_without_queries(kv):
    b = batch_of("t", (8, 2), 128, "bf16", kv, ("uniform", 0, 30), ("uniform", 1, 40), 31)
    gen = torch.Generator().manual_seed(7)
    wide = rows_of(gen, b.total_q, 13, 128, "bf16")                # q, k, v and a head of something else
    q, k, v, _ = wide.split([8, 2, 2, 1], dim=1)
    table = table_of(100, 128)
    got, want = both(b, q, k, v, table)
    same(got, want)
    assert torch.equal(wide, torch.cat([q, k, v, wide[:, 12:]], dim=1))
    # queries rotated where they lie
    mine = q.contiguous()
    again, want = both(b, mine, k, v, table, q_out=mine)
    assert again[0].data_ptr() == mine.data_ptr()
    same(again, want)
    # keys and values alone
    alone, want = both(b, None, k, v, table)
    same(alone, want)
    for x, y in zip(alone[1:3], got[1:3]):                         # (as bytes: slots nobody has hold undefined values)
        assert alone[0] is None and torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # values elsewhere than keys, at another stride
    elsewhere, want = both(b, q, k, v.contiguous(), table)
    same(elsewhere, want)


@pytest.mark.parametrize("kv", ["fp8_e4m3", "fp8_e4m3_head", "int8_head"])
def test_pages_fill_up_turn_by_turn(kv):
    """Scales grow now and then; tokens one by one and a few at a time, rows of zeros first in some pages."""
    batch, heads, d = 6, (8, 4), 64
    gen = torch.Generator().manual_seed(8)
    total = np.zeros(batch, dtype=np.int64)
    state = None
    for turn, n in enumerate([3, 1, 1, 17, 1, 5, 1, 1, 30, 2]):
        new = np.array([n, 1, 0, n, 2, 1])
        total = total + new
        b = batch_of("t", heads, d, "bf16", kv, ("const", 96), ("const", 0), 41, batch=batch)
        for name, x in (("q_lens", new), ("ctx_lens", total)):
            setattr(b, name + "_host", x.copy())
            setattr(b, name, torch.from_numpy(x.astype(np.int32)).to(DEV))
        b.q_offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        rows = int(new.sum())
        mag = torch.exp(1.5 * torch.randn((rows, 1, 1), generator=gen)) * (torch.rand((rows, heads[1], 1), generator=gen) > 0.3)
        q, k, v = rows_of(gen, rows, 8, d, "bf16"), rows_of(gen, rows, 4, d, "bf16", mag), rows_of(gen, rows, 4, d, "bf16", mag.flip(0))
        if turn == 0:
            k.zero_()
        got, want = both(b, q, k, v, table_of(128, d), state=state)
        same(got, want, f"turn {turn}")
        state = got[1:]


def test_values_of_every_magnitude():
    """Scales from the least to far above one, zeros and subnormal numbers among the rows."""
    for kv in ("fp8_e4m3_head", "int8_head"):
        b = batch_of("t", (4, 4), 64, "bf16", kv, ("const", 0), ("const", 48), 51, batch=40)
        gen = torch.Generator().manual_seed(9)
        mag = torch.exp2(torch.randint(-133, 110, (b.total_q // 16, 1, 4, 1), generator=gen).float()).expand(-1, 16, -1, -1).reshape(-1, 4, 1)
        k, v = rows_of(gen, b.total_q, 4, 64, "bf16", mag), rows_of(gen, b.total_q, 4, 64, "bf16", mag.flip(0))
        k[::7] = 0
        got, want = both(b, None, k, v, table_of(64, 64))
        same(got, want, kv)
        assert float(got[3].min()) == 2.0 ** -64


@pytest.mark.parametrize("kv", ["fp8_e4m3_head", "int8_head"])
def test_the_plain_write_takes_the_new_pools(kv):
    b = batch_of("t", (8, 8), 128, "bf16", kv, ("uniform", 0, 60), ("uniform", 0, 80), 61)
    gen = torch.Generator().manual_seed(10)
    k, v = rows_of(gen, b.total_q, 8, 128, "bf16"), rows_of(gen, b.total_q, 8, 128, "bf16")
    want = R.kv_write_rope(None, W.raw_numpy(k), W.raw_numpy(v), b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table), W.raw_numpy(b.k_pages),
                           W.raw_numpy(b.v_pages), src_dtype="bf16", kv_dtype=kv, k_scale=W.raw_numpy(b.k_scale), v_scale=W.raw_numpy(b.v_scale))
    B.kv_write(k, v, b.q_lens, b.q_offsets, b.k_pages, b.v_pages, b.page_table, b.ctx_lens, max_q_len=int(b.q_lens_host.max()), k_scale=b.k_scale, v_scale=b.v_scale)
    same((None, b.k_pages, b.v_pages, b.k_scale, b.v_scale), want)


def test_without_rotation_the_page_rule_is_kv_writes():
    b = batch_of("t", (4, 4), 128, "bf16", "fp8_e4m3", ("uniform", 0, 60), ("uniform", 0, 80), 71)
    gen = torch.Generator().manual_seed(11)
    k, v = rows_of(gen, b.total_q, 4, 128, "bf16"), rows_of(gen, b.total_q, 4, 128, "bf16")
    still = torch.cat([torch.ones(200, 64), torch.zeros(200, 64)], dim=1).to(DEV)
    got, _ = both(b, None, k, v, still)
    B.kv_write(k, v, b.q_lens, b.q_offsets, b.k_pages, b.v_pages, b.page_table, b.ctx_lens, max_q_len=int(b.q_lens_host.max()), k_scale=b.k_scale, v_scale=b.v_scale)
    for x, y in zip(got[1:], (b.k_pages, b.v_pages, b.k_scale, b.v_scale)):
        assert torch.equal(x, y)


def test_a_pool_past_four_gigabytes():
    """Pages whose bytes, and tokens of a projection whose elements, lie behind 32 bits."""
    pages, hkv, d, kv = 270_000, 8, 128, "int8_head"
    pool = torch.empty((pages, hkv, 16, d), dtype=torch.int8, device=DEV)
    other = torch.empty_like(pool)
    ids = [pages - 1, 3, pages - 2, 262_145]
    for p in ids:
        pool[p], other[p] = 1, 2
    scale, vscale = torch.full((pages, hkv), 0.5, device=DEV), torch.full((pages, hkv), 0.25, device=DEV)
    table = torch.tensor([ids], dtype=torch.int32, device=DEV)
    gen = torch.Generator().manual_seed(12)
    rows = rows_of(gen, 40, hkv, d, "bf16")
    wide = torch.empty((40, 120_000_000), dtype=torch.bfloat16, device=DEV)
    k = wide[:, :hkv * d].view(40, hkv, d)
    k.copy_(rows)
    ctx, new, off = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([60], [40], [0, 40]))
    cos = table_of(64, d)
    B.kv_write_rope(None, k, rows, new, off, pool, other, table, ctx, cos_sin=cos, max_q_len=40, k_scale=scale, v_scale=vscale)
    want = R.kv_write_rope(None, W.raw_numpy(rows), W.raw_numpy(rows), [40], [60], np.array([[0, 1, 2, 3]]), np.full((4, hkv, 16, d), 1, np.int8),
                           np.full((4, hkv, 16, d), 2, np.int8), src_dtype="bf16", kv_dtype=kv, cos_sin=W.raw_numpy(cos),
                           k_scale=np.full((4, hkv), 0.5, np.float32), v_scale=np.full((4, hkv), 0.25, np.float32))
    same((None, pool[ids], other[ids], scale[ids], vscale[ids]), want)


@pytest.mark.parametrize("heads,d,tokens", [((8, 2), 64, 5000), ((8, 2), 64, 10000), ((4, 1), 64, 36000), ((3, 1), 128, 9000), ((1, 1), 128, 20000), ((20, 4), 64, 5000)])
@pytest.mark.parametrize("kv", ["int8_head", "bf16"])
def test_many_tokens_of_few_heads(heads, d, tokens, kv):
    """Several tokens to a wave, of trajectories that come and go between them; workgroups that take several pages of one chunk."""
    rng = np.random.default_rng(tokens)
    new = rng.integers(0, 3, 400) * rng.integers(0, 2, 400)
    long = rng.permutation(400)[:12]
    new[long] = 0
    new[long] = rng.multinomial(tokens - int(new.sum()), np.arange(1, 13) / 78)
    b = batch_of("t", heads, d, "bf16", kv, ("uniform", 0, 40), ("const", 0), 97, batch=400)
    ctx = b.ctx_lens_host + new
    pages = -(-ctx // 16)
    perm, at = rng.permutation(int(pages.sum())), 0
    table = np.full((400, int(pages.max())), -1, dtype=np.int32)
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    ints = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)
    b.ctx_lens_host, b.q_lens_host, b.ctx_lens, b.q_lens = ctx, new, ints(ctx), ints(new)
    b.q_offsets, b.page_table = ints(np.concatenate([[0], np.cumsum(new)])), ints(table)
    grow = lambda t: None if t is None else torch.zeros((at, *t.shape[1:]), dtype=t.dtype, device=DEV) + (1 if t.dtype == torch.float32 else 0)
    b.k_pages, b.v_pages, b.k_scale, b.v_scale = (grow(t) for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
    gen = torch.Generator().manual_seed(16)
    q, k, v = (rows_of(gen, tokens, h, d, "bf16") for h in (heads[0], heads[1], heads[1]))
    got, want = both(b, q, k, v, table_of(int(ctx.max()), d))
    same(got, want)


def test_queries_past_what_the_caches_hold():
    """More than 128 MB of them are written with another kind of store."""
    b = batch_of("t", (96, 2), 128, "bf16", "int8_head", ("uniform", 0, 30), ("uniform", 500, 900), 85)
    gen = torch.Generator().manual_seed(15)
    q, k, v = (rows_of(gen, b.total_q, h, 128, "bf16") for h in (96, 2, 2))
    assert q.numel() * 2 > 128 << 20
    for interleaved in (False, True):
        got, want = both(b, q, k, v, table_of(1024, 128), interleaved=interleaved)
        same(got, want)


def test_the_write_is_captured_and_replayed():
    b = batch_of("t", (8, 4), 128, "bf16", "int8_head", ("uniform", 0, 30), ("const", 1), 81)
    gen = torch.Generator().manual_seed(13)
    q, k, v = (rows_of(gen, b.total_q, h, 128, "bf16") for h in (8, 4, 4))
    table, out = table_of(64, 128), torch.empty((b.total_q, 8, 128), dtype=torch.bfloat16, device=DEV)
    call = lambda pools, o: B.kv_write_rope(q, k, v, b.q_lens, b.q_offsets, pools[0], pools[1], b.page_table, b.ctx_lens, cos_sin=table,
                                            max_q_len=1, k_scale=pools[2], v_scale=pools[3], q_out=o)
    kept = [t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    call([t.clone() for t in kept], torch.empty_like(out))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(kept, out)
    for _ in range(3):
        q.copy_(rows_of(gen, b.total_q, 8, 128, "bf16"))
        k.mul_(-1.5)
        eager = [t.clone() for t in kept]
        graph.replay()
        want = call(eager, torch.empty_like(out))
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(kept, eager))


def test_another_stream_than_the_default_one():
    b = batch_of("t", (8, 4), 128, "bf16", "fp8_e4m3_head", ("uniform", 0, 30), ("uniform", 1, 30), 91)
    gen = torch.Generator().manual_seed(14)
    q, k, v = (rows_of(gen, b.total_q, h, 128, "bf16") for h in (8, 4, 4))
    table = table_of(64, 128)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got, want = both(b, q, k, v, table)
    same(got, want)


def test_nothing_new_writes_nothing():
    b = batch_of("t", (4, 2), 64, "bf16", "int8_head", ("uniform", 0, 30), ("const", 0), 95)
    k = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    kept = b.k_pages.clone()
    out = B.kv_write_rope(q, k, k, b.q_lens, b.q_offsets, b.k_pages, b.v_pages, b.page_table, b.ctx_lens, cos_sin=table_of(8, 64), max_q_len=0,
                          k_scale=b.k_scale, v_scale=b.v_scale)
    assert out.shape == q.shape and torch.equal(kept, b.k_pages)

"""The write with norms and rotation on the GPU against its definition, bit for bit: queries, pools, scales."""
import numpy as np
import pytest
import torch

from oracle import kv_write_rope as R
from oracle import tree as T
from oracle.kv_write import _to_float32
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.tree_common import KINDS, drafts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SRC = {"f32": torch.float32, "bf16": torch.bfloat16}


def table_of(rows, rot, base=1000.0):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32).to(DEV)


def rows_of(gen, total, heads, d, src, loud=0.7):
    x = torch.randn((total, heads, d), generator=gen) * torch.exp(loud * torch.randn((1, heads, 1), generator=gen))
    return x.to(SRC[src]).to(DEV)


def weights(gen, d):
    return [(1 + 0.3 * torch.randn(d, generator=gen)).to(DEV) for _ in range(2)]


def check(b, q, k, v, cos_sin, qw, kw, what="", eps=1e-6, max_q=None, **more):
    w = b.workload
    state = [None if t is None else t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    got = B.kv_write_norm_rope(q, k, v, b.q_lens, b.q_offsets, state[0], state[1], b.page_table, b.ctx_lens, q_weight=qw, k_weight=kw, eps=eps, cos_sin=cos_sin,
                               max_q_len=max_q or int(max(1, b.q_lens_host.max(initial=1))), k_scale=state[2], v_scale=state[3], **more)
    # rows of the definition's norm as float32, then the plain rotating write's definition; its pools take v as it came
    f32 = lambda t: _to_float32(W.raw_numpy(t), w.q_dtype)
    nk = T.normalise(f32(k), kw.cpu().numpy(), eps)
    args = dict(kv_dtype=w.kv_dtype, cos_sin=W.raw_numpy(cos_sin), positions=W.raw_numpy(more.get("positions")), pair_axes=more.get("pair_axes"), interleaved=more.get("interleaved", False))
    lens = (b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table))
    pools = [W.raw_numpy(t) for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    nq = None if q is None else T.normalise(f32(q), qw.cpu().numpy(), eps)
    real = R._to_float32
    try:                                               # (float32 rows of both, whatever the call's type is)
        R._to_float32 = lambda raw, dtype: np.asarray(raw, dtype=np.float32)
        want = R.kv_write_rope(nq, nk, f32(v), *lens, pools[0], pools[1], src_dtype=w.q_dtype, k_scale=pools[2], v_scale=pools[3], **args)
    finally:
        R._to_float32 = real
    for name, g, r in zip(("q", "k_pages", "v_pages", "k_scale", "v_scale"), [got] + state, want):
        if r is None:
            assert g is None
            continue
        g, r = W.raw_numpy(g), np.ascontiguousarray(r)
        if g.dtype == np.float32:
            g, r = g.view(np.uint32), r.astype(np.float32).view(np.uint32)
        bad = np.argwhere(g != r)
        assert bad.size == 0, f"{what}: {name} differs at {bad[:4].tolist()} ({len(bad)} elements)"
    return got, state


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [1.0, 0.5, 24, 8])
@pytest.mark.parametrize("src,kv", KINDS)
def test_chunks_and_single_tokens(src, kv, rot, interleaved):
    d = 128 if rot == 1.0 else 64
    rot = int(rot * d) if rot <= 1 else rot
    for heads, prefix, new, seed in (((8, 2), ("uniform", 0, 40), ("uniform", 0, 50), 1), ((32, 8), ("uniform", 0, 90), ("const", 1), 2),
                                     ((6, 3), ("uniform", 0, 20), ("uniform", 1, 20), 3)):
        b = drafts(heads, d, src, kv, prefix, new, seed)
        gen = torch.Generator().manual_seed(seed)
        q, k, v = (rows_of(gen, b.total_q, h, d, src) for h in (heads[0], heads[1], heads[1]))
        check(b, q, k, v, table_of(160, rot), *weights(gen, d), f"{heads} {new}", interleaved=interleaved)


@pytest.mark.parametrize("heads", [(1, 1), (20, 1), (40, 40), (72, 24)])
@pytest.mark.parametrize("src,kv", KINDS)
def test_head_counts(src, kv, heads):
    for d, new in ((128, ("uniform", 1, 40)), (64, ("const", 1)), (64, ("const", 3))):
        b = drafts(heads, d, src, kv, ("uniform", 0, 33), new, 11, batch=4)
        gen = torch.Generator().manual_seed(5)
        q, k, v = (rows_of(gen, b.total_q, h, d, src) for h in (heads[0], heads[1], heads[1]))
        check(b, q, k, v, table_of(128, d), *weights(gen, d), f"{d} {new}")


@pytest.mark.parametrize("src,kv", KINDS)
def test_positions_of_a_draft_and_of_several_axes(src, kv):
    b = drafts((12, 4), 128, src, kv, ("uniform", 0, 60), ("uniform", 0, 40), 21)
    rng, gen = np.random.default_rng(3), torch.Generator().manual_seed(6)
    q, k, v = (rows_of(gen, b.total_q, h, 128, src) for h in (12, 4, 4))
    at = rng.integers(0, 310, (3, b.total_q)).astype(np.int32)
    check(b, q, k, v, table_of(300, 128), *weights(gen, 128), positions=torch.from_numpy(at[0]).to(DEV))
    check(b, q, k, v, table_of(300, 64), *weights(gen, 128), positions=torch.from_numpy(at).to(DEV), pair_axes=rng.integers(0, 3, 32).tolist())


@pytest.mark.parametrize("kv", ["bf16", "int8_head"])
def test_rows_of_one_projection_in_place_and_without_queries(kv):
    b = drafts((8, 2), 128, "bf16", kv, ("uniform", 0, 30), ("uniform", 1, 40), 31)
    gen = torch.Generator().manual_seed(7)
    wide = rows_of(gen, b.total_q, 13, 128, "bf16")
    q, k, v, _ = wide.split([8, 2, 2, 1], dim=1)
    qw, kw = weights(gen, 128)
    table = table_of(100, 128)
    out, _ = check(b, q, k, v, table, qw, kw)
    mine = q.contiguous()
    B.kv_write_norm_rope(mine, k, v, b.q_lens, b.q_offsets, b.k_pages.clone(), b.v_pages.clone(), b.page_table, b.ctx_lens, q_weight=qw, k_weight=kw, eps=1e-6, cos_sin=table,
                         max_q_len=40, k_scale=b.k_scale, v_scale=b.v_scale, q_out=mine)
    assert torch.equal(mine, out)
    check(b, None, k, v, table, None, kw)


@pytest.mark.parametrize("src,kv", KINDS)
def test_zero_faint_and_loud_rows(src, kv):
    """Rows of zeros are zeros; rows whose squares are far below eps, and near the largest float32, are what the formula says."""
    b = drafts((4, 2), 64, src, kv, ("uniform", 0, 30), ("uniform", 3, 40), 41)
    gen = torch.Generator().manual_seed(8)
    q, k, v = (rows_of(gen, b.total_q, h, 64, src) for h in (4, 2, 2))
    for x in (q, k):
        x[::4] = 0
        x[1::4] *= 2.0 ** -30
        x[2::4] *= 2.0 ** 55
    check(b, q, k, v, table_of(100, 64), *weights(gen, 64))
    check(b, q, k, v, table_of(100, 64), *weights(gen, 64), eps=0.1)


def test_long_chunks_and_one_that_stands_out():
    for new, batch in ((("uniform", 200, 900), 5), (("const", 1), 40)):
        b = drafts((8, 2), 64, "bf16", "int8_head", ("uniform", 0, 40), new, 51, batch=batch)
        gen = torch.Generator().manual_seed(9)
        q, k, v = (rows_of(gen, b.total_q, h, 64, "bf16") for h in (8, 2, 2))
        check(b, q, k, v, table_of(1000, 64), *weights(gen, 64), max_q=2000)


def test_queries_that_the_caches_cannot_hold():
    b = drafts((64, 1), 128, "bf16", "bf16", ("uniform", 0, 20), ("const", 4200), 61, batch=2)
    gen = torch.Generator().manual_seed(9)
    q, k, v = (rows_of(gen, b.total_q, h, 128, "bf16") for h in (64, 1, 1))
    qw, kw = weights(gen, 128)
    table = table_of(4300, 128)
    whole = B.kv_write_norm_rope(q, k, v, b.q_lens, b.q_offsets, b.k_pages.clone(), b.v_pages.clone(), b.page_table, b.ctx_lens, q_weight=qw, k_weight=kw, eps=1e-6,
                                 cos_sin=table, max_q_len=4200)
    few = slice(0, 50)
    small = b.select(np.array([0]))
    for h in (0, 63):
        nq = T.normalise(_to_float32(W.raw_numpy(q[few, h:h + 1]), "bf16"), qw.cpu().numpy(), 1e-6)
        at = int(small.ctx_lens_host[0]) - 4200 + np.arange(50)
        want = R.float32_to_bf16(R.rotate(nq, np.repeat(at[:, None], 64, axis=1), W.raw_numpy(table)))
        assert np.array_equal(W.raw_numpy(whole[few, h:h + 1].contiguous()), want)

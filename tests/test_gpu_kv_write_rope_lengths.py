"""The rotating KV write where chunks differ a lot, and where fewer rows are in use than the call was made for.  Bit for bit."""
import numpy as np
import pytest
import torch

from oracle import kv_write_rope as R
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.test_gpu_kv_write_rope import DEV, batch_of, both, rows_of, same, table_of

pytestmark = pytest.mark.gpu
ints = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)


def shorter(b, new):
    """The batch with other new tokens, at the ends of the contexts that it has."""
    ctx = b.ctx_lens_host - b.q_lens_host + new
    b.ctx_lens_host, b.q_lens_host, b.ctx_lens, b.q_lens = ctx, new, ints(ctx), ints(new)
    b.q_offsets = ints(np.concatenate([[0], np.cumsum(new)]))
    return b


@pytest.mark.parametrize("heads,d", [((8, 4), 128), ((4, 1), 64)])
@pytest.mark.parametrize("kv", ["int8_head", "bf16"])
def test_single_tokens_of_trajectories_that_have_ended(kv, heads, d):
    """As many rows as trajectories, as when all generate, but some have no new token and the last rows belong to nobody."""
    b = batch_of("t", heads, d, "bf16", kv, ("uniform", 0, 60), ("const", 1), 51, batch=70)
    new = (np.arange(70) % 7 != 2).astype(np.int64)
    new[:1] = new[-3:] = 0
    b = shorter(b, new)
    used = int(new.sum())
    gen = torch.Generator().manual_seed(52)
    q, k, v = (rows_of(gen, 70, h, d, "bf16") for h in (heads[0], heads[1], heads[1]))
    table = table_of(64, d)
    pools = [None if t is None else t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    before = [W.raw_numpy(t) for t in pools]
    got = B.kv_write_rope(q, k, v, b.q_lens, b.q_offsets, pools[0], pools[1], b.page_table, b.ctx_lens, cos_sin=table, max_q_len=1, k_scale=pools[2], v_scale=pools[3])
    want = R.kv_write_rope(*(W.raw_numpy(x[:used]) for x in (q, k, v)), new, b.ctx_lens_host, W.raw_numpy(b.page_table), *before[:2], src_dtype="bf16", kv_dtype=kv,
                           cos_sin=W.raw_numpy(table), k_scale=before[2], v_scale=before[3])
    same((got[:used], *pools), want)


def test_a_captured_write_is_replayed_with_trajectories_that_have_ended():
    b = batch_of("t", (8, 4), 128, "bf16", "int8_head", ("uniform", 0, 60), ("const", 1), 53, batch=20)
    gen = torch.Generator().manual_seed(54)
    q, k, v = (rows_of(gen, 20, h, 128, "bf16") for h in (8, 4, 4))
    table, out = table_of(80, 128), torch.empty((20, 8, 128), dtype=torch.bfloat16, device=DEV)
    pools = [t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    call = lambda p, o: B.kv_write_rope(q, k, v, b.q_lens, b.q_offsets, p[0], p[1], b.page_table, b.ctx_lens, cos_sin=table, max_q_len=1, k_scale=p[2], v_scale=p[3], q_out=o)
    call([t.clone() for t in pools], torch.empty_like(out))
    torch.cuda.synchronize()
    lens, offsets, ctx = b.q_lens, b.q_offsets, b.ctx_lens
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(pools, out)
    for ended in ([], [3], [0, 3, 4], [0, 3, 4, 19], list(range(19))):
        new = np.ones(20, dtype=np.int64)
        new[ended] = 0
        b.q_lens_host = np.ones(20, dtype=np.int64)
        b.ctx_lens_host = W.raw_numpy(ctx).astype(np.int64)
        now = b.ctx_lens_host - (new == 0)
        for t, x in ((lens, new), (offsets, np.concatenate([[0], np.cumsum(new)]))):
            t.copy_(ints(x))
        before, used = [W.raw_numpy(t) for t in pools], int(new.sum())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        # (a trajectory without a new token keeps its length: nothing of it is looked at)
        want = R.kv_write_rope(*(W.raw_numpy(x[:used]) for x in (q, k, v)), new, np.where(new > 0, b.ctx_lens_host, now), W.raw_numpy(b.page_table), *before[:2],
                               src_dtype="bf16", kv_dtype="int8_head", cos_sin=W.raw_numpy(table), k_scale=before[2], v_scale=before[3])
        same((out[:used], *pools), want, f"{ended}")


def skewed(kv, heads, d, new, seed):
    """A batch whose chunks are `new` behind short prefixes, pages in any order."""
    new = np.asarray(new)
    rng = np.random.default_rng(seed)
    b = batch_of("t", heads, d, "f32" if kv == "f32" else "bf16", kv, ("const", 1), ("const", 0), seed, batch=len(new))
    prefix = rng.integers(0, 40, len(new))
    ctx = prefix + new
    pages = -(-ctx // 16)
    perm, at = rng.permutation(int(pages.sum())), 0
    table = np.full((len(new), max(1, int(pages.max()))), -1, dtype=np.int32)
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    b.ctx_lens_host, b.q_lens_host, b.ctx_lens, b.q_lens = ctx, new, ints(ctx), ints(new)
    b.q_offsets, b.page_table = ints(np.concatenate([[0], np.cumsum(new)])), ints(table)
    grow = lambda t: None if t is None else torch.zeros((at, *t.shape[1:]), dtype=t.dtype, device=DEV) + (1 if t.dtype == torch.float32 else 0)
    b.k_pages, b.v_pages, b.k_scale, b.v_scale = (grow(t) for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
    return b


def chunks(kind, rng):
    if kind == "one long among single tokens":
        new = np.ones(300, dtype=np.int64)
        new[111] = 5000
    elif kind == "the first":
        new = rng.integers(0, 2, 65)
        new[0] = 3000
    elif kind == "the last":
        new = rng.integers(0, 2, 4100)
        new[-1] = 2000
    elif kind == "alone":
        new = np.zeros(500, dtype=np.int64)
        new[250] = 4000
    else:
        new = np.exp(rng.uniform(0, np.log(700), 130)).astype(np.int64) * rng.integers(0, 2, 130)
    return new


@pytest.mark.parametrize("kind", ["one long among single tokens", "the first", "the last", "alone", "uneven"])
@pytest.mark.parametrize("kv,heads,d", [("int8_head", (8, 2), 64), ("int8_head", (4, 4), 128), ("fp8_e4m3_head", (8, 2), 64), ("fp8_e4m3", (6, 2), 64), ("bf16", (8, 2), 64), ("f32", (2, 2), 64)])
def test_chunks_that_differ_a_lot(kv, heads, d, kind):
    new = chunks(kind, np.random.default_rng(55))
    b = skewed(kv, heads, d, new, 56)
    gen = torch.Generator().manual_seed(57)
    src = b.workload.q_dtype
    q, k, v = (rows_of(gen, int(new.sum()), h, d, src) for h in (heads[0], heads[1], heads[1]))
    table = table_of(int(b.ctx_lens_host.max()), d)
    got, want = both(b, q, k, v, table)
    same(got, want)
    got, want = both(b, None, k, v, table, max_q=100_000)                 # (more than the longest is allowed)
    same(got, want)


def test_more_page_places_than_a_launch_has():
    """A batch of 4200 with one chunk of 33000 tokens: the longest chunk's pages for every trajectory would be 17 million workgroups."""
    new = np.ones(4200, dtype=np.int64)
    new[1234] = 33_000
    b = skewed("int8_head", (8, 8), 64, new, 58)
    gen = torch.Generator().manual_seed(59)
    k, v = (rows_of(gen, int(new.sum()), 8, 64, "bf16") for _ in range(2))
    got, want = both(b, None, k, v, table_of(4096, 64))
    same(got, want)
    kept = [t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    B.kv_write(k, v, b.q_lens, b.q_offsets, kept[0], kept[1], b.page_table, b.ctx_lens, max_q_len=33_000, k_scale=kept[2], v_scale=kept[3])
    assert torch.equal(kept[1], got[2]) and torch.equal(kept[3], got[4])


@pytest.mark.parametrize("heads,d", [((96, 2), 128), ((128, 4), 64)])
def test_chunks_that_differ_a_lot_with_more_queries_than_the_caches_hold(heads, d):
    """More than 128 MB of rotated queries are written with another kind of store."""
    new = np.ones(200, dtype=np.int64)
    new[77] = (130 << 20) // (heads[0] * d * 2)
    b = skewed("int8_head", heads, d, new, 60)
    gen = torch.Generator().manual_seed(61)
    q, k, v = (rows_of(gen, int(new.sum()), h, d, "bf16") for h in (heads[0], heads[1], heads[1]))
    assert q.numel() * 2 > 128 << 20
    got, want = both(b, q, k, v, table_of(int(b.ctx_lens_host.max()), d))
    same(got, want)

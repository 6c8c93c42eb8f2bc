"""A step with drafts as an engine makes it: attn_tree_mask, kv_write_norm_rope, attn_tree, kv_accept, then decode.  Eager and as a graph, on
other streams, two at a time.

Tolerances: attn_tree and attn_decode each are within 2^-7 + 1e-4 of the largest value a row sees of the formula over 16-bit queries (weights
and results rounded to bf16, half a step each), 1e-4 over float32; two of them differ by twice that."""
import numpy as np
import pytest
import torch

from oracle import tree as T
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.helpers import oracle_args
from tests.test_gpu_kv_write_norm_rope import rows_of, table_of, weights
from tests.tree_common import KINDS, drafts, parents_of, words_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)


class Step:
    """Inputs and buffers of a batch's step, as an engine keeps them."""

    def __init__(self, b, seed, chain=False):
        w = b.workload
        gen = torch.Generator().manual_seed(seed)
        self.b, self.w = b, w
        self.parents_host = parents_of(b, seed, chain)
        self.parents = ints(self.parents_host)
        self.q, self.k, self.v = (rows_of(gen, b.total_q, h, w.head_dim, w.q_dtype) for h in (w.num_q_heads, w.num_kv_heads, w.num_kv_heads))
        self.qw, self.kw = weights(gen, w.head_dim)
        self.table = table_of(int(b.ctx_lens_host.max()) + 1, w.head_dim)
        self.most = int(max(1, b.q_lens_host.max()))
        self.choose(seed)
        self.mask = torch.zeros((b.total_q, words_of(b)), dtype=torch.int64, device=DEV)
        self.positions = torch.zeros_like(self.parents)
        self.q_out, self.out = torch.empty_like(self.q), torch.empty_like(self.q)
        self.lse = torch.zeros((b.total_q, w.num_q_heads), device=DEV)
        self.ws = B.alloc_tree_workspace(self.q_out, b.k_pages, b.v_pages, b.page_table, b.ctx_lens, max_q_len=self.most, k_scale=b.k_scale, v_scale=b.v_scale)

    def choose(self, seed):
        """A node of every draft and its ancestors."""
        rng, rows, lens, at = np.random.default_rng(seed), [], [], 0
        for n in self.b.q_lens_host.tolist():
            i, path = int(rng.integers(0, n)) if n else -1, []
            while i >= 0:
                path.append(i)
                i = int(self.parents_host[at + i])
            rows.append(np.array(path[::-1] + [-1] * (n - len(path)), dtype=np.int64))
            lens.append(len(path))
            at += n
        self.paths, self.path_lens = rows, np.array(lens)
        self.accepted, self.accept_lens = ints(np.concatenate(rows)), ints(lens)

    def run(self, accept=True):
        b = self.b
        where = (b.q_lens, b.q_offsets)
        pools = (b.k_pages, b.v_pages, b.page_table, b.ctx_lens)
        scales = dict(k_scale=b.k_scale, v_scale=b.v_scale)
        B.attn_tree_mask(self.parents, *where, b.ctx_lens, max_q_len=self.most, tree_mask=self.mask, positions=self.positions)
        B.kv_write_norm_rope(self.q, self.k, self.v, *where, *pools, q_weight=self.qw, k_weight=self.kw, eps=1e-6, cos_sin=self.table, max_q_len=self.most,
                             positions=self.positions, q_out=self.q_out, **scales)
        B.attn_tree(self.q_out, *where, self.mask, *pools, sm_scale=self.w.sm_scale, max_q_len=self.most, out=self.out, lse=self.lse, workspace=self.ws, **scales)
        if accept:
            B.kv_accept(self.accepted, self.accept_lens, *where, *pools, max_q_len=self.most, **scales)

    def state(self):
        b = self.b
        return [t for t in (self.out, self.lse, self.q_out, self.mask, self.positions, b.k_pages, b.v_pages, b.k_scale, b.v_scale) if t is not None]


def bits(t):
    return t.contiguous().view(torch.uint8)


def same(x, y):
    return all(torch.equal(bits(i), bits(j)) for i, j in zip(x, y))


def bound(src):
    return 2 * ((0.0 if src == "f32" else 2.0 ** -7) + 1e-4)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS)
def test_an_accepted_path_is_what_its_tokens_one_after_the_other_are(src, kv, d):
    for heads, prefix, new in (((8, 2), ("uniform", 3, 150), ("uniform", 1, 20)), ((4, 1), ("uniform", 900, 1500), ("uniform", 2, 70))):
        b = drafts(heads, d, src, kv, prefix, new, 5)
        for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
            setattr(b, "before_" + name, None if getattr(b, name) is None else getattr(b, name).clone())
        s = Step(b, 9)
        s.run()
        out = s.out.clone()
        # the path's tokens as a chain, over the caches as they were before
        chain = torch.cat([torch.from_numpy(p[:n]) + int(o) for p, n, o in zip(s.paths, s.path_lens, b.q_offsets.cpu().tolist())]).to(DEV)
        ctx = b.ctx_lens_host - b.q_lens_host + s.path_lens
        pools = [getattr(b, "before_" + name) for name in ("k_pages", "v_pages")]
        scales = dict(k_scale=b.before_k_scale, v_scale=b.before_v_scale)
        offsets = np.concatenate([[0], np.cumsum(s.path_lens)])
        where = (ints(s.path_lens), ints(offsets))
        q = B.kv_write_norm_rope(s.q[chain], s.k[chain], s.v[chain], *where, *pools, b.page_table, ints(ctx), q_weight=s.qw, k_weight=s.kw, eps=1e-6,
                                 cos_sin=s.table, max_q_len=int(s.path_lens.max()), **scales)
        assert torch.equal(bits(q), bits(s.q_out[chain]))                # (positions: behind the prefix and the ancestors)
        if kv in ("f32", "bf16"):
            for t, n in enumerate(ctx.tolist()):
                for g in range(heads[1]):
                    for now, then in ((b.k_pages, pools[0]), (b.v_pages, pools[1])):
                        assert torch.equal(bits(B.debug_gather(now, b.page_table, ints(ctx), t, g, n)), bits(B.debug_gather(then, b.page_table, ints(ctx), t, g, n)))
        # decode of the last accepted token over the caches as the step leaves them
        last = torch.from_numpy(np.cumsum(s.path_lens) - 1).to(DEV)
        got = B.attn_decode(q[last].contiguous(), b.k_pages, b.v_pages, b.page_table, ints(ctx), sm_scale=s.w.sm_scale, k_scale=b.k_scale, v_scale=b.v_scale)
        rows = chain[last]
        most = float(torch.cat([s.v.float().abs().amax().reshape(1), out.float().abs().amax().reshape(1)]).max())
        if kv in ("f32", "bf16"):
            ref, _, top = T.attn_tree(W.raw_numpy(q[last].contiguous()), np.ones(len(ctx), np.int64), np.ones((len(ctx), 1), np.uint64),
                                      **dict(oracle_args(b), ctx_lens=ctx))
            for x in (got, out[rows]):
                assert (np.abs(x.double().cpu().numpy() - ref) <= bound(src) * top[:, :, None]).all()
        else:
            # (a page whose scale has grown rounds its codes anew: half a step of the largest, 2^-4 of an E4M3 code and 1/254 of an int8 page's largest, twice)
            step = 2.0 ** -3 if kv.startswith("fp8") else 1 / 127
            assert float((got.float() - out[rows].float()).abs().max()) <= (bound(src) + 4 * step) * most


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "fp8_e4m3_head", "int8_head"])
@pytest.mark.parametrize("new", [("uniform", 1, 7), ("uniform", 4, 16), ("uniform", 20, 90)])
def test_replays_from_a_graph_like_eager(kv, new):
    b = drafts((8, 2), 128, "bf16", kv, ("uniform", 0, 1600), new, 21, batch=70 if new[2] == 7 else 9)
    s = Step(b, 3)
    pools = [t for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale) if t is not None]
    first = [t.clone() for t in pools]
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    ctx0, lens0 = b.ctx_lens.clone(), b.q_lens_host.copy()
    gen = torch.Generator().manual_seed(4)
    for it in range(4):
        # other values, shorter contexts, other trees and paths
        for t in (s.q, s.k, s.v):
            t.copy_((torch.randn(t.shape, generator=gen) * (1 + it)).to(t.dtype))
        shorter = torch.minimum(torch.full_like(ctx0, 37 * it), ctx0 - b.q_lens)
        b.ctx_lens.copy_(ctx0 - shorter)
        s.parents_host = parents_of(b, 50 + it)
        s.parents.copy_(ints(s.parents_host))
        kept = (s.accepted, s.accept_lens)
        s.choose(60 + it)
        for old, new_one, name in zip(kept, (s.accepted, s.accept_lens), ("accepted", "accept_lens")):
            old.copy_(new_one)
            setattr(s, name, old)
        for t, f in zip(pools, first):
            t.copy_(f)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in s.state()]
        for t, f in zip(pools, first):
            t.copy_(f)
        for t in (s.out, s.lse, s.q_out, s.mask, s.positions):
            t.zero_()
        s.run()
        torch.cuda.synchronize()
        assert same(got, s.state()), it
        assert torch.isfinite(got[0].float()).all()


def test_two_graphs_with_a_workspace_each_and_a_shared_one():
    """Replayed side by side with a workspace each, one after the other with one for both."""
    a, c = (Step(drafts((8, 2), 128, "bf16", "bf16", ("uniform", 1100, 3000), ("uniform", 1, 16), seed, batch=6), seed) for seed in (31, 32))
    want = []
    for s in (a, c):
        s.run(accept=False)
        want.append([t.clone() for t in s.state()])
    torch.cuda.synchronize()
    own = c.ws
    for ws, together in ((own, True), (a.ws, False)):
        c.ws = ws
        graphs = []
        for s in (a, c):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                s.run(accept=False)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if together else [torch.cuda.current_stream()] * 2
        for _ in range(3):
            for s in (a, c):
                s.out.zero_()
            torch.cuda.synchronize()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            torch.cuda.synchronize()
            assert same(a.state(), want[0]) and same(c.state(), want[1])


def test_on_another_stream():
    s = Step(drafts((8, 2), 64, "bf16", "int8_head", ("uniform", 0, 2000), ("uniform", 1, 9), 41, batch=20), 41)
    pools = [t for t in (s.b.k_pages, s.b.v_pages, s.b.k_scale, s.b.v_scale) if t is not None]
    first = [t.clone() for t in pools]
    s.run()
    want = [t.clone() for t in s.state()]
    for t, f in zip(pools, first):
        t.copy_(f)
    s.out.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.run()
    side.synchronize()
    assert same(s.state(), want)


def test_trajectories_that_share_their_prefix():
    """Pages of a common prefix in several tables: read by all, written by none (the drafts begin behind it, on their own pages)."""
    b = drafts((8, 2), 128, "bf16", "bf16", ("const", 1600), ("uniform", 1, 12), 51, batch=6)
    alone = b.page_table.clone()
    b.page_table[1:, :100] = alone[:1, :100]
    s = Step(b, 51)
    s.run(accept=False)
    shared = s.out.clone()
    # the same contexts with pages of their own
    for pool in (b.k_pages, b.v_pages):
        for t in range(1, 6):
            pool[alone[t, :100].long()] = pool[alone[0, :100].long()]
    b.page_table.copy_(alone)
    s.run(accept=False)
    assert torch.equal(bits(shared), bits(s.out))


@pytest.mark.parametrize("kv", ["fp8_e4m3_head", "int8_head"])
@pytest.mark.parametrize("q_mag,k_mag", [(2.0 ** 60, 2.0 ** -60), (2.0 ** -60, 2.0 ** 60), (2.0 ** 12, 2.0 ** -9), (2.0 ** -70, 1.0)])
def test_queries_and_scales_of_all_sizes(kv, q_mag, k_mag):
    """Products of ordinary size from large queries over faint keys and the reverse; queries too faint to matter (all weights alike)."""
    for new in (("uniform", 1, 8), ("uniform", 20, 40)):
        b = drafts((8, 2), 64, "bf16", kv, ("uniform", 0, 1500), new, 61, batch=5)
        b.q = (b.q.float() * q_mag).to(torch.bfloat16)
        b.k_scale *= k_mag
        mask = T.tree_mask(parents_of(b, 3), b.q_lens_host, b.ctx_lens_host, words_of(b))[0]
        got = B.attn_tree(b.q, b.q_lens, b.q_offsets, torch.from_numpy(mask.view(np.int64)).to(DEV), b.k_pages, b.v_pages, b.page_table, b.ctx_lens,
                          sm_scale=b.workload.sm_scale, max_q_len=int(b.q_lens_host.max()), k_scale=b.k_scale, v_scale=b.v_scale)
        ref, _, most = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **oracle_args(b))
        assert (np.abs(got.double().cpu().numpy() - ref) <= bound("bf16") / 2 * most[:, :, None]).all()

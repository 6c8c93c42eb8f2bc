"""What the calls around drafts refuse before anything is launched (no GPU needed), and pins of their definitions."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import attention as O
from oracle import tree as T
from paper_2512_22560_amd import binding as B
from paper_2512_22560_amd import workloads as W
from tests.helpers import oracle_args
from tests.tree_common import any_masks, drafts, parents_of, words_of

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first, or there is nothing to launch
ODD = ctypes.c_void_p(0x1008)


def _desc(**kw):
    base = dict(batch=4, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_pages_per_seq=16, num_pages=43,
                q_dtype=B.BF16, kv_dtype=B.INT8_HEAD, sm_scale=0.125, k_scale=0x1000, v_scale=0x1000)
    base.update(kw)
    return B.Desc(**base)


def _tree(d=None, q=FAKE, lens=FAKE, total=4, most=1, mask=FAKE, words=1, out=FAKE, lse=None, ws=FAKE, room=1 << 40):
    return B.lib().attn_tree(ctypes.byref(d or _desc()), q, lens, FAKE, total, most, mask, words, FAKE, FAKE, FAKE, FAKE, out, lse, ws, room, None)


def test_attention_of_drafts_refuses():
    assert _tree(total=0) == 0 and _tree(_desc(batch=0)) == 0                     # nothing to do
    assert _tree(total=-1) == -1 and _tree(most=-1) == -1 and _tree(most=0) == -1
    for words in (0, -1, 17):
        assert _tree(words=words) == -2
    for name in ("q", "lens", "mask", "out", "ws"):
        assert _tree(**{name: None}) == -1 and _tree(**{name: ODD}) == -4, name
    assert _tree(lse=ODD) == -4 and _tree(room=16) == -5
    assert _tree(_desc(head_dim=96)) == -2 and _tree(_desc(page_size=32)) == -2 and _tree(_desc(num_q_heads=9)) == -2 and _tree(_desc(batch=70000)) == -2
    assert _tree(_desc(num_q_heads=514, num_kv_heads=2)) == -2                    # more query heads to a KV head than attn_append takes
    assert _tree(_desc(k_scale=None)) == -3 and _tree(_desc(q_dtype=B.F32)) == -3 and _tree(_desc(sm_scale=float("nan"))) == -1
    assert B.lib().attn_tree(None, *([FAKE] * 3), 4, 1, FAKE, 1, *([FAKE] * 5), None, FAKE, 1 << 40, None) == -1
    size = lambda d, total=4, most=1: B.lib().rollattn_tree_workspace_bytes(ctypes.byref(d), total, most)
    assert size(_desc()) > 0 and size(_desc(), 0, 0) > 0
    assert size(_desc(head_dim=96)) == 0 and size(_desc(), -1) == 0 and size(_desc(), 4, -1) == 0


def test_masks_refuse():
    def call(parents=FAKE, lens=FAKE, off=FAKE, ctx=FAKE, batch=4, total=4, most=1, mask=FAKE, words=1, positions=None):
        return B.lib().attn_tree_mask(parents, lens, off, ctx, batch, total, most, mask, words, positions, None)
    assert call(batch=0) == 0 and call(total=0) == 0
    assert call(batch=-1) == -1 and call(total=-1) == -1 and call(most=-1) == -1 and call(batch=70000) == -2
    for words in (0, -1, 17):
        assert call(words=words) == -2
    for name in ("parents", "lens", "off", "ctx", "mask"):
        assert call(**{name: None}) == -1 and call(**{name: ODD}) == -4, name
    assert call(positions=ODD) == -4


def test_the_move_refuses():
    def call(d=None, accepted=FAKE, m=FAKE, lens=FAKE, total=4, most=1, pages=FAKE, ks=FAKE):
        return B.lib().kv_accept(ctypes.byref(d or _desc()), accepted, m, lens, FAKE, total, most, pages, FAKE, FAKE, FAKE, ks, FAKE, None)
    assert call(total=0) == 0 and call(_desc(batch=0)) == 0
    assert call(total=-1) == -1 and call(most=-1) == -1 and call(_desc(batch=70000)) == -2 and call(_desc(head_dim=32)) == -2
    for name in ("accepted", "m", "lens", "pages"):
        assert call(**{name: None}) == -1 and call(**{name: ODD}) == -4, name
    assert call(ks=None) == -3 and call(ks=ODD) == -4 and call(_desc(kv_dtype=B.BF16, k_scale=None, v_scale=None), ks=None, total=0) == 0


def test_the_write_with_norms_refuses():
    def call(norm=(0x1000, 0x1000, 1e-6), q=FAKE, rot=64, scale=FAKE):
        rope = B.Rope(cos_sin=0x1000, num_positions=64, rot_dim=rot, num_axes=1)
        n = None if norm is None else ctypes.byref(B.Norm(*norm))
        return B.lib().kv_write_norm_rope(ctypes.byref(_desc()), ctypes.byref(rope), n, q, FAKE, FAKE, FAKE, FAKE, 4, 1, q, FAKE, FAKE, FAKE, FAKE, scale, FAKE, None)
    assert call(None) == -1
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert call((0x1000, 0x1000, eps)) == -1
    assert call((None, 0x1000, 1e-6)) == -1 and call((0x1000, None, 1e-6)) == -1
    assert call((0x1008, 0x1000, 1e-6)) == -4 and call((0x1000, 0x1008, 1e-6)) == -4
    assert call(rot=20) == -2
    assert call(scale=None) == -3 and call((None, 0x1000, 1e-6), q=None, scale=None) == -3             # (what is left to object to: a scale is missing)


ints = lambda *s: torch.zeros(s, dtype=torch.int32)
bf = torch.bfloat16


def refuses(name, args, what):
    with pytest.raises((ValueError, TypeError), match=what):
        getattr(B, name)(**args)


def test_the_binding_refuses():
    pools = dict(k_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8), v_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8), page_table=ints(3, 4), ctx_lens=ints(3),
                 k_scale=torch.zeros(5, 2), v_scale=torch.zeros(5, 2))
    chunk = dict(q_lens=ints(3), q_offsets=ints(4), stream=0)
    mask = torch.zeros(6, 1, dtype=torch.int64)
    tree = dict(q=torch.zeros(6, 4, 64, dtype=bf), tree_mask=mask, sm_scale=0.1, max_q_len=2, workspace=torch.zeros(16, dtype=torch.uint8), **chunk, **pools)
    for change, what in (({}, "one GPU"), ({"tree_mask": mask[:5]}, "tree_mask"), ({"tree_mask": mask.int()}, "tree_mask"), ({"tree_mask": mask[:, 0]}, "tree_mask"),
                         ({"lse": torch.zeros(6, 3)}, "lse"), ({"lse": torch.zeros(6, 4, dtype=bf)}, "lse"), ({"q_lens": ints(2)}, "q_lens"), ({"q_offsets": ints(3)}, "q_offsets"),
                         ({"ctx_lens": ints(2)}, "ctx_lens"), ({"q": torch.zeros(6, 4, 32, dtype=bf)}, "query rows"), ({"v_pages": torch.zeros(5, 2, 16, 32, dtype=torch.int8)}, "both pools"),
                         ({"out": torch.zeros(5, 4, 64, dtype=bf)}, "out"), ({"k_scale": torch.zeros(5)}, "scales"), ({"q": torch.zeros(6, 4, 128, dtype=bf)[:, :, ::2]}, "dense")):
        refuses("attn_tree", dict(tree, **change), what)
    par = dict(parents=ints(6), ctx_lens=ints(3), max_q_len=2, tree_mask=mask, positions=ints(6), **chunk)
    for change, what in (({}, "one GPU"), ({"tree_mask": mask.int()}, "tree_mask"), ({"tree_mask": mask[:4]}, "tree_mask"), ({"positions": ints(5)}, "positions"),
                         ({"positions": torch.zeros(6)}, "positions"), ({"parents": ints(6, 1)}, "parents"), ({"parents": torch.zeros(6, dtype=torch.int64)}, "parents"),
                         ({"q_offsets": ints(3)}, "q_offsets"), ({"ctx_lens": ints(1)}, "ctx_lens")):
        refuses("attn_tree_mask", dict(par, **change), what)
    move = dict(accepted=ints(6), accept_lens=ints(3), max_q_len=2, **chunk, **pools)
    for change, what in (({}, "one GPU"), ({"accept_lens": ints(2)}, "accept_lens"), ({"accepted": torch.zeros(6)}, "accepted"), ({"accepted": ints(6, 1)}, "accepted"),
                         ({"v_pages": torch.zeros(4, 2, 16, 64, dtype=torch.int8)}, "both pools"), ({"page_table": ints(3)}, "page_table"), ({"v_scale": torch.zeros(5)}, "scales")):
        refuses("kv_accept", dict(move, **change), what)
    write = dict(q=torch.zeros(6, 4, 64, dtype=bf), k_new=torch.zeros(6, 2, 64, dtype=bf), v_new=torch.zeros(6, 2, 64, dtype=bf), cos_sin=torch.zeros(8, 64), max_q_len=2, eps=1e-6,
                 q_weight=torch.zeros(64), k_weight=torch.zeros(64), **chunk, **pools)
    for change, what in (({}, "one GPU"), ({"q_weight": torch.zeros(32)}, "weights"), ({"k_weight": torch.zeros(64, dtype=bf)}, "weights"), ({"q_weight": None}, "weights"),
                         ({"k_weight": torch.zeros(128)[::2]}, "dense"), ({"cos_sin": torch.zeros(8)}, "cos_sin"), ({"k_new": torch.zeros(6, 1, 64, dtype=bf)}, "rows of the pools")):
        refuses("kv_write_norm_rope", dict(write, **change), what)


# ---- pins of the definitions

def test_a_chain_is_causal():
    b = drafts((4, 2), 16, "f32", "f32", ("uniform", 0, 20), ("uniform", 1, 70), 3, device="cpu")
    mask, positions = T.tree_mask(parents_of(b, 1, chain=True), b.q_lens_host, b.ctx_lens_host, words_of(b))
    args = oracle_args(b)
    out, lse, _ = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **args)
    assert np.allclose(out, O.attn_append(W.raw_numpy(b.q), b.q_lens_host, **args), atol=1e-12)
    assert np.array_equal(positions, np.concatenate([np.arange(l - n, l) for n, l in zip(b.q_lens_host, b.ctx_lens_host)]))


def test_every_path_of_a_tree_is_its_own_trajectory():
    """A node's row is what a trajectory gives whose context is the cached tokens and the node's ancestors."""
    b = drafts((2, 1), 16, "f32", "f32", ("const", 16), ("const", 9), 4, batch=1, device="cpu")
    parents = parents_of(b, 2)
    mask, positions = T.tree_mask(parents, b.q_lens_host, b.ctx_lens_host, 1)
    out, _, _ = T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **oracle_args(b))
    for i in range(9):
        path, j = [], i
        while j >= 0:
            path.append(j)
            j = int(parents[j])
        path = path[::-1]
        k, v, _, _ = T.accept(np.array(path + [0] * (9 - len(path))), [len(path)], b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table), W.raw_numpy(b.k_pages),
                              W.raw_numpy(b.v_pages), kv_dtype="f32")
        alone = O.attn_decode(W.raw_numpy(b.q[i:i + 1]), **dict(oracle_args(b), k_pages=k, v_pages=v, ctx_lens=np.array([16 + len(path)])))
        assert np.allclose(alone[0], out[i], atol=1e-12) and positions[i] == 16 + len(path) - 1


def test_the_norm_is_the_formula():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 3, 64)).astype(np.float32), rng.standard_normal(64).astype(np.float32)
    want = x.astype(np.float64) / np.sqrt((x.astype(np.float64) ** 2).mean(axis=-1, keepdims=True) + 1e-5) * w
    assert np.abs(T.normalise(x, w, 1e-5) - want).max() < 8 * 2.0 ** -24 * np.abs(want).max()
    assert (T.normalise(np.zeros((1, 64), np.float32), w, 1e-6) == 0).all()


@pytest.mark.parametrize("kv,step", [("fp8_e4m3", 2.0 ** -4), ("fp8_e4m3_head", 2.0 ** -4), ("int8_head", 1.0 / 254)])
def test_moved_rows_keep_their_values_within_a_step(kv, step):
    """Rows of 8-bit pools are off by half a step of the new scale at most: int8 magnitudes of normal values stay below 5, so steps below 5 / 127; E4M3
    2^-4 of the value, 2^-10 of the scale (5 / 448) where it is smallest."""
    b = drafts((4, 4), 64, "bf16", kv, ("uniform", 0, 30), ("const", 40), 5, device="cpu")
    accepted = np.concatenate([np.concatenate([np.arange(1, 40, 3), np.zeros(27, dtype=np.int64)]) for _ in range(7)])
    before = [W.raw_numpy(t) for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)]
    after = T.accept(accepted, [13] * 7, b.q_lens_host, b.ctx_lens_host, W.raw_numpy(b.page_table), before[0], before[1], kv_dtype=kv, k_scale=before[2], v_scale=before[3])
    table = W.raw_numpy(b.page_table)
    for t in range(7):
        first = int(b.ctx_lens_host[t]) - 40
        for g in range(4):
            old = O.gather_tokens(before[0], table, t, g, first + 40, kv, before[2])
            new = O.gather_tokens(after[0], table, t, g, first + 13, kv, after[2])
            assert np.allclose(new[first:], old[first + 1 + 3 * np.arange(13)], rtol=step if kv != "int8_head" else 0, atol=0.02 if kv == "int8_head" else 1e-3)
            assert np.allclose(new[:first], old[:first], rtol=step if kv != "int8_head" else 0, atol=0.02 if kv == "int8_head" else 1e-3)


def test_masks_with_more_words_than_the_draft():
    b = drafts((2, 1), 16, "f32", "f32", ("const", 0), ("const", 3), 6, batch=2, device="cpu")
    mask = any_masks(b, 1)
    wide = np.concatenate([mask, np.full_like(mask, 2 ** 64 - 1)], axis=1)
    args = oracle_args(b)
    assert np.array_equal(T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, mask, **args)[0], T.attn_tree(W.raw_numpy(b.q), b.q_lens_host, wide, **args)[0])

"""What the rotating write and the pools with scales for heads refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2512_22560_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first, or there is nothing to launch


def _desc(**kw):
    base = dict(batch=4, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_pages_per_seq=16, num_pages=43,
                q_dtype=B.BF16, kv_dtype=B.INT8_HEAD, sm_scale=0.125, k_scale=None, v_scale=None)
    base.update(kw)
    return B.Desc(**base)


def _rope(**kw):
    base = dict(cos_sin=0x1000, positions=None, pair_axes=None, num_positions=64, rot_dim=64, num_axes=1, interleaved=0, q_stride=0, k_stride=0, v_stride=0)
    base.update(kw)
    return B.Rope(**base)


def _write(d=None, r=None, q=FAKE, q_out=FAKE, total_q=4, max_q=1, k_new=FAKE, ks=FAKE, rope=True):
    d, r = d or _desc(), r or _rope()
    return B.lib().kv_write_rope(ctypes.byref(d), ctypes.byref(r) if rope else None, q, k_new, FAKE, FAKE, FAKE, total_q, max_q, q_out, FAKE, FAKE,
                                 FAKE, FAKE, ks, FAKE, None)


def test_the_rotating_write_refuses():
    odd = ctypes.c_void_p(0x1008)
    assert _write(total_q=0) == 0 and _write(_desc(batch=0)) == 0              # nothing to do
    assert _write(rope=False) == -1 and _write(total_q=-1) == -1 and _write(max_q=-1) == -1
    assert B.lib().kv_write_rope(None, ctypes.byref(_rope()), *([FAKE] * 5), 4, 1, *([FAKE] * 7), None) == -1
    assert _write(r=_rope(num_positions=0)) == -1 and _write(r=_rope(cos_sin=None)) == -1
    for rot in (0, -8, 4, 20, 72, 128):
        assert _write(r=_rope(rot_dim=rot)) == -2
    for axes in (0, 5, -1):
        assert _write(r=_rope(num_axes=axes)) == -2
    assert _write(r=_rope(num_axes=2)) == -1                                    # several axes without positions
    assert _write(r=_rope(num_axes=2, positions=0x1000, pair_axes=bytes([0, 2] * 16))) == -1
    assert _write(r=_rope(positions=0x1008)) == -4 and _write(r=_rope(cos_sin=0x1008)) == -4
    assert _write(r=_rope(q_stride=8 * 64 - 8)) == -2 and _write(r=_rope(k_stride=64)) == -2 and _write(r=_rope(v_stride=-128)) == -2
    assert _write(r=_rope(v_stride=2 * 64 + 4)) == -4                           # rows that start between 16-byte places
    assert _write(q=None) == -1 and _write(q_out=None) == -1
    assert _write(r=_rope(q_stride=1024)) == -1                                 # in place, but the rows do not lie densely
    assert _write(k_new=None) == -1 and _write(k_new=odd) == -4 and _write(q_out=odd) == -4
    assert _write(ks=None) == -3 and _write(ks=odd) == -4
    assert _write(_desc(batch=70000)) == -2 and _write(_desc(head_dim=96)) == -2
    assert _write(_desc(q_dtype=B.F32)) == -3                                   # 8-bit pools are written from bf16 rows
    assert _write(_desc(q_dtype=B.INT8_HEAD)) == -3 and _write(_desc(kv_dtype=5)) == -3


@pytest.mark.parametrize("kv", [B.FP8_E4M3_HEAD, B.INT8_HEAD])
def test_attention_over_the_new_pools_refuses(kv):
    lib = B.lib()
    def decode(d, ws=1 << 40):
        return lib.attn_decode(ctypes.byref(d), *([FAKE] * 7), ws, None)
    scales = dict(k_scale=0x1000, v_scale=0x1000)
    assert decode(_desc(kv_dtype=kv)) == -3                                     # no scales
    assert decode(_desc(kv_dtype=kv, k_scale=0x1000, v_scale=0x1004)) == -4
    assert decode(_desc(kv_dtype=kv, **scales), ws=16) == -5
    assert decode(_desc(kv_dtype=kv, q_dtype=B.F32, **scales)) == -3
    assert decode(_desc(kv_dtype=kv, num_pages=1 << 31, **scales)) == -2
    assert decode(_desc(kv_dtype=kv, batch=0, **scales)) == 0
    assert lib.rollattn_workspace_bytes(ctypes.byref(_desc(kv_dtype=kv, **scales)), 4) == lib.rollattn_workspace_bytes(
        ctypes.byref(_desc(kv_dtype=B.FP8_E4M3, **scales)), 4) > 0
    assert lib.kv_write(ctypes.byref(_desc(kv_dtype=kv)), *([FAKE] * 4), 4, 1, *([FAKE] * 4), None, FAKE, None) == -3
    assert lib.kv_write(ctypes.byref(_desc(kv_dtype=kv, q_dtype=B.F32)), *([FAKE] * 4), 4, 1, *([FAKE] * 6), None) == -3


def test_the_binding_refuses_what_the_library_cannot_see():
    bf, f32, i8 = torch.bfloat16, torch.float32, torch.int8
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    base = dict(q=torch.zeros(3, 4, 64, dtype=bf), k_new=torch.zeros(3, 2, 64, dtype=bf), v_new=torch.zeros(3, 2, 64, dtype=bf), q_lens=ints(1), q_offsets=ints(2),
                k_pages=torch.zeros(5, 2, 16, 64, dtype=i8), v_pages=torch.zeros(5, 2, 16, 64, dtype=i8), page_table=ints(1, 4), ctx_lens=ints(1),
                cos_sin=torch.zeros(8, 64), max_q_len=3, k_scale=torch.zeros(5, 2), v_scale=torch.zeros(5, 2))
    bad = [dict(k_scale=torch.zeros(5)), dict(v_scale=torch.zeros(4, 2)), dict(cos_sin=torch.zeros(8, 64, dtype=bf)), dict(cos_sin=torch.zeros(64)),
           dict(positions=ints(2, 4)), dict(positions=ints(2, 3)), dict(positions=torch.zeros(3, dtype=torch.int64)), dict(pair_axes=[0] * 31),
           dict(k_new=torch.zeros(3, 4, 64, dtype=bf)[:, ::2]), dict(q=torch.zeros(3, 64, 4, dtype=bf).transpose(1, 2)), dict(q=torch.zeros(2, 4, 64, dtype=bf)),
           dict(v_new=torch.zeros(3, 2, 64)), dict(q_out=torch.zeros(3, 4, 64)), dict(q=None, q_out=torch.zeros(3, 4, 64, dtype=bf)),
           dict(k_pages=torch.zeros(5, 4, 16, 64, dtype=i8)), dict(page_table=ints(4, 2).T)]
    for change in bad:
        args = dict(base, **change)
        with pytest.raises((ValueError, TypeError)):
            B.kv_write_rope(*(args.pop(n) for n in ("q", "k_new", "v_new", "q_lens", "q_offsets", "k_pages", "v_pages", "page_table", "ctx_lens")), **args,
                            stream=0)
    with pytest.raises(ValueError):
        B.make_desc(base["q"], base["k_pages"], base["page_table"], sm_scale=1.0, k_scale=torch.zeros(5), v_scale=torch.zeros(5))


@pytest.mark.parametrize("name", ["q", "k_new", "v_new"])
def test_one_row_for_all_tokens_is_refused(name):
    """A step of zero between tokens means dense rows to the library, which would read past an expanded row."""
    bf = torch.bfloat16
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    rows = {n: torch.zeros(3, h, 64, dtype=bf) for n, h in (("q", 4), ("k_new", 2), ("v_new", 2))}
    rows[name] = rows[name][:1].expand(3, -1, -1)
    with pytest.raises(ValueError, match="overlap"):
        B.kv_write_rope(*rows.values(), ints(1), ints(2), torch.zeros(5, 2, 16, 64, dtype=bf), torch.zeros(5, 2, 16, 64, dtype=bf), ints(1, 4), ints(1),
                        cos_sin=torch.zeros(8, 64), max_q_len=3, stream=0)


def test_decode_refuses_what_the_library_cannot_see():
    bf = torch.bfloat16
    base = dict(q=torch.zeros(3, 4, 64, dtype=bf), k_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8), v_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8),
                page_table=torch.zeros(3, 4, dtype=torch.int32), ctx_lens=torch.zeros(3, dtype=torch.int32), sm_scale=0.1, k_scale=torch.zeros(5, 2),
                v_scale=torch.zeros(5, 2), out=torch.zeros(3, 4, 64, dtype=bf), workspace=torch.zeros(16, dtype=torch.uint8))
    bad = [dict(q=torch.zeros(3, 64, 4, dtype=bf).transpose(1, 2)), dict(out=torch.zeros(4, 3, 64, dtype=bf).transpose(0, 1)), dict(q=torch.zeros(3, 4, 64, dtype=torch.float64)),
           dict(k_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int16)), dict(page_table=torch.zeros(4, 3, dtype=torch.int32).T), dict(k_scale=torch.zeros(5)),
           dict(k_pages=torch.zeros(5, 2, 64, dtype=torch.int8)), dict(ctx_lens=[1, 2, 3]), dict(sm_scale="0.1"), dict(workspace=None, k_scale=torch.zeros(4, 2))]
    for change in bad:
        with pytest.raises((ValueError, TypeError)):
            B.attn_decode(**dict(base, **change), stream=0)
    with pytest.raises(B.RollattnError) as e:                       # what the library says comes back as it is
        B.attn_decode(**base, stream=0)
    assert e.value.status == -5                                     # 16 bytes of workspace
    assert B.attn_decode(**dict(base, q=base["q"][:0], page_table=base["page_table"][:0], ctx_lens=base["ctx_lens"][:0], out=base["out"][:0]), stream=0).shape == (0, 4, 64)


def test_append_refuses_what_the_library_cannot_see():
    bf = torch.bfloat16
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    base = dict(q_chunk=torch.zeros(6, 4, 64, dtype=bf), q_lens=ints(3), q_offsets=ints(4), k_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8),
                v_pages=torch.zeros(5, 2, 16, 64, dtype=torch.int8), page_table=ints(3, 4), ctx_lens=ints(3), sm_scale=0.1, max_q_len=4, k_scale=torch.zeros(5, 2),
                v_scale=torch.zeros(5, 2), out=torch.zeros(6, 4, 64, dtype=bf), workspace=torch.zeros(16, dtype=torch.uint8))
    bad = [dict(q_chunk=torch.zeros(6, 64, 4, dtype=bf).transpose(1, 2)), dict(q_lens=ints(6)[::2]), dict(v_pages=torch.zeros(5, 16, 2, 64, dtype=torch.int8).transpose(1, 2)),
           dict(q_chunk=torch.zeros(6, 4, 64, dtype=torch.int64)), dict(v_scale=torch.zeros(5)), dict(page_table=ints(12)), dict(ctx_lens=None), dict(max_q_len=1 << 40),
           dict(max_q_len=None), dict(workspace=None, v_scale=torch.zeros(4, 2))]
    for change in bad:
        with pytest.raises((ValueError, TypeError)):
            B.attn_append(**dict(base, **change), stream=0)
    with pytest.raises(B.RollattnError) as e:
        B.attn_append(**base, stream=0)
    assert e.value.status == -5
    none = dict(base, q_chunk=base["q_chunk"][:0], out=base["out"][:0])
    assert B.attn_append(**none, stream=0).shape == (0, 4, 64)

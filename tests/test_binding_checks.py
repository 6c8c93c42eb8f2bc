"""What the binding refuses of its tensors' types and sizes, before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2512_22560_amd import binding as B

bf = torch.bfloat16
ints = lambda *s: torch.zeros(s, dtype=torch.int32)
CODES = [torch.int8, torch.uint8, torch.float8_e4m3fn]


def pool(dtype, hkv=2):
    return torch.zeros(5, hkv, 16, 64, dtype=torch.uint8).view(dtype)


def calls(dtype, **change):
    """The calls of every step with pools of that type, as functions, and some argument of theirs changed."""
    scales = dict(k_scale=torch.zeros(5, 2), v_scale=torch.zeros(5, 2))
    pools = dict(k_pages=pool(dtype), v_pages=pool(dtype), page_table=ints(3, 4), ctx_lens=ints(3), **scales)
    room = dict(workspace=torch.zeros(16, dtype=torch.uint8), sm_scale=0.1, stream=0)          # (too little: nothing could be launched)
    chunk = dict(q_lens=ints(3), q_offsets=ints(4))
    args = {
        "attn_decode": dict(q=torch.zeros(3, 4, 64, dtype=bf), out=torch.zeros(3, 4, 64, dtype=bf), **pools, **room),
        "attn_append": dict(q_chunk=torch.zeros(6, 4, 64, dtype=bf), out=torch.zeros(6, 4, 64, dtype=bf), max_q_len=4, **chunk, **pools, **room),
        "kv_write_rope": dict(q=torch.zeros(6, 4, 64, dtype=bf), k_new=torch.zeros(6, 2, 64, dtype=bf), v_new=torch.zeros(6, 2, 64, dtype=bf), cos_sin=torch.zeros(8, 64),
                              max_q_len=4, stream=0, **chunk, **pools),
    }
    for name, a in args.items():
        if set(change) <= set(a):
            yield name, dict(a, **change)


def refused(dtype, **change):
    seen = 0
    for name, a in calls(dtype, **change):
        seen += 1
        with pytest.raises((ValueError, TypeError)):
            getattr(B, name)(**a)
    return seen


@pytest.mark.parametrize("dtype", CODES)
def test_scales_of_both_pools_are_looked_at(dtype):
    page, head = torch.zeros(5), torch.zeros(5, 2)
    for k, v in ((page, head), (head, page), (head.half(), head.half()), (page.half(), page.half()), (head, head.to(torch.float64)), (torch.zeros(4), torch.zeros(4)),
                 (page, torch.zeros(4)), (torch.zeros(2, 5), torch.zeros(2, 5)), (torch.zeros(5, 3), torch.zeros(5, 3))):
        assert refused(dtype, k_scale=k, v_scale=v) == 3
        with pytest.raises((ValueError, TypeError)):
            B.make_desc(torch.zeros(3, 4, 64, dtype=bf), pool(dtype), ints(3, 4), sm_scale=1.0, k_scale=k, v_scale=v)


def test_scales_that_are_taken():
    q, one = torch.zeros(3, 4, 64, dtype=bf), lambda *s: torch.zeros(s)
    kind = lambda dtype, hkv, k, v: B.make_desc(q, pool(dtype, hkv), ints(3, 4), sm_scale=1.0, k_scale=k, v_scale=v).kv_dtype
    for dtype in CODES[1:]:
        assert kind(dtype, 2, one(5), one(5)) == kind(dtype, 2, one(5, 1), one(5)) == kind(dtype, 2, one(1, 5), one(5, 1)) == kind(dtype, 2, one(7), one(6)) == B.FP8_E4M3
        assert kind(dtype, 2, one(5, 2), one(5, 2)) == kind(dtype, 1, one(5, 1), one(5, 1)) == B.FP8_E4M3_HEAD
        assert kind(dtype, 2, None, None) == B.FP8_E4M3
    assert kind(torch.int8, 2, one(5, 2), one(5, 2)) == kind(torch.int8, 1, one(5, 1), one(5, 1)) == B.INT8_HEAD


@pytest.mark.parametrize("dtype", CODES)
def test_lengths_tables_and_rows_are_looked_at(dtype):
    long = lambda *s: torch.zeros(s, dtype=torch.int64)
    for name, least, n in (("ctx_lens", 3, 3), ("q_lens", 3, 2), ("q_offsets", 4, 2)):
        for bad in (long(least), ints(least - 1), torch.zeros(least), torch.zeros(least, dtype=torch.int16)):
            assert refused(dtype, **{name: bad}) == n
    for bad in (long(3, 4), torch.zeros(3, 4), ints(12)):
        assert refused(dtype, page_table=bad) == 3
    assert refused(dtype, page_table=ints(4, 4)) == 3                                          # more trajectories than lengths, offsets and rows
    other = torch.bfloat16
    for bad in (pool(dtype, 4), pool(dtype)[:4], pool(dtype, 4).view(5, 2, 32, 64), torch.zeros(5, 2, 16, 64, dtype=other)):
        assert refused(dtype, v_pages=bad) == 3
    for name, shape in (("attn_decode", (3, 4, 64)), ("attn_append", (6, 4, 64))):
        rows = "q" if name == "attn_decode" else "q_chunk"
        for bad in ({"out": torch.zeros(shape)}, {"out": torch.zeros(shape, dtype=bf)[:-1]}, {"out": torch.zeros(shape, dtype=torch.int16)},
                    {rows: torch.zeros(shape[0], 4, 32, dtype=bf), "out": torch.zeros(shape[0], 4, 32, dtype=bf)}):
            (_, args), = ((n, a) for n, a in calls(dtype) if n == name)
            with pytest.raises((ValueError, TypeError)):
                getattr(B, name)(**dict(args, **bad))
    for _, args in calls(dtype, q=torch.zeros(2, 4, 64, dtype=bf), out=torch.zeros(2, 4, 64, dtype=bf)):
        with pytest.raises(ValueError):
            B.attn_decode(**args)


@pytest.mark.parametrize("dtype", CODES)
def test_buffers_that_are_larger_are_taken(dtype):
    """Lengths and offsets of a longer batch, more rows of output, a workspace of any type: what the library says of that is all that is wrong."""
    for name, args in calls(dtype, ctx_lens=ints(9)):
        if "out" in args:
            args.update(out=torch.zeros(9, 4, 64, dtype=bf))
        if "q_lens" in args:
            args.update(q_lens=ints(8), q_offsets=ints(9))
        if name == "kv_write_rope":
            continue
        for room, status in ((torch.zeros(16, dtype=torch.uint8), -5), (torch.zeros(4), -5)):
            with pytest.raises(B.RollattnError) as e:
                getattr(B, name)(**dict(args, workspace=room))
            assert e.value.status == status

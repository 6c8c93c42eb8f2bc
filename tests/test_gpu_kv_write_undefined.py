"""Undefined elements in rows on their way into 8-bit pools through the rotating write, and through the plain write into pools with a
scale for each page and head: they count for no scale and become the lowest code.  Bit for bit, so there is no tolerance."""
import pytest
import torch

from paper_2512_22560_amd import binding as B
from tests.test_gpu_kv_write_rope import DEV, batch_of, both, rows_of, same, table_of

pytestmark = pytest.mark.gpu
LOWEST = {"fp8_e4m3": 0xFE, "fp8_e4m3_head": 0xFE, "int8_head": 0x81}


@pytest.mark.parametrize("mag", [1.0, 2.0 ** -40])
@pytest.mark.parametrize("prefix,new", [(0, 1), (7, 1), (0, 5), (9, 30)])
@pytest.mark.parametrize("kv,plain", [("fp8_e4m3", False), ("fp8_e4m3_head", False), ("int8_head", False), ("fp8_e4m3_head", True), ("int8_head", True)])
def test_undefined_elements_count_for_no_scale(kv, plain, prefix, new, mag):
    """Quiet and signalling ones of either sign, next to the largest element of their row, in the same lane's eight and in others, and
    alone in it; keys only in dims that are not rotated (a rotation quiets, and takes the partner along)."""
    b = batch_of("t", (8, 6), 128, "bf16", kv, ("const", prefix), ("const", new), 31, batch=3)
    gen = torch.Generator().manual_seed(32)
    spots = {(0, 0, 67): 0x7F81, (0, 1, 64): 0xFF81, (0, 2, 127): 0x7FC0, (new, 3, 90): 0xFFC0, (new, 4, 71): 0x7FBF, (2 * new, 0, 100): 0xFFBF, (2 * new, 5, 65): 0x7F81}
    zeroed, rows = [], []
    for i in range(2):
        x = rows_of(gen, b.total_q, 6, 128, "bf16", mag).contiguous()
        for token, head, at in spots:
            x[token, head, at - 1 if at % 8 else at + 1] = 60.0 * mag        # the largest of the head in its page, beside an undefined one
        x[2 * new, 5] = 0                                                   # nothing else in the row
        zeros = x.clone()
        for at, pattern in spots.items():
            x.view(torch.int16)[at] = pattern - ((pattern & 0x8000) << 1)
            zeros[at] = 0.0
        assert [int(x.view(torch.int16)[at]) & 0xFFFF for at in spots] == list(spots.values())
        rows.append(x)
        zeroed.append(zeros)
    table = table_of(64, 64)
    pools = lambda: tuple(t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
    got = pools()
    args = (b.q_lens, b.q_offsets, got[0], got[1], b.page_table, b.ctx_lens)
    scales = dict(k_scale=got[2], v_scale=got[3])
    if plain:
        B.kv_write(*rows, *args, max_q_len=new, **scales)
        want = pools()
        B.kv_write(*zeroed, b.q_lens, b.q_offsets, want[0], want[1], b.page_table, b.ctx_lens, max_q_len=new, k_scale=want[2], v_scale=want[3])
    else:
        B.kv_write_rope(None, *rows, *args, cos_sin=table, max_q_len=new, **scales)
        (_, *want), ref = both(b, None, *zeroed, table)
        same((None, *want), ref, "zeros in their place")
    for g, z in zip(got[2:], want[2:]):
        assert torch.equal(g.view(torch.int32), z.view(torch.int32))
    for g, z in zip(got[:2], want[:2]):
        differ = g.view(torch.uint8) != z.view(torch.uint8)
        assert int(differ.sum()) == len(spots)
        assert bool((g.view(torch.uint8)[differ] == LOWEST[kv]).all())

"""Undefined and infinite elements in rows that are normalised on their way into the pools.  An undefined element makes its head's mean, and so
the whole row of that head, undefined; an infinite one makes the row's factor zero and itself undefined (infinity times zero) with the element
it is turned with.  Over 8-bit pools undefined elements count for no scale and become the lowest code, as in the rotating write: everything else
is what it is with zeros in the row's place, whose norm is zero.  Bit for bit, but for the sign of a zero, so there is no tolerance."""
import pytest
import torch

from paper_2512_22560_amd import binding as B
from tests.test_gpu_kv_write_norm_rope import DEV, rows_of, table_of, weights
from tests.tree_common import KINDS, drafts

pytestmark = pytest.mark.gpu
LOWEST = {"fp8_e4m3": 0xFE, "fp8_e4m3_head": 0xFE, "int8_head": 0x81}


@pytest.mark.parametrize("kind", ["undefined", "infinite"])
@pytest.mark.parametrize("prefix,new", [(0, 1), (7, 1), (0, 5), (9, 30)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS)
def test_rows_with_elements_that_are_no_numbers(src, kv, d, prefix, new, kind):
    b = drafts((12, 6), d, src, kv, ("const", prefix), ("const", new), 31, batch=3)
    gen = torch.Generator().manual_seed(32)
    q, k, v = (rows_of(gen, b.total_q, h, d, src) for h in (12, 6, 6))
    qw, kw = weights(gen, d)
    table = table_of(64, d)
    spots = [(0, 0, 3), (0, 5, d - 1), (new, 1, d // 2), (2 * new, 4, 0), (3 * new - 1, 2, d // 2 - 1)]      # row, head, dim
    zeros = [t.clone() for t in (q, k)]
    for row, head, dim in spots:
        for t, z, h in ((q, zeros[0], head + 2), (k, zeros[1], head)):
            t[row, h, dim] = float("nan") if kind == "undefined" else (float("inf") if dim % 2 else -float("inf"))
            z[row, h] = 0
    runs = []
    for rows in ((q, k), zeros):
        pools = tuple(None if t is None else t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale))
        out = B.kv_write_norm_rope(*rows, v, b.q_lens, b.q_offsets, pools[0], pools[1], b.page_table, b.ctx_lens, q_weight=qw, k_weight=kw, eps=1e-6, cos_sin=table,
                                   max_q_len=new, k_scale=pools[2], v_scale=pools[3])
        runs.append((out, *pools))
    got, want = runs
    # where something undefined has to be: [rows, heads, D]
    marks = {"q": torch.zeros(q.shape, dtype=torch.bool), "k": torch.zeros(k.shape, dtype=torch.bool)}
    for row, head, dim in spots:
        dims = slice(None) if kind == "undefined" else [dim, (dim + d // 2) % d]
        marks["q"][row, head + 2, dims] = True
        marks["k"][row, head, dims] = True
    there = marks["q"].to(DEV)
    assert torch.equal(torch.isnan(got[0]), there) and torch.equal(got[0][~there], want[0][~there])
    there = torch.zeros(b.k_pages.shape, dtype=torch.bool)
    for t in range(3):
        for i in range(new):
            at = prefix + i
            there[int(b.page_table[t, at // 16]), :, at % 16] = marks["k"][t * new + i]
    there = there.to(DEV)
    bits = lambda x: x.view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[x.element_size()])

    def same(x, y):
        if kv.startswith("fp8"):                      # (the code of a negative zero)
            x, y = (torch.where(t == 0x80, 0, t) for t in (x, y))
        return torch.equal(x, y)

    # (places that no token has hold undefined values)
    live = torch.zeros(b.k_pages.shape, dtype=torch.bool)
    for t in range(3):
        for at in range(prefix + new):
            live[int(b.page_table[t, at // 16]), :, at % 16] = True
    live = live.to(DEV)
    assert same(got[1][live & ~there], want[1][live & ~there]) and torch.equal(bits(got[1])[~live], bits(want[1])[~live]) and torch.equal(bits(got[2]), bits(want[2]))
    if kv in LOWEST:
        assert (bits(got[1])[there] == LOWEST[kv]).all()
        assert torch.equal(bits(got[3]), bits(want[3])) and torch.equal(bits(got[4]), bits(want[4]))
    else:
        assert torch.isnan(got[1][there]).all()

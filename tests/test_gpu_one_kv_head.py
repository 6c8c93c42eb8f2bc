"""E4M3 pools of one KV head whose scales are shaped [num_pages, 1]: a page and its head are the same."""
import pytest
import torch

from paper_2512_22560_amd import binding as B
from tests.test_gpu_kv_write_rope import batch_of, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 40])
def test_the_plain_write_follows_the_rule_of_pages(new):
    """The bytes and scales that scales [num_pages] get: pages of zeros have the scale 1, and faint ones that of their magnitude."""
    b = batch_of("t", (8, 1), 64, "bf16", "fp8_e4m3", ("const", 0), ("const", new), 61, batch=6)
    gen = torch.Generator().manual_seed(62)
    k, v = rows_of(gen, b.total_q, 1, 64, "bf16"), rows_of(gen, b.total_q, 1, 64, "bf16")
    k[: 2 * new] = 0
    v[3 * new:5 * new] = 0
    v[:new] *= 2.0 ** -80
    got, flat = ([t.clone() for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale)] for _ in range(2))
    for i, shape in ((got, (-1, 1)), (flat, (-1,))):
        B.kv_write(k, v, b.q_lens, b.q_offsets, i[0], i[1], b.page_table, b.ctx_lens, max_q_len=new, k_scale=i[2].view(shape), v_scale=i[3].view(shape))
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, flat))
    first = b.page_table[:, 0].long()
    assert (got[2][first[:2]] == 1).all() and (got[3][first[3:5]] == 1).all() and 0 < float(got[3][first[0]]) < 2.0 ** -64

"""attn_tree with one workspace for all steps, made for the largest of them: shorter drafts, fewer rows, fewer trajectories.  The same kernels
run, so results are those of a workspace of the step's own, bit for bit."""
import pytest
import torch

from paper_2512_22560_amd import binding as B
from tests.test_gpu_tree import call
from tests.test_gpu_tree_cut import widened
from tests.tree_common import KINDS, any_masks

pytestmark = pytest.mark.gpu
HEADS = ((64, 4), (32, 8), (8, 8))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kv", KINDS)
def test_smaller_steps_in_the_largest_ones_workspace(src, kv, d):
    for heads in HEADS:
        steps = [widened(heads, d, src, kv, ("uniform", 0, 900), ("uniform", 1, most), 100 + most, batch=batch)
                 for most, batch in ((72, 12), (20, 12), (9, 12), (8, 12), (4, 12), (2, 12), (1, 12), (72, 3), (4, 1), (1, 1))]
        room = B.alloc_tree_workspace(steps[0].q, steps[0].k_pages, steps[0].v_pages, steps[0].page_table, steps[0].ctx_lens, max_q_len=72,
                                      k_scale=steps[0].k_scale, v_scale=steps[0].v_scale)
        room.fill_(0xA5)
        for b in steps:
            mask = any_masks(b, 1)
            got, alone = call(b, mask, workspace=room), call(b, mask)
            assert torch.equal(got, alone) and torch.isfinite(got).all(), (heads, int(b.q_lens_host.max()), len(b.q_lens_host))

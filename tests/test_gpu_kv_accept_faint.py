"""Rows of E4M3 pages whose scale is subnormal, where a code times its scale keeps few of its bits: accepted rows as defined, bit for bit."""
import pytest
import torch

from tests.test_gpu_kv_accept import DEV, check, some
from tests.tree_common import drafts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low,high", [(-141, -141), (-149, -149), (-149, -140), (-130, -120)])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_of_subnormal_scales(d, low, high):
    b = drafts((4, 4), d, "bf16", "fp8_e4m3", ("uniform", 0, 40), ("uniform", 20, 90), 61)
    gen = torch.Generator().manual_seed(low - high)
    for s in (b.k_scale, b.v_scale):
        s.copy_(torch.exp2(torch.randint(low, high + 1, s.shape, generator=gen).float()).to(DEV))
    for seed in range(3):
        check(b, *some(b, seed), f"{seed}")

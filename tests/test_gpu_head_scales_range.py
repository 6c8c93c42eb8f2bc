"""Queries of any magnitude over 8-bit pools with a scale for each page and KV head.  The bound is that of tests/test_gpu_head_scales.py."""
import pytest
import torch

from tests.test_gpu_head_scales import KV, build, call, check

pytestmark = pytest.mark.gpu
# (32 rows of a wave and more; appended chunks on half tiles and on whole ones)
SHAPES = [("decode", ("const", 1)), ("append", ("const", 20)), ("append", ("const", 60))]


def batch(kv, which, qlen, d=128, seed=41):
    return build(kv, (8, 2), d, ("uniform", 100, 400), qlen=qlen, batch=4, seed=seed, prefix=which == "append")


@pytest.mark.parametrize("q_mag", [2.0 ** -70, 2.0 ** -78, 2.0 ** -110, 2.0 ** -130])
@pytest.mark.parametrize("faint_keys", [True, False])
@pytest.mark.parametrize("which,qlen", SHAPES)
@pytest.mark.parametrize("kv", KV)
def test_faint_queries_and_faint_keys_together(kv, which, qlen, faint_keys, q_mag):
    """All scores are next to nothing: outputs are means of the visible values."""
    b = batch(kv, which, qlen, d=128 if q_mag < 2.0 ** -100 else 64)
    b.q = (b.q.float() * q_mag).to(torch.bfloat16)
    if faint_keys:
        b.k_scale.fill_(2.0 ** -64)                       # the least that a write leaves
    check(call(b, which), b, which)

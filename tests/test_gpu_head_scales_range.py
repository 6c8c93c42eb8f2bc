"""Queries of any magnitude over 8-bit pools with a scale for each page and KV head: faint ones over faint keys, rows of very
different magnitudes side by side, scores past what float32 resolves.

The bound is that of tests/test_gpu_head_scales.py, with one more term where appended queries meet E4M3 keys.  There a query is
the sum of two E4M3 numbers, under a power of two that puts its row's largest element between 2^7 and 2^8.  The nearest E4M3 number
leaves at most 2^-4 of an element, on the element's own grid of eight bits; that rest is exact unless it needs a step below E4M3's
least, 2^-9, and then off by at most 2^-10: 2^-17 of the row's largest element.  A score is off by at most d = sm_scale * 2^-17 * max|q| *
sum|k|, so a weight by the factor exp(2 d), and an output by exp(2 d) - 1 of the weighted sum of |v|."""
import numpy as np
import pytest
import torch

from oracle import attention as O
from tests.helpers import oracle_args
from tests.test_gpu_head_scales import DEV, KV, SCORE_ROOM, build, call, check, oracle

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


def key_sums(b):
    """The largest sum of a key's magnitudes, for every trajectory and query head."""
    w, a = b.workload, oracle_args(b)
    top = np.array([[np.abs(O.gather_tokens(a["k_pages"], a["page_table"], i, g, int(n), w.kv_dtype, a["k_scale"])).sum(1).max(initial=0.0)
                     for g in range(w.num_kv_heads)] for i, n in enumerate(b.ctx_lens_host)])
    return np.repeat(top, w.num_q_heads // w.num_kv_heads, axis=1)


@pytest.mark.parametrize("which,qlen", SHAPES)
@pytest.mark.parametrize("kv", KV)
def test_ordinary_rows_next_to_loud_ones(kv, which, qlen):
    """Heads and tokens of the same wave 2^4 .. 2^24 times as loud, and stray finite rows of 1e30."""
    b = batch(kv, which, qlen, seed=42)
    rng = np.random.default_rng(43)
    power = rng.choice([0, 0, 0, 4, 12, 18, 24, 100], size=b.q.shape[:2]).astype(np.float32)
    b.q = (b.q.float() * torch.exp2(torch.from_numpy(power).to(DEV))[:, :, None]).to(torch.bfloat16)
    got = call(b, which).double().cpu().numpy()
    ref, room = oracle(b, which), oracle(b, which, True)
    extra = 0.0
    if kv == "fp8_e4m3_head" and which == "append":
        loudest = b.q.float().abs().amax(dim=2).double().cpu().numpy()
        off = b.workload.sm_scale * 2.0 ** -17 * loudest * np.repeat(key_sums(b), b.q_lens_host, axis=0)
        extra = np.expm1(2 * np.where(power == 0, off, 0.0))[:, :, None]
    bound = (2.0 ** -8) * np.abs(ref) + (2.0 ** -11 + SCORE_ROOM + extra) * room + 1e-30
    ordinary = power == 0
    assert np.isfinite(got[ordinary]).all()
    worst = float((np.abs(got - ref) / bound)[ordinary].max())
    assert worst <= 1.0, f"{worst:.2f} times the bound"


@pytest.mark.parametrize("power", [22, 23, 24, 25, 26, 27, 28, 40, 96])
@pytest.mark.parametrize("which,qlen", SHAPES)
@pytest.mark.parametrize("kv", KV)
def test_scores_past_what_float32_resolves(kv, which, qlen, power):
    """Which of the largest scores' tokens win is a matter of rounding there, but an output stays a mean of values."""
    b = batch(kv, which, qlen, seed=44)
    b.q = (b.q.float() * 2.0 ** power).to(torch.bfloat16)
    got = call(b, which).float()
    a = oracle_args(b)
    most = max(np.abs(O.gather_tokens(a["v_pages"], a["page_table"], i, g, int(n), kv, a["v_scale"])).max() for i, n in enumerate(b.ctx_lens_host) for g in range(2))
    assert torch.isfinite(got).all() and float(got.abs().max()) <= most * (1 + 2.0 ** -7)


@pytest.mark.parametrize("ends", [("v", 36), ("v", 20), ("k", 100)])
@pytest.mark.parametrize("which,qlen", SHAPES)
@pytest.mark.parametrize("kv", KV)
def test_scales_at_both_ends_of_their_range(kv, which, qlen, ends):
    """Every other page has the least scale that a write leaves, as a page of zeros does.  Its values are next to nothing beside the other
    pages', but its tokens take their part of the weights; its keys leave the scores at nothing."""
    b = batch(kv, which, qlen, seed=45)
    least = (torch.arange(b.k_scale.shape[0], device=DEV) % 2 == 0)[:, None]
    name, top = ends
    scale = getattr(b, name + "_scale")
    scale.copy_(torch.where(least, torch.full_like(scale, 2.0 ** -64), torch.full_like(scale, 2.0 ** top)))
    if name == "k":
        b.q = (b.q.float() * 2.0 ** -110).to(torch.bfloat16)
    check(call(b, which), b, which)

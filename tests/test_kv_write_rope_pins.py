"""Pins of the oracle of the rotating KV write (CPU): closed forms, invariants of the rotation, and the older oracles wherever
the two define the same thing."""
import numpy as np
import pytest

from oracle import attention as A
from oracle import kv_write as KW
from oracle import kv_write_rope as R


def _table(n, rot, base=100.0):
    j = np.arange(rot // 2)
    angle = np.arange(n)[:, None] * base ** (-2.0 * j / rot)
    return np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32), angle


def _batch(rng, ctx, n, hkv, d, kv_dtype, hq=0):
    ctx, n = np.asarray(ctx), np.asarray(n)
    pages = -(-ctx // 16)
    perm = rng.permutation(int(pages.sum()) + 2).astype(np.int32)
    table = np.full((len(ctx), max(1, int(pages.max()))), -1, dtype=np.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = perm[at:at + p]
        at += p
    t = int(n.sum())
    f = lambda h: rng.standard_normal((t, h, d)).astype(np.float32)
    shape = (len(perm), hkv, 16, d)
    pool = {"f32": lambda: rng.standard_normal(shape).astype(np.float32), "bf16": lambda: R.float32_to_bf16(rng.standard_normal(shape)),
            "int8_head": lambda: rng.integers(-127, 128, shape).astype(np.int8)}.get(
                kv_dtype, lambda: KW.float32_to_e4m3fn(100 * rng.standard_normal(shape)))
    sshape = shape[:2] if kv_dtype.endswith("_head") else shape[:1]
    scale = lambda: (0.01 * (1 + rng.random(sshape))).astype(np.float32)
    return dict(q=f(hq) if hq else None, k_new=f(hkv), v_new=f(hkv), q_lens=n, ctx_lens=ctx, page_table=table, k_pages=pool(), v_pages=pool()), \
        dict(k_scale=scale(), v_scale=scale()) if kv_dtype not in ("f32", "bf16") else {}


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_pair_is_a_complex_number_times_a_unit(interleaved):
    rng = np.random.default_rng(0)
    table, angle = _table(50, 12)
    x = rng.standard_normal((7, 3, 20)).astype(np.float32)
    at = rng.integers(0, 50, 7)
    y = R.rotate(x, np.repeat(at[:, None], 6, axis=1), table, interleaved)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    z = x[..., 0:12:2] + 1j * x[..., 1:12:2] if interleaved else x[..., :6] + 1j * x[..., 6:12]
    w = y[..., 0:12:2] + 1j * y[..., 1:12:2] if interleaved else y[..., :6] + 1j * y[..., 6:12]
    assert np.abs(w - z * np.exp(1j * angle[at])[:, None, :]).max() < 1e-5


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    table, _ = _table(200, 16)
    q, k = rng.standard_normal((2, 1, 1, 16)).astype(np.float32)
    dot = lambda a, b: float((R.rotate(q, [[a] * 8], table) * R.rotate(k, [[b] * 8], table)).sum())
    assert abs(dot(7, 3) - dot(150, 146)) < 1e-4 < abs(dot(7, 3) - dot(150, 140))


def test_each_pair_follows_its_axis():
    rng = np.random.default_rng(2)
    table, _ = _table(64, 12)
    args, _ = _batch(rng, [20, 9], [20, 5], 2, 16, "f32", hq=4)
    t = 25
    axes = [0, 0, 1, 1, 2, 2]
    positions = rng.integers(0, 64, (3, t))
    write = lambda p, a: R.kv_write_rope(**args, src_dtype="f32", kv_dtype="f32", cos_sin=table, positions=p, pair_axes=a)[0]
    q = write(positions, axes)
    for pair, axis in enumerate(axes):
        alone = write(positions[axis], None)
        for dim in (pair, pair + 6):
            assert np.array_equal(q[..., dim], alone[..., dim])
    place = np.concatenate([np.arange(0, 20), np.arange(4, 9)])
    plain = R.kv_write_rope(**args, src_dtype="f32", kv_dtype="f32", cos_sin=table)
    assert np.array_equal(plain[0], write(place, None)) and np.array_equal(plain[0], write(np.stack([place] * 3), axes))
    beyond = place.copy()
    beyond[3], beyond[7] = 64, -1                       # past either end: the last row
    last = place.copy()
    last[[3, 7]] = 63
    assert np.array_equal(write(beyond, None), write(last, None))


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8_e4m3"])
def test_without_a_turn_it_is_kv_write(kv):
    rng = np.random.default_rng(3)
    args, scales = _batch(rng, [5, 33, 40, 16], [5, 17, 1, 0], 3, 8, kv)
    src = "f32" if kv == "f32" else "bf16"
    if src == "bf16":
        args["k_new"], args["v_new"] = R.float32_to_bf16(args["k_new"]), R.float32_to_bf16(args["v_new"])
    still = np.concatenate([np.ones((64, 4)), np.zeros((64, 4))], axis=1).astype(np.float32)
    old = {k: v for k, v in args.items() if k != "q"}
    want = KW.kv_write(**old, src_dtype=src, kv_dtype=kv, **scales)
    for table in (None, still):
        got = R.kv_write_rope(**args, src_dtype=src, kv_dtype=kv, cos_sin=table, **scales)[1:]
        for a, b in zip(got, want):
            assert (a is None and b is None) or np.array_equal(a, b)


@pytest.mark.parametrize("kv", ["fp8_e4m3_head", "int8_head"])
def test_a_head_with_its_own_scale_is_a_pool_of_one_head(kv):
    """Each head of a pool with scales for heads is what a pool of that head alone holds; E4M3 codes by the older rule."""
    rng = np.random.default_rng(4)
    args, scales = _batch(rng, [5, 33, 40, 16, 1], [5, 17, 1, 0, 1], 3, 8, kv)
    args["k_new"] = R.float32_to_bf16(args["k_new"] * np.array([0.1, 1, 30])[None, :, None])
    args["v_new"] = R.float32_to_bf16(args["v_new"])
    _, kp, vp, ks, vs = R.kv_write_rope(**args, src_dtype="bf16", kv_dtype=kv, **scales)
    for h in range(3):
        one = dict(args, **{n: args[n][:, h:h + 1] for n in ("k_new", "v_new", "k_pages", "v_pages")})
        if kv == "int8_head":
            got = R.kv_write_rope(**one, src_dtype="bf16", kv_dtype=kv, **{n: s[:, h:h + 1] for n, s in scales.items()})[1:]
        else:
            one.pop("q")
            got = KW.kv_write(**one, src_dtype="bf16", kv_dtype="fp8_e4m3", **{n: s[:, h] for n, s in scales.items()})
        assert np.array_equal(kp[:, h:h + 1], got[0]) and np.array_equal(vp[:, h:h + 1], got[1])
        assert np.array_equal(ks[:, h], got[2].reshape(-1)) and np.array_equal(vs[:, h], got[3].reshape(-1))


@pytest.mark.parametrize("kv,step", [("int8_head", 0.5 / 127), ("fp8_e4m3_head", 2.0 ** -4)])
def test_what_is_read_back_is_within_half_a_step(kv, step):
    rng = np.random.default_rng(5)
    args, scales = _batch(rng, [48], [48], 2, 16, kv)
    args["k_new"] *= np.exp(rng.standard_normal((48, 1, 1)))
    x = R.float32_to_bf16(args["k_new"])
    args["k_new"], args["v_new"] = x, x
    _, kp, vp, ks, vs = R.kv_write_rope(**args, src_dtype="bf16", kv_dtype=kv, **scales)
    assert np.array_equal(kp[args["page_table"][0]], vp[args["page_table"][0]])
    for h in range(2):
        got = A.gather_tokens(kp, args["page_table"], 0, h, 48, kv, ks)
        want = KW._to_float32(x, "bf16").astype(np.float64)[:, h]
        amax = np.abs(want.reshape(3, -1)).max(axis=1).repeat(16)[:, None]
        room = step * amax if kv == "int8_head" else np.maximum(step * np.abs(want), amax / 448 * 2.0 ** -10)
        assert (np.abs(got - want) <= room * (1 + 1e-6)).all()
        assert np.allclose(ks[args["page_table"][0], h], amax[::16, 0] / (127 if kv == "int8_head" else 448), rtol=1e-6)


def test_scales_grow_and_codes_follow():
    table = np.array([[1]], dtype=np.int32)
    pool = np.zeros((2, 1, 16, 8), dtype=np.int8)
    scale = np.full((2, 1), 7.0, dtype=np.float32)
    rows = lambda v: R.float32_to_bf16(np.full((1, 1, 8), v, dtype=np.float32))
    state = (pool, pool, scale, scale)
    for i, (v, want) in enumerate([(0.0, 2.0 ** -64), (1.0, 1 / 127), (0.25, 1 / 127), (2.0, 2 / 127), (-0.5, 2 / 127)]):
        state = R.kv_write_rope(None, rows(v), rows(v), [1], [i + 1], table, state[0], state[1], src_dtype="bf16", kv_dtype="int8_head",
                                k_scale=state[2], v_scale=state[3])[1:]
        assert state[2][1, 0] == np.float32(want) and state[2][0, 0] == 7.0
    # 0; 127 at the scale of 1, 64 (63.5 to even) at that of 2; 32 (31.75), then 16; 127; -32 (-31.75)
    assert state[0][1, 0, :5, 0].tolist() == [0, 64, 16, 127, -32] and not state[0][0].any()


def test_rounding_to_bf16_is_nearest_even():
    ties = np.array([0x3F808000, 0x3F818000, 0x3F808001, 0x3F807FFF, 0xBF818000], dtype=np.uint32).view(np.float32)
    assert R.float32_to_bf16(ties).tolist() == [0x3F80, 0x3F82, 0x3F81, 0x3F80, 0xBF82]


PLANTED = [
    ("sum and difference swapped", "(lo * c).astype(np.float32) - (hi * s)", "(lo * c).astype(np.float32) + (hi * s)"),
    ("partner of the wrong layout", "second = first + (1 if interleaved else half)", "second = first + (half if interleaved else 1)"),
    ("sines of the neighbouring pair", "t[rows, half + np.arange(half)]", "t[rows, half + (np.arange(half) + 1) % half]"),
    ("positions count from the chunk's start", "np.arange(l - n, l) for", "np.arange(n) for"),
    ("first axis for every pair", "np.atleast_2d(positions)[axes].T", "np.atleast_2d(positions)[axes * 0].T"),
    ("past the table: its first row", "t.shape[0] - 1, rows)", "0, rows)"),
    ("int8 scale as of E4M3", "np.float32(127.0) if int8", "np.float32(448.0) if int8"),
    ("zero rows leave a scale of one", "need = max(need, LEAST)", "need = need or np.float32(1.0)"),
    ("scales never grow", "now = max(old, need)", "now = old"),
    ("old codes stay", "if now > old:", "if False:"),
    ("int8 rounds towards zero", "np.clip(np.rint(x), -127, 127)", "np.clip(np.trunc(x), -127, 127)"),
    ("bf16 ties up", "+ 0x7FFF + ((u >> 16) & 1)", "+ 0x8000"),
    ("the first head's scale for all", "at = (page, i) if per_head", "at = (page, 0) if per_head"),
]


def test_every_planted_mistake_fails_a_pin(tmp_path):
    from tests.test_pins_catch_planted_mistakes import CONTROL, _run
    jobs = [(CONTROL, None, None)] + PLANTED
    import concurrent.futures
    import os
    if os.environ.get("ROPE_PINS_INNER"):
        pytest.skip("this is a copy's own run")
    os.environ["ROPE_PINS_INNER"] = "1"
    try:
        with concurrent.futures.ThreadPoolExecutor(max_workers=6) as pool:
            results = list(pool.map(lambda c: _run(str(tmp_path), "kv_write_rope.py", "tests/test_kv_write_rope_pins.py", *c), jobs))
    finally:
        del os.environ["ROPE_PINS_INNER"]
    assert results[0][1] == 0, results[0][2]
    assert not [n for n, rc, _ in results[1:] if rc != 1]

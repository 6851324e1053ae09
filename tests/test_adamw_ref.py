"""The 8-bit moments as the tests' CPU code forms them: against torch's own e4m3 and e5m2 types, the bounds
of the rounding, and what the thresholds are for."""
import numpy as np
import pytest
import torch

import adamw_ref

TYPES = {"M": torch.float8_e4m3fn, "V": torch.float8_e5m2}


@pytest.mark.parametrize("kind", ["M", "V"])
def test_every_code_is_the_types_value(kind):
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code).view(TYPES[kind]).float().numpy()
    got = adamw_ref.decode(code, np.ones(2, np.float32), kind)
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("kind", ["M", "V"])
@pytest.mark.parametrize("t", [1, 2, 1000, (1 << 24) + 5])
def test_codes_are_a_neighbour_of_the_value(kind, t):
    rng = np.random.default_rng(t)
    man, top, low, _ = adamw_ref.KIND[kind]
    x = (rng.normal(size=1000) * np.exp(rng.normal(size=1000) * 4)).astype(np.float32)
    x = np.abs(x) if kind == "V" else x
    x[:7] = [0, 1e-45, -1e-45 if kind == "M" else 1e-45, 1e-30, 3e-38, 2e-20, 1]
    code, scale = adamw_ref.encode(x, t, kind)
    back = adamw_ref.decode(code, scale, kind).astype(np.float64)
    s = np.repeat(scale.astype(np.float64), 128)[:x.size]
    step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(x) / s, 1e-300))) - man), 2.0 ** (low - man))
    assert (np.abs(back - x) <= step * s).all()
    assert np.isfinite(back).all() and (back[x == 0] == 0).all()


@pytest.mark.parametrize("kind", ["M", "V"])
def test_the_thresholds_lose_nothing_on_average(kind):
    """A value between two codes is on average itself: over 4096 steps to a thousandth of a step (a random
    threshold would leave 1 / 128), within a block of 128 at one step to a tenth."""
    man = adamw_ref.KIND[kind][0]
    x = np.full(128, np.float32(1.0 + 0.3 / 2 ** man))
    x[0] = 1.9
    got = np.mean([adamw_ref.decode(*adamw_ref.encode(x, t, kind), kind)[5] for t in range(1, 4097)])
    assert abs(got - x[5]) < 2.0 ** -man / 1000
    one = adamw_ref.decode(*adamw_ref.encode(x, 77, kind), kind)[1:]
    assert abs(one.mean() - x[5]) < 2.0 ** -man / 10


def test_second_moments_follow_small_changes():
    """With b2 = 0.999 a constant gradient's second moment ends at its square, where rounding to the
    nearest code would leave it as soon as a step adds less than half a code's distance: an eighth."""
    g = np.full(128, np.float32(0.01))
    code, scale = np.zeros(128, np.uint8), np.ones(1, np.float32)
    seen = []
    for t in range(1, 6001):
        v = adamw_ref.decode(code, scale, "V")
        _, v = adamw_ref.moments(g, 1.0, v, v, 0.9, 0.999)
        code, scale = adamw_ref.encode(v, t, "V")
        if t > 5000:
            seen.append(adamw_ref.decode(code, scale, "V").mean())
    assert abs(np.mean(seen) / (g[0] ** 2) - 1) < 0.05


def test_infinities_and_nan_are_stored_as_nan_and_alone():
    x = np.linspace(0.5, 1.5, 130).astype(np.float32)
    want = adamw_ref.encode(x, 9, "M")
    y = x.copy()
    y[3], y[70] = np.inf, np.nan
    code, scale = adamw_ref.encode(y, 9, "M")
    keep = np.ones(130, bool)
    keep[[3, 70]] = False
    assert np.array_equal(code[keep], want[0][keep]) and np.array_equal(scale, want[1])
    assert np.isnan(adamw_ref.decode(code, scale, "M")[[3, 70]]).all()


def trajectory(factor, steps, alike, seed=0, blocks=4):
    """Largest update in units of lr, after a fifth of the steps, of elements that share their block with one whose
    gradients are `factor` times larger: with 8-bit moments and with fp32 ones.  alike: every step has the same
    gradients."""
    rng = np.random.default_rng(seed)
    n = 128 * blocks
    size = np.where(np.arange(n) % 128 == 0, 1e-3 * factor, 1e-3)
    g = rng.normal(size=n) * size
    M, V = np.zeros(n, np.float32), np.zeros(n, np.float32)
    codes = [(np.zeros(n, np.uint8), np.ones(blocks, np.float32))] * 2
    largest = [0.0, 0.0]
    for t in range(1, steps + 1):
        if not alike:
            g = rng.normal(size=n) * size
        G = g.astype(np.float32)
        m, v = adamw_ref.moments(G, 1.0, adamw_ref.decode(*codes[0], "M"), adamw_ref.decode(*codes[1], "V"), 0.9, 0.999)
        codes = [adamw_ref.encode(m, t, "M"), adamw_ref.encode(v, t, "V")]
        M, V = adamw_ref.moments(G, 1.0, M, V, 0.9, 0.999)
        if 5 * t > steps:
            for k, (a, b) in enumerate(((m, v), (M, V))):
                w, _ = adamw_ref.update(np.zeros(n), a, b, 1.0, 0.9, 0.999, 1e-8, t, 0.0)
                largest[k] = max(largest[k], np.abs(w)[np.arange(n) % 128 != 0].max())
    return largest


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("factor", [1.0, 1e4, 3e4, 1e5, 1e6, 1e8])
def test_no_step_explodes_where_gradients_of_a_block_differ(factor, alike):
    """|m| / sqrt(v) is at most k = (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)) = 7.3 for every sequence of gradients.
    The cut of M adds at most one of its smallest codes, 2^-16 of the largest M's power of two, where sqrt(v) is
    at least 2^-15 of the largest V's root: another k / sqrt(2).  Before, V could be zero there: 30000 lr at 3e4."""
    with_codes, plain = trajectory(factor, 1000, alike)
    k = 0.1 / np.sqrt(0.001 * (1 - 0.81 / 0.999))
    assert plain < k and with_codes < k * (1 + 2 ** -0.5)


def test_a_second_moment_that_is_not_zero_is_not_stored_as_zero():
    x = np.zeros(256, np.float32)
    x[0], x[1], x[2:100], x[130] = 1.0, 1e-45, 1e-20, 1e-45
    for t in range(1, 50):
        code, _ = adamw_ref.encode(x, t, "V")
        assert ((code == 0) == (x == 0)).all()
        assert (code[1:100] == 1).all()


@pytest.mark.parametrize("alike", [False, True])
def test_8_bit_moments_beside_fp32_ones(alike):
    """How far they are apart over 750 steps after 750.  A step moves V by about a thousandth of itself, c, where codes lie
    q <= V / 4 apart: it takes the next code with probability c / q, which adds c q to the variance, and loses 2 c of what
    is there, so that it settles at q V / 2: a relative deviation of at most 8^-1/2 = 0.354, half of that for the root.
    M's cut is off by at most q / 6^1/2, q <= M / 8, and 0.81 of its variance stays: 0.117.  Together 0.21 of an update."""
    rng = np.random.default_rng(11)
    n = 512
    M, V = np.zeros(n, np.float32), np.zeros(n, np.float32)
    codes = [(np.zeros(n, np.uint8), np.ones(n // 128, np.float32))] * 2
    ratio, apart, size = [], 0.0, 0.0
    g = (rng.normal(size=n) * 1e-3).astype(np.float32)
    for t in range(1, 1501):
        if not alike:
            g = (rng.normal(size=n) * 1e-3).astype(np.float32)
        m, v = adamw_ref.moments(g, 1.0, adamw_ref.decode(*codes[0], "M"), adamw_ref.decode(*codes[1], "V"), 0.9, 0.999)
        codes = [adamw_ref.encode(m, t, "M"), adamw_ref.encode(v, t, "V")]
        M, V = adamw_ref.moments(g, 1.0, M, V, 0.9, 0.999)
        if t > 750:
            ratio.append(adamw_ref.decode(*codes[1], "V") / V)
            u8, u = (adamw_ref.update(np.zeros(n), a, b, 1.0, 0.9, 0.999, 1e-8, t, 0.0)[0] for a, b in ((m, v), (M, V)))
            apart, size = apart + ((u8 - u) ** 2).sum(), size + (u ** 2).sum()
    ratio = np.array(ratio)
    assert ratio.std() < 8 ** -0.5
    assert abs(ratio.mean() - 1) < 4 * 8 ** -0.5 / n ** 0.5  # the cut takes nothing on average: four deviations of a mean of n
    assert np.sqrt(apart / size) < 0.21

"""Pins of the 4-bit cache's oracle: formats, borders, exactness, brute force; rotary frequencies and transforms."""
import numpy as np
import pytest

from oracle import paged4
from oracle.fp8 import e4m3_decode


def test_format_constants():
    codes = np.arange(256, dtype=np.uint8)
    v = paged4.values(np.tile(codes[:, None], (1, 8)), np.full((256, 1), 0x38, np.uint8))  # scale 1
    np.testing.assert_array_equal(v[:16, 0], [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
    np.testing.assert_array_equal(v[:, 1], v[codes >> 4, 0])


def test_quantise_against_brute_force():
    """The nearest representable value given the scale, and the nearest scale to max / 6."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 16)) * np.exp(2 * rng.standard_normal((400, 1)))
    codes, scales = paged4.quantise(x)
    grid = e4m3_decode(np.arange(0x7F, dtype=np.uint8))
    want = np.abs(grid[None] - np.abs(x).max(1, keepdims=True) / 6).min(1)
    got = np.abs(grid[scales[:, 0]] - np.abs(x).max(1) / 6)
    np.testing.assert_allclose(got, want, rtol=1e-12)
    steps = np.concatenate([paged4.E2M1, -paged4.E2M1])[None, None] * grid[scales][:, :, None]
    err = np.abs(paged4.values(codes, scales) - x)
    np.testing.assert_allclose(err, np.abs(steps - x[:, :, None]).min(-1), atol=1e-12)


def test_ties_go_to_the_even_code():
    """max 6 fixes the scale at 1; the borders of E2M1 lie at 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5."""
    x = np.array([[6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0]])
    c, s = paged4.quantise(x)
    assert s[0, 0] == 0x38
    np.testing.assert_array_equal(paged4.values(c, s)[0], [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 0])
    # one step of a double on either side
    for d, want in ((np.inf, [.5, 1, 1.5, 2, 3, 4, 6]), (-np.inf, [0, .5, 1, 1.5, 2, 3, 4])):
        y = x.copy()
        y[0, 1:8] = np.nextafter(x[0, 1:8], d)
        np.testing.assert_array_equal(paged4.values(*paged4.quantise(y))[0, 1:8], want)
    # scales: 6 * (1 + 1/16) lies between 1 (even) and 1.125
    for v, want in ((6 * 1.0625, 0x38), (np.nextafter(6 * 1.0625, 9), 0x39), (6 * 1.1875, 0x3A)):
        assert paged4.quantise(np.r_[v, np.zeros(15)][None])[1][0, 0] == want


def test_small_large_and_non_finite():
    x = np.zeros((6, 16))
    x[1, 0], x[2, 0], x[3, 0], x[4, 3], x[5, 3] = 6 * 2.0 ** -10, 6 * 2.0 ** -10 * (1 + 2.0 ** -40), 1e30, np.inf, np.nan
    c, s = paged4.quantise(x)
    v = paged4.values(c, s)
    assert (v[0] == 0).all() and (v[1] == 0).all()        # half of the smallest scale: ties to 0
    assert v[2, 0] == 3 * 2.0 ** -9 and v[3, 0] == 2688 and s[3, 0] == 0x7E  # (the smallest scale, 2^-9: 3 steps of it)
    assert (s[4:, 0] == 0x7F).all() and np.isnan(v[4:]).all()


def test_every_value_has_six_significant_bits_and_is_its_own_code():
    """Reading back is exact in bf16, and storing what was read gives the same values again where the largest code is 6."""
    from pd_inputs import bf16_round
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 256, (500, 8)).astype(np.uint8)
    codes[:, 0] = 0x7
    scales = rng.integers(0, 0x7F, (500, 1)).astype(np.uint8)
    v = paged4.values(codes, scales)
    np.testing.assert_array_equal(bf16_round(v.astype(np.float32)), v)
    np.testing.assert_array_equal(paged4.values(*paged4.quantise(v)), v)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "turns", "index"])
def test_frequencies(scaling):
    f0 = paged4.frequencies(64, 1e4)
    f = paged4.frequencies(64, 1e4, scaling, 8.0, 4096, 1.0, 32.0)
    assert f.shape == (32,) and (f > 0).all() and (np.diff(f) <= 0).all() and (f <= f0 * (1 + 1e-12)).all()
    if scaling == "linear":
        np.testing.assert_allclose(f * 8, f0)
    if scaling == "base":
        assert f[0] == 1 and np.isclose(f[-1] * 8, f0[-1])      # the slowest pair is slowed by the factor
    if scaling in ("turns", "index"):
        turns = 4096 * f0 / (2 * np.pi)
        assert np.isclose(f, f0)[turns > 60].all() and np.isclose(f * 8, f0)[turns < 0.5].all()
        assert ((f > f0 / 8) & (f < f0)).any()
    np.testing.assert_allclose(paged4.frequencies(64, 1e4, scaling, 1.0), f0)


def test_transform_is_a_rotation_of_the_normalised_head():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 3, 64))
    cs = paged4.table(paged4.frequencies(32, 1e4), np.arange(5) * 7)
    for pairs in (False, True):
        y, mag = paged4.transform(x, np.ones(64), 0.0, cs, pairs)
        np.testing.assert_allclose((y ** 2).mean(-1), 1.0)
        assert (mag >= np.abs(y) - 1e-12).all()
        z, _ = paged4.transform(x, None, 0.0, cs, pairs)
        np.testing.assert_array_equal(z[..., 32:], x[..., 32:])
        np.testing.assert_allclose(z[0], x[0])
        # turning back
        back = cs.copy()
        back[..., 1] *= -1
        np.testing.assert_allclose(paged4.transform(z, None, 0.0, back, pairs)[0], x)
    # the layouts are the same rotation of differently ordered features
    order = np.r_[np.arange(32).reshape(2, 16).T.reshape(-1), np.arange(32, 64)]
    a, _ = paged4.transform(x, None, 0.0, cs, False)
    b, _ = paged4.transform(x[..., order], None, 0.0, cs, True)
    np.testing.assert_allclose(b, a[..., order])


def test_append_and_sequence():
    rng = np.random.default_rng(3)
    codes, scales = np.zeros((4, 2, 16, 32), np.uint8), np.full((4, 2, 16, 4), 0x7F, np.uint8)
    exp = np.array([3, -2])
    x = rng.standard_normal((20, 2, 64)) * np.exp2(exp)[:, None]
    paged4.append(codes, scales, [2, 0], 5, x, exp)
    v = paged4.sequence(codes, scales, [2, 0], 25, exp)
    assert np.isnan(v[:5]).all() and np.isfinite(v[5:]).all()
    # half a step of E2M1 at its largest, a sixth of the group's maximum, and the rounding of the scale
    amax = np.abs(x).reshape(20, 2, 4, 16).max(-1).repeat(16, -1)
    assert (np.abs(v[5:] - x) <= amax * (1 / 6 + 1 / 16)).all()

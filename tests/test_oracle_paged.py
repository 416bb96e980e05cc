"""Pins of oracle/paged.py (no GPU)."""
import numpy as np
import pytest

import pd_inputs as gen
from oracle import fp8, paged


def test_page_scale_is_the_smallest_power_of_two():
    rng = np.random.default_rng(0)
    amax = np.concatenate([np.exp2(rng.uniform(-100, 100, 2000)), 448.0 * np.exp2(np.arange(-40, 40.0)),
                           np.nextafter(np.float32(448.0), np.float32(1e9)) * np.exp2(np.arange(-40, 40.0))])
    s = paged.page_scale(amax)
    assert np.all(np.log2(s) == np.round(np.log2(s)))
    assert np.all(amax <= 448.0 * s) and np.all(amax > 448.0 * s / 2)
    assert paged.page_scale(448.0) == 1.0 and paged.page_scale(np.nextafter(448.0, 449.0)) == 2.0
    assert paged.page_scale(0.0) == 2.0 ** -117 and paged.page_scale(1e-44) == 2.0 ** -117
    assert paged.page_scale(float(np.finfo(np.float32).max)) == 2.0 ** 120


def _empty(n_pages, hkv, page_len, hd):
    return np.full((n_pages, hkv, page_len, hd), 0xAB, np.uint8), np.full((n_pages, hkv), np.nan, np.float32)


@pytest.mark.parametrize("page_len", [16, 32])
def test_append_one_by_one_equals_one_call_up_to_subnormal_codes(page_len):
    """The scale ends up the same; values a page held when its scale grew keep their code's value except where it became a
    subnormal code, which may then be off by one more half step (2^-10 scales)."""
    rng = np.random.default_rng(1)
    rows = rng.standard_normal((75, 2, 64)) * np.exp(rng.standard_normal((75, 2, 1)))
    ids = [3, 0, 4, 1, 2]
    ca, sa = _empty(5, 2, page_len, 64)
    cb, sb = _empty(5, 2, page_len, 64)
    paged.append(ca, sa, ids, 0, rows)
    for i in range(75):
        paged.append(cb, sb, ids, i, rows[i:i + 1])
    used = ids[:-(-75 // page_len)]
    assert np.array_equal(sa[used], sb[used])
    va, vb = paged.sequence(ca, sa, ids, 75), paged.sequence(cb, sb, ids, 75)
    step = np.repeat(sa[used].astype(np.float64), page_len, axis=0)[:75, :, None] * 2.0 ** -9
    assert np.all(np.abs(va - vb) <= step)
    assert np.array_equal(va[np.abs(va) >= 32 * step], vb[np.abs(va) >= 32 * step])
    err = np.abs(vb - rows)
    assert np.all(err <= 2.0 ** -4 * np.abs(rows) + step)


def test_append_leaves_other_rows_alone_and_restarts_a_page():
    c, s = _empty(3, 1, 16, 64)
    before = c.copy()
    paged.append(c, s, [2, 0], 0, np.full((18, 1, 64), 100.0))
    assert np.array_equal(c[1], before[1]) and np.array_equal(c[0, :, 2:], before[0, :, 2:])
    assert s[2, 0] == 0.25 and s[0, 0] == 0.25
    paged.append(c, s, [2, 0], 5, np.full((1, 1, 64), 1.0))     # a rewritten row inside the page: the scale stays
    assert s[2, 0] == 0.25
    paged.append(c, s, [2, 0], 0, np.full((1, 1, 64), 1.0))     # the first row again: the page begins anew
    assert s[2, 0] == 2.0 ** -8


def test_non_finite_values_become_nan_codes():
    c, s = _empty(1, 1, 16, 64)
    rows = np.ones((2, 1, 64))
    rows[0, 0, 0], rows[1, 0, 1], rows[1, 0, 2] = np.inf, np.nan, -np.inf
    paged.append(c, s, [0], 0, rows)
    assert s[0, 0] == 2.0 ** -8
    assert np.all((c[0, 0, [0, 1, 1], [0, 1, 2]] & 0x7F) == 0x7F)


def test_values_decode_to_bf16_exactly():
    codes = np.arange(256, dtype=np.uint8)
    for e in (-117, -30, 0, 60):
        v = (fp8.e4m3_decode(codes) * 2.0 ** e).astype(np.float32)
        ok = np.isfinite(v)
        assert np.array_equal(gen.bf16_round(v[ok]), v[ok])


def test_rotation_is_the_complex_product():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((9, 3, 64))
    pos = np.array([0, 1, 5, 100, 4095, 32767, 7, 8, 9])
    y = paged.rotate(x, pos, 1e4)
    z = (x[..., :32] + 1j * x[..., 32:]) * np.exp(1j * pos[:, None] * 1e4 ** (-np.arange(32) / 32.0))[:, None]
    np.testing.assert_allclose(y, np.concatenate([z.real, z.imag], -1), atol=1e-11)
    np.testing.assert_array_equal(y[0], x[0])


def test_rope_table_of_the_library(pdlib):
    cfg = pdlib.LayerConfig(512, 8, 2, 64, 64, rope_theta=1e4, max_pos=5000)
    tab = pdlib.pd_rope_table(cfg)
    ang = np.arange(5000)[:, None] * 1e4 ** (-2.0 * np.arange(32) / 64)
    # one rounding to float32, and the angles' own double rounding (5000 * 2^-53 is far below it)
    assert np.all(np.abs(tab[..., 0] - np.cos(ang)) <= 2.0 ** -24 + 1e-11)
    assert np.all(np.abs(tab[..., 1] - np.sin(ang)) <= 2.0 ** -24 + 1e-11)
    x = gen.normal_bf16(1, 2, (4, 2, 64))
    pos = np.array([0, 17, 1000, 4999])
    np.testing.assert_allclose(paged.rotate_f32(x, tab[pos]), paged.rotate(x, pos, 1e4), atol=2e-6)


def test_attend_matches_a_loop():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    o, spread, _ = paged.attend(q, k, v, [4, 0, -1])
    for h in range(4):
        w = np.exp([q[0, h] @ k[j, h // 2] / np.sqrt(8) for j in range(5)])
        np.testing.assert_allclose(o[0, h], sum(w[j] * v[j, h // 2] for j in range(5)) / w.sum())
        np.testing.assert_allclose(o[1, h], v[0, h // 2])
    assert not o[2].any() and np.all(spread >= np.abs(o) - 1e-12)


def test_add_rmsnorm_against_the_row_quantiser():
    x, r = gen.normal_bf16(4, 1, (5, 256), 2.0), gen.normal_bf16(4, 2, (5, 256), 1.0)
    g = gen.normal_bf16(4, 3, (256,), 0.1, 1.0)
    h, n, s = paged.add_rmsnorm(x, r, g, 1e-6, 128)
    assert np.array_equal(h, gen.bf16_round(x + r).astype(np.float64))   # (float32 sums of these are exact enough here)
    np.testing.assert_allclose((n / g) @ np.ones(256) * 0 + np.sqrt(((n / g) ** 2).mean(-1)), 1.0, rtol=1e-6)
    assert s.shape == (5, 2) and np.allclose(s * 448, np.abs(n.reshape(5, 2, 128)).max(-1))
    _, n1, s1 = paged.add_rmsnorm(x, None, g, 1e-6, 0)
    assert s1.shape == (5,) and np.allclose(s1 * 448, np.abs(n1).max(-1))

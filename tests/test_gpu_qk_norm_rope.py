"""GPU: tables of scaled rotary positions, and the norm and rotation of q and k heads, against the float64 oracle."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from kv4_util import Transform, transform_bound
from oracle import paged4

pytestmark = pytest.mark.gpu
SCALINGS = ["none", "linear", "base", "turns", "index"]


def run_table(pd, rot, scaling, first, n, factor=8.0, trained=4096, low=1.0, high=32.0, magnitude=1.0, theta=1e4):
    import torch
    rope = pd.RopeConfig(rot, theta, SCALINGS.index(scaling), factor, trained, low, high, magnitude)
    t = torch.full((n + 1, rot // 2, 2), 7.0, device="cuda")
    pd.pd_rope_table_scaled(rope, first, n, t)
    torch.cuda.synchronize()
    assert (t[n] == 7.0).all()
    return t[:n].cpu().numpy()


def check_table(got, f, positions, magnitude):
    """One rounding to fp32 (2^-24 of at most the magnitude), and the angle in double: position * f has a relative error of some
    2^-51 on either side."""
    want = paged4.table(f, positions, magnitude)
    bound = magnitude * (2.0 ** -24 + positions[:, None, None] * 2.0 ** -50)
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("rot,first,n", [(64, 0, 1000), (128, 0, 1), (16, 5, 3), (112, 1 << 20, 257), (32, 2 ** 31 - 100, 99)])
def test_table(pdlib, scaling, rot, first, n):
    m = 1.25 if scaling == "index" else 1.0
    got = run_table(pdlib, rot, scaling, first, n, magnitude=m)
    check_table(got, paged4.frequencies(rot, 1e4, scaling, 8.0, 4096, 1.0, 32.0), first + np.arange(n), m)


@pytest.mark.parametrize("rot,theta,trained,low,high", [(128, 5e5, 8192, 1.0, 4.0), (64, 10.0, 1, 1e-3, 2.0), (96, 1e6, 2 ** 30, 1.0, 1e9)])
@pytest.mark.parametrize("scaling", ["turns", "index"])
def test_table_with_other_bounds(pdlib, scaling, rot, theta, trained, low, high):
    got = run_table(pdlib, rot, scaling, 0, 70, 40.0, trained, low, high, 1.0, theta)
    check_table(got, paged4.frequencies(rot, theta, scaling, 40.0, trained, low, high), np.arange(70), 1.0)


def test_long_table(pdlib):
    n = 131072 + 3
    got = run_table(pdlib, 128, "turns", 11, n)
    at = np.unique(np.r_[np.arange(40), np.random.default_rng(0).integers(0, n, 500), np.arange(n - 40, n)])
    check_table(got[at], paged4.frequencies(128, 1e4, "turns", 8.0, 4096, 1.0, 32.0), 11 + at, 1.0)


class Rows:
    """Projection rows with a pitch, on the device; columns that are no head hold NaN."""

    def __init__(self, pd, rows, hq, hkv, hd, pad=16, seed=0):
        self.pd, self.rows, self.hq, self.hkv, self.hd = pd, rows, hq, hkv, hd
        self.ld = (hq + 2 * hkv) * hd + pad
        self.x = np.full((rows, self.ld), np.nan, np.float32)
        n = (hq + 2 * hkv) * hd
        self.x[:, :n] = gen.normal_bf16(seed, gen.S_X, (rows, n), 1.5)
        self.cfg = pd.LayerConfig(hq * hd, hq, hkv, hd, 64)

    def q(self):
        return self.x[:, :self.hq * self.hd].reshape(self.rows, self.hq, self.hd)

    def k(self):
        return self.x[:, self.hq * self.hd:(self.hq + self.hkv) * self.hd].reshape(self.rows, self.hkv, self.hd)


def check_rows(got, want, live, untouched=0):
    y, mag = want
    err = np.abs(got.reshape(y.shape)[live] - y[live])
    over = err / transform_bound(y, mag)[live]
    assert over.max(initial=0.0) <= 1.0, over.max()
    assert (got.reshape(y.shape)[~live] == untouched).all()


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (5, 5, 64), (16, 1, 128), (3, 1, 128)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rows", [1, 33, 200])
def test_norm_and_rotation(pdlib, hq, hkv, hd, pairs, rows):
    import torch
    rng = np.random.default_rng(rows)
    for rot in {16, 48, hd // 2, hd - 16, hd, 0}:
        r = Rows(pdlib, rows, hq, hkv, hd, seed=rot)
        for gains in (True, False) if rot else (True,):
            t = Transform(pdlib, hd, rot, 500, pairs, gains, magnitude=1.1)
            pos = rng.integers(0, 500, rows)
            if rows > 10:
                pos[[3, 7]] = [-1, -1 << 31]
                if rot:
                    pos[5] = 500
            live = (pos >= 0) & ((pos < 500) | (rot == 0))
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            q, k = empty_bf16(rows, hq * hd + 8), empty_bf16(rows, hkv * hd + 24)
            pdlib.pd_qk_norm_rope(r.cfg, t.struct, to_dev(r.x), r.ld, q, hq * hd + 8, k, hkv * hd + 24, i32_dev(pos), rows, err_word=err)
            assert int(err.item()) == (2 if rows > 10 and rot else 0)
            q, k = from_dev(q), from_dev(k)
            assert not q[:, hq * hd:].any() and not k[:, hkv * hd:].any()
            at = np.where(live, pos, 0)
            check_rows(q[:, :hq * hd], t.q(r.q(), at), live)
            check_rows(k[:, :hkv * hd], t.k(r.k(), at), live)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("gains", [False, True])
def test_in_place_and_one_of_the_two(pdlib, pairs, gains):
    hq, hkv, hd, rows = 6, 2, 128, 70
    r = Rows(pdlib, rows, hq, hkv, hd)
    t = Transform(pdlib, hd, 96, 100, pairs, gains)
    pos = np.arange(rows)
    dev = to_dev(r.x)
    pdlib.pd_qk_norm_rope(r.cfg, t.struct, dev, r.ld, dev, r.ld, dev.data_ptr() + hq * hd * 2, r.ld, i32_dev(pos), rows)
    q, k = empty_bf16(rows, hq * hd), empty_bf16(rows, hkv * hd)
    src = to_dev(r.x)
    pdlib.pd_qk_norm_rope(r.cfg, t.struct, src, r.ld, q, hq * hd, None, 0, i32_dev(pos), rows)
    pdlib.pd_qk_norm_rope(r.cfg, t.struct, src, r.ld, None, 0, k, hkv * hd, i32_dev(pos), rows)
    both = np.concatenate([from_dev(q), from_dev(k)], axis=1)
    got = from_dev(dev)
    np.testing.assert_array_equal(got[:, :both.shape[1]], both)
    np.testing.assert_array_equal(got[:, both.shape[1]:], r.x[:, both.shape[1]:])
    live = np.ones(rows, bool)
    check_rows(both[:, :hq * hd], t.q(r.q(), pos), live)
    check_rows(both[:, hq * hd:], t.k(r.k(), pos), live)


def test_unusual_heads(pdlib):
    """Zeros under eps, one large feature, magnitudes from 1e-15 to 1e15, and a NaN that stays in its head."""
    hq, hkv, hd, rows = 4, 4, 64, 8
    r = Rows(pdlib, rows, hq, hkv, hd, pad=0)
    q = r.x[:, :hq * hd].reshape(rows, hq, hd)
    q[0] = 0
    q[1, :, 1:] = 0
    q[2] = gen.bf16_round(q[2] * np.float32(1e-15))
    q[3] = gen.bf16_round(q[3] * np.float32(1e15))
    t = Transform(pdlib, hd, 64, 10, gains=True)
    r.x[4, 2 * hd + 5] = np.nan
    out, k = empty_bf16(rows, hq * hd), empty_bf16(rows, hkv * hd)
    pdlib.pd_qk_norm_rope(r.cfg, t.struct, to_dev(r.x), r.ld, out, hq * hd, k, hkv * hd, i32_dev(np.arange(rows)), rows)
    got = from_dev(out).reshape(rows, hq, hd)
    assert np.isnan(got[4, 2]).all()
    got[4, 2], q[4, 2] = 0, 0
    check_rows(got, t.q(q, np.arange(rows)), np.ones(rows, bool))
    check_rows(from_dev(k), t.k(r.k(), np.arange(rows)), np.ones(rows, bool))

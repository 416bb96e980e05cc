"""GPU: appending more rows in one call than the form of the kernel for few rows takes, against the float64 oracle: heads that
are no multiple of what a warp has at a time, both layouts, part of a head rotated, with and without norms."""
import numpy as np
import pytest

from kv4_util import Cache4, Transform
from test_gpu_kv4_append import append, expect, rows_of

pytestmark = pytest.mark.gpu


def check(pd, hq, hkv, hd, new, kv_len, pairs, rot, gains, page_len):
    cu = np.r_[0, np.cumsum(new)].tolist() if new is not None else None
    after = [max(0, k) + n for k, n in zip(kv_len, new if new is not None else [1] * len(kv_len))]
    c = Cache4(pd, hkv, hd, page_len, after, seed=hq).upload()
    t = Transform(pd, hd, rot, max(after), pairs, gains, seed=hkv)
    x = rows_of(hq + rot, cu[-1] if cu else len(kv_len), hq, hkv, hd)
    q = append(pd, c, t, x, kv_len, cu)
    expect(c, t, x, kv_len, cu, q)
    c.assert_equal()


@pytest.mark.parametrize("hq,hkv,hd", [(32, 8, 128), (64, 8, 128), (36, 9, 128), (40, 5, 128), (33, 3, 128), (80, 5, 64), (72, 18, 64), (130, 10, 64)])
@pytest.mark.parametrize("pairs,rot_part,gains", [(False, 1.0, True), (True, 1.0, True), (False, 0.5, True), (True, 0.75, False), (False, 0.25, False)])
def test_ragged_runs(pdlib, hq, hkv, hd, pairs, rot_part, gains):
    """1,103 rows: runs that begin and end inside pages, an empty one, one that is left out, one of a single row."""
    check(pdlib, hq, hkv, hd, [501, 0, 1, 77, 390, 5, 129], [0, 9, 15, -1, 40, 127, 3], pairs, int(hd * rot_part), gains, 32)


@pytest.mark.parametrize("rows", [1023, 1024, 1025, 1026, 1031])
@pytest.mark.parametrize("pairs", [False, True])
def test_around_the_border_of_the_two_forms(pdlib, rows, pairs):
    check(pdlib, 40, 8, 128, [rows - 300, 300], [0, 33], pairs, 128, True, 64)


@pytest.mark.parametrize("pairs", [False, True])
def test_a_decode_step_of_many_sequences(pdlib, pairs):
    """A row per request, no runs."""
    kv_len = np.random.default_rng(5).integers(-1, 60, 1100).tolist()
    check(pdlib, 36, 4, 128, None, kv_len, pairs, 96, True, 16)


def test_one_call_and_many_give_the_same_cache(pdlib):
    """The forms for many and for few rows, bit for bit, q as well."""
    hq, hkv, hd, n = 40, 8, 128, 1500
    for pairs in (False, True):
        t = Transform(pdlib, hd, 128, n, pairs)
        x = rows_of(6, n, hq, hkv, hd)
        got = []
        for pieces in ([(0, n)], [(0, 1000), (1000, 1001), (1001, n)]):
            c = Cache4(pdlib, hkv, hd, 64, [n], seed=7).upload()
            got.append((c, np.concatenate([append(pdlib, c, t, x[a:b], [a], [0, b - a]) for a, b in pieces])))
        (a, qa), (b, qb) = got
        np.testing.assert_array_equal(qa, qb)
        for name in ("dk", "dv", "dks", "dvs"):
            assert (getattr(a, name) == getattr(b, name)).all()

"""GPU: writing the 4-bit paged KV cache and reading it back, bit for bit against the float64 oracle (keys are normalised and
rotated in double, so their codes are those of the exact values)."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from kv4_util import Cache4, Transform, transform_bound
from oracle import paged4

pytestmark = pytest.mark.gpu


def rows_of(seed, n, hq, hkv, hd, spread=0.7):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, hq + 2 * hkv, hd)) * np.exp(spread * rng.standard_normal((n, hq + 2 * hkv, 1)))
    return gen.bf16_round(x)


def append(pd, c, t, x, kv_len, cu=None, q=True, pad=8, err=None, hq=None, stream=None):
    """Rows x [T, H, hd] through the library; returns q."""
    import torch
    n = len(x)
    width = x.shape[1] * x.shape[2]
    flat = np.full((n, width + pad), np.nan, np.float32)
    flat[:, :width] = x.reshape(n, width)
    hq = x.shape[1] - 2 * c.hkv
    cfg = pd.LayerConfig(hq * c.hd, hq, c.hkv, c.hd, 64)
    out = empty_bf16(n + 1, hq * c.hd) if q else None
    pd.pd_paged_kv4_append(cfg, t.struct, to_dev(flat), width + pad, out, c.struct, i32_dev(kv_len), len(kv_len),
                           cu_seqlens_dev=None if cu is None else i32_dev(cu), cu_seqlens_host=cu, err_word=err, stream=stream)
    torch.cuda.synchronize()
    if not q:
        return None
    assert not out[n].any()
    return from_dev(out[:n]).reshape(n, hq, c.hd)


def expect(c, t, x, kv_len, cu, q=None):
    """The oracle's append; q is held to its transform."""
    hq = x.shape[1] - 2 * c.hkv
    cu = cu if cu is not None else list(range(len(kv_len) + 1))
    for s, n0 in enumerate(kv_len):
        part = x[cu[s]:cu[s + 1]]
        if n0 < 0 or not len(part):
            if q is not None:
                assert not q[cu[s]:cu[s + 1]].any()
            continue
        pos = n0 + np.arange(len(part))
        paged4.append(c.k, c.ks, c.table[s], n0, t.k(part[:, hq:hq + c.hkv], pos)[0], c.ke)
        paged4.append(c.v, c.vs, c.table[s], n0, part[:, hq + c.hkv:], c.ve)
        if q is not None:
            y, mag = t.q(part[:, :hq], pos)
            assert (np.abs(q[cu[s]:cu[s + 1]] - y) <= transform_bound(y, mag)).all()


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (64, 8, 128), (5, 5, 64), (16, 1, 128)])
@pytest.mark.parametrize("page_len", [16, 64, 128])
@pytest.mark.parametrize("pairs,rot_part,gains", [(False, 1.0, True), (True, 0.5, True), (False, 0.25, False), (True, 0.75, False), (False, 0.75, True)])
def test_one_token_per_sequence(pdlib, hq, hkv, hd, page_len, pairs, rot_part, gains):
    kv_len = [0, 1, 15, 16, 17, 63, -1, 64, 100, 127, 128, 300, 511]
    c = Cache4(pdlib, hkv, hd, page_len, [max(0, n + 1) for n in kv_len], seed=hq).upload()
    t = Transform(pdlib, hd, int(hd * rot_part), 512, pairs, gains, seed=hq)
    x = rows_of(hq + page_len, len(kv_len), hq, hkv, hd)
    q = append(pdlib, c, t, x, kv_len)
    expect(c, t, x, kv_len, None, q)
    c.assert_equal()


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (4, 4, 128)])
@pytest.mark.parametrize("page_len", [16, 32, 64, 128])
@pytest.mark.parametrize("pairs,rot,gains", [(False, 64, True), (True, 32, False), (False, 16, True), (False, 48, False)])
def test_runs_of_tokens(pdlib, hq, hkv, hd, page_len, pairs, rot, gains):
    """Ragged runs that begin and end inside pages, empty ones among them, and a request that is left out."""
    new, kv_len = [70, 0, 1, 33, 5, 130, 0], [0, 9, 15, 40, -1, 3, -1]
    cu = np.r_[0, np.cumsum(new)].tolist()
    c = Cache4(pdlib, hkv, hd, page_len, [max(0, k) + n for k, n in zip(kv_len, new)], seed=page_len).upload()
    t = Transform(pdlib, hd, rot, 200, pairs, gains, seed=rot)
    x = rows_of(hq + page_len, cu[-1], hq, hkv, hd)
    q = append(pdlib, c, t, x, kv_len, cu)
    expect(c, t, x, kv_len, cu, q)
    c.assert_equal()


def test_many_requests(pdlib):
    """More requests than a warp has lanes, most of them empty or of one row."""
    rng = np.random.default_rng(3)
    new = rng.integers(0, 4, 150)
    new[[0, 77, 149]] = [0, 40, 0]
    kv_len = rng.integers(0, 60, 150)
    cu = np.r_[0, np.cumsum(new)].tolist()
    c = Cache4(pdlib, 2, 64, 16, list(kv_len + new), seed=4).upload()
    t = Transform(pdlib, 64, 64, 200)
    x = rows_of(5, cu[-1], 4, 2, 64)
    q = append(pdlib, c, t, x, kv_len.tolist(), cu)
    expect(c, t, x, kv_len.tolist(), cu, q)
    c.assert_equal()


def test_pieces_give_the_same_cache_as_one_call(pdlib):
    """Whatever the order and the division into calls; without q as well."""
    hq, hkv, hd, n = 8, 2, 128, 90
    t = Transform(pdlib, hd, 128, 200)
    x = rows_of(6, n, hq, hkv, hd)
    whole = Cache4(pdlib, hkv, hd, 32, [n], seed=7).upload()
    append(pdlib, whole, t, x, [0], [0, n])
    parts = Cache4(pdlib, hkv, hd, 32, [n], seed=7).upload()
    for a, b in ((40, 41), (41, 90), (0, 40)):
        append(pdlib, parts, t, x[a:b], [a], [0, b - a] if b - a > 1 else None, q=False)
    append(pdlib, parts, t, x[10:30], [10], [0, 20])
    for a, b in ((whole.dk, parts.dk), (whole.dv, parts.dv), (whole.dks, parts.dks), (whole.dvs, parts.dvs)):
        assert (a == b).all()


def test_values_of_every_size(pdlib):
    """Ties of both formats, values beyond the largest and below the smallest, zeros of either sign, infinities and NaN, exponents
    beyond their limits."""
    hq, hkv, hd, n = 2, 2, 64, 64
    rng = np.random.default_rng(8)
    x = rows_of(9, n, hq, hkv, hd)
    flat = x.reshape(n, -1, 4, 16)
    steps = np.array([.25, .5, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 1, 1.5, 2, 3, 4, 0, -0.])
    for i in range(12):
        flat[i, :, 1] = gen.bf16_round(np.where(rng.random(16) < 0.5, -1, 1) * rng.permutation(steps) * 2.0 ** (i - 6))
        flat[i, :, 2] = gen.bf16_round(rng.permutation(steps) * 1.125 * 2.0 ** (i - 12))   # scales that tie: 6 * (1 + k / 8 + 1/16)
        flat[i, :, 2, 0] = 6 * (1 + i % 8 / 8 + 1 / 16) * 2.0 ** (i - 8)
        flat[i, :, 3] = 0.0 if i % 2 else -0.0
    flat[12:18, :, 0] *= np.float32(2.0 ** 100)
    flat[18:24, :, 0] *= np.float32(2.0 ** -100)
    flat[24, :, 0, 3], flat[25, :, 1, 4], flat[26, :, 2, 5] = np.inf, -np.inf, np.nan
    flat[27] = 3.38e38
    flat[28] = 1e-40
    x = gen.bf16_round(x)
    for exps in ([0, 5], [30, -30], [77, -77]):
        c = Cache4(pdlib, hkv, hd, 16, [n], seed=10)
        c.k_exp = c.v_exp = np.array(exps, np.int32)
        c.ke = c.ve = paged4.head_exp(c.k_exp, hkv)
        c.upload()
        t = Transform(pdlib, hd, 0, 0, gains=False)
        append(pdlib, c, t, x, [0], [0, n])
        expect(c, t, x, [0], [0, n])
        c.assert_equal(str(exps))


def test_rows_without_a_place(pdlib):
    import torch
    hq, hkv, hd, p = 4, 2, 64, 16
    t = Transform(pdlib, hd, 64, 70)
    kv_len = [5, 20, 31, 70, 2 ** 31 - 1]
    x = rows_of(11, len(kv_len), hq, hkv, hd)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for which, sentinel in (("bad page", 99), ("negative page", -5), ("table end", None), ("no table", None)):
        c = Cache4(pdlib, hkv, hd, p, [32, 32, 32, 32, 32], seed=12, extra_cols=0)
        if sentinel is not None:
            c.table[1, 1] = sentinel
        c.upload()
        err.zero_()
        kv = list(kv_len)
        if which == "table end":
            kv[1] = 32
        tt = Transform(pdlib, hd, 0, 0) if which == "no table" else t
        q = append(pdlib, c, tt, x, kv, err=err)
        assert int(err.item()) == 2, which
        if sentinel is not None:
            c.table[1, 1] = c.n_pages - 1    # (a page of the pool that the oracle may fill, and that stayed as it was)
        spare = (c.k.copy(), c.ks.copy(), c.v.copy(), c.vs.copy())
        for s in (0, 2) if which != "no table" else (0, 1, 2):
            pos = [kv[s]]
            paged4.append(c.k, c.ks, c.table[s], kv[s], tt.k(x[s:s + 1, hq:hq + hkv], pos)[0], c.ke)
            paged4.append(c.v, c.vs, c.table[s], kv[s], x[s:s + 1, hq + hkv:], c.ve)
        assert (spare[0] != c.k).any()
        c.assert_equal(which)
        # q of a row without a page is there, that of a row beyond the rotation table is not
        y, mag = tt.q(x[1:2, :hq], [kv[1]])
        assert (np.abs(q[1:2] - y) <= transform_bound(y, mag)).all()
        if which != "no table":
            assert not q[3:].any()
        else:
            y, mag = tt.q(x[3:, :hq], [0, 0])
            assert (np.abs(q[3:] - y) <= transform_bound(y, mag)).all()


def test_rows_behind_the_last_position(pdlib):
    """Positions 2^31 - 1 and 2^31 have no place; without a rotation table their q is there all the same."""
    import torch
    c, t = Cache4(pdlib, 2, 64, 16, [32], seed=13).upload(), Transform(pdlib, 64, 0, 0)
    x, err = rows_of(12, 2, 4, 2, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = append(pdlib, c, t, x, [2 ** 31 - 1], cu=[0, 2], err=err)
    assert int(err.item()) == 2
    y, mag = t.q(x[:, :4], [0, 0])
    assert (np.abs(q - y) <= transform_bound(y, mag)).all()
    c.assert_equal()


# ------------------------------------------------------------------------------------------------------ read and write
@pytest.mark.parametrize("hkv,hd,page_len", [(2, 64, 16), (8, 128, 64), (1, 128, 32), (3, 64, 128)])
def test_read_back(pdlib, hkv, hd, page_len):
    import torch
    lens = [0, 1, 17, 64, 200, 333, 40]
    begin, end = [0, 0, 3, 0, 16, 100, 30], [0, 1, 17, 64, 200, 333, 20]
    slots, origin = [2, 7, 0, 1, 6, 3, 4], [0, 0, 3, -5, 0, 90, 0]
    c = Cache4(pdlib, hkv, hd, page_len, lens, seed=hd).fill(lens, np.random.default_rng(hd)).upload()
    cfg = pdlib.LayerConfig(hkv * hd, hkv, hkv, hd, 64)
    for use_slots in (True, False):
        k, v = (torch.full((8, hkv, 340, hd), -1, dtype=torch.int16, device="cuda") for _ in range(2))
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        pdlib.pd_paged_kv4_read(cfg, c.struct, i32_dev(begin), i32_dev(end), len(lens), 240, pdlib.kv_cache_struct(k, v, 8, 340),
                                slots_dev=i32_dev(slots) if use_slots else None, origin_dev=i32_dev(origin) if use_slots else None, err_word=err)
        assert int(err.item()) == 0
        want_k, want_v = (np.full((8, hkv, 340, hd), np.nan, np.float32) for _ in range(2))
        for s, n in enumerate(lens):
            if end[s] > begin[s]:
                slot, at = (slots[s], begin[s] - origin[s]) if use_slots else (s, begin[s])
                for w, x in zip((want_k, want_v), c.kv(s, n)):
                    w[slot, :, at:at + end[s] - begin[s]] = x[begin[s]:end[s]].transpose(1, 0, 2)
        np.testing.assert_array_equal(from_dev(k), want_k)     # (exactly; -1 is a NaN: rows outside are as they were)
        np.testing.assert_array_equal(from_dev(v), want_v)


@pytest.mark.parametrize("hd", [64, 128])
def test_read_into_a_cache_that_starts_on_sixteen_bytes(pdlib, hd):
    import torch
    hkv, n = 3, 50
    c = Cache4(pdlib, hkv, hd, 16, [n], seed=hd).fill([n], np.random.default_rng(hd)).upload()
    cfg = pdlib.LayerConfig(hkv * hd, hkv, hkv, hd, 64)
    k, v = (torch.zeros(hkv * 60 * hd + 16, dtype=torch.int16, device="cuda") for _ in range(2))
    assert k.data_ptr() % 32 == 0
    back = pdlib.kv_cache_struct(k.data_ptr() + 16, v.data_ptr() + 16, 1, 60)
    pdlib.pd_paged_kv4_read(cfg, c.struct, None, i32_dev([n]), 1, n, back)
    for dev, want in zip((k, v), c.kv(0, n)):
        got = from_dev(dev)
        assert not got[:8].any() and not got[-8:].any()
        got = got[8:-8].reshape(hkv, 60, hd)
        np.testing.assert_array_equal(got[:, :n].transpose(1, 0, 2), want)
        assert not got[:, n:].any()


def test_read_reports_what_has_no_place(pdlib):
    import torch
    hkv, hd, p = 2, 64, 16
    cfg = pdlib.LayerConfig(hkv * hd, hkv, hkv, hd, 64)
    cases = [dict(end=[50, 33]), dict(begin=[0, -2]), dict(slots=[0, 2]), dict(slots=[0, -1]), dict(origin=[0, 5]), dict(origin=[0, -20]), dict(page=-1), dict(page=77),
             dict(begin=[0, -2 ** 31], end=[32, -2 ** 31 + 4]), dict(origin=[0, -2 ** 31])]
    for case in cases:
        c = Cache4(pdlib, hkv, hd, p, [32, 32], seed=1, extra_cols=0).fill([32, 32], np.random.default_rng(1))
        good = c.kv(0, 32)[0]
        if "page" in case:
            c.table[1, 0] = case["page"]
        c.upload()
        for write in (False, True):
            k, v = (torch.zeros((2, hkv, 40, hd), dtype=torch.int16, device="cuda") for _ in range(2))
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            a = [i32_dev(case.get("begin", [0, 0])), i32_dev(case.get("end", [32, 32])), 2, 64, pdlib.kv_cache_struct(k, v, 2, 40)]
            kw = dict(slots_dev=i32_dev(case.get("slots", [0, 1])), origin_dev=i32_dev(case.get("origin", [0, 0])), err_word=err)
            (pdlib.pd_paged_kv4_write if write else pdlib.pd_paged_kv4_read)(cfg, c.struct, *a, **kw)
            torch.cuda.synchronize()
            assert int(err.item()) == 2, case
            if not write:
                np.testing.assert_array_equal(from_dev(k)[0, :, :32].transpose(1, 0, 2), good)


@pytest.mark.parametrize("hkv,hd,page_len", [(2, 64, 16), (8, 128, 64), (1, 128, 128)])
def test_write(pdlib, hkv, hd, page_len):
    """A bf16 cache into the pages; what lies outside the ranges stays as it was, and what is read back is what was stored."""
    import torch
    lens, begin, slots, origin = [5, 64, 130, 0], [0, 10, 33, 0], [1, 3, 0, 2], [0, 10, 0, 0]
    c = Cache4(pdlib, hkv, hd, page_len, lens, seed=2).fill([n // 3 for n in lens], np.random.default_rng(2)).upload()
    cfg = pdlib.LayerConfig(hkv * hd, hkv, hkv, hd, 64)
    x = [gen.normal_bf16(5 + i, gen.S_KCACHE, (4, hkv, 140, hd), 1.0) * np.float32(2.0 ** i) for i in range(2)]
    k, v = to_dev(x[0]), to_dev(x[1])
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    flat = pdlib.kv_cache_struct(k, v, 4, 140)
    args = (i32_dev(begin), i32_dev(lens), 4, 130)
    kw = dict(slots_dev=i32_dev(slots), origin_dev=i32_dev(origin), err_word=err)
    pdlib.pd_paged_kv4_write(cfg, c.struct, *args, flat, **kw)
    assert int(err.item()) == 0
    for s, n in enumerate(lens):
        rows = slice(begin[s] - origin[s], n - origin[s])
        paged4.append(c.k, c.ks, c.table[s], begin[s], x[0][slots[s], :, rows].transpose(1, 0, 2), c.ke)
        paged4.append(c.v, c.vs, c.table[s], begin[s], x[1][slots[s], :, rows].transpose(1, 0, 2), c.ve)
    c.assert_equal()
    pdlib.pd_paged_kv4_read(cfg, c.struct, *args, flat, **kw)
    for s, n in enumerate(lens):
        for dev, want in zip((k, v), c.kv(s, n)):
            got = from_dev(dev[slots[s]])[:, begin[s] - origin[s]:n - origin[s]]
            np.testing.assert_array_equal(got.transpose(1, 0, 2), want[begin[s]:])

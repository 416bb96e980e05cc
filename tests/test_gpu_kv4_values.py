"""GPU: what the 4-bit cache stores of values far beyond its largest, of zeros and of small values of either sign, bit for bit
against the float64 oracle, by append (K and V, both layouts) and by write."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import i32_dev, to_dev
from kv4_util import Cache4, Transform
from oracle import paged4
from test_gpu_kv4_append import append, expect, rows_of

pytestmark = pytest.mark.gpu
HKV, N = 2, 40


def cache(pd, hd, exps, page_len=16):
    c = Cache4(pd, HKV, hd, page_len, [N], seed=hd)
    c.k_exp = c.v_exp = np.array(exps, np.int32)
    c.ke = c.ve = paged4.head_exp(c.k_exp, HKV)
    return c.upload()


def write(pd, c, k, v):
    """k, v [N, Hkv, hd] from a bf16 cache, and by the oracle."""
    dk, dv = (to_dev(np.ascontiguousarray(a.transpose(1, 0, 2))[None]) for a in (k, v))
    cfg = pd.LayerConfig(HKV * c.hd, HKV, HKV, c.hd, 64)
    pd.pd_paged_kv4_write(cfg, c.struct, None, i32_dev([N]), 1, N, pd.kv_cache_struct(dk, dv, 1, N))
    paged4.append(c.k, c.ks, c.table[0], 0, k, c.ke)
    paged4.append(c.v, c.vs, c.table[0], 0, v, c.ve)


def large(hd):
    """Rows of both signs beyond 448 * 6 * 2^exp, in whole groups, in some features and beside small ones."""
    rng = np.random.default_rng(hd)
    x = rows_of(3, N, HKV, HKV, hd).reshape(N, -1, hd // 16, 16)
    sign = np.where(rng.random(x.shape) < 0.5, -1.0, 1.0).astype(np.float32)
    for i, v in enumerate((3.38e38, 1e33, 1e30, 1.5e32, 2.0 ** 127, 2.0 ** 100)):
        x[4 * i] = v * sign[4 * i]
        x[4 * i + 1, ..., ::3] = v * sign[4 * i + 1, ..., ::3]
        x[4 * i + 2, :, 1] = -v
        x[4 * i + 3, ..., 5] = -v
    x[24:32] *= np.float32(2.0 ** 90) * np.exp2(rng.integers(0, 30, (8, *x.shape[1:]))).astype(np.float32)
    return gen.bf16_round(x.reshape(N, -1, hd))


@pytest.mark.parametrize("exps", [(-9, -8), (-20, 30), (-30, -10), (-99, 0)])
@pytest.mark.parametrize("hd", [64, 128])
def test_values_beyond_the_largest_keep_their_sign(pdlib, hd, exps):
    x = large(hd)
    for pairs, rot in ((False, 0), (True, 0), (False, hd), (True, hd // 2)):
        c, t = cache(pdlib, hd, exps), Transform(pdlib, hd, rot, N, pairs, gains=False)
        append(pdlib, c, t, x, [0], [0, N], q=False)
        expect(c, t, x, [0], [0, N])
        c.assert_equal(f"append, {pairs} {rot}")
    c = cache(pdlib, hd, exps)
    write(pdlib, c, x[:, HKV:2 * HKV], x[:, 2 * HKV:])
    c.assert_equal("write")


def small(hd):
    """Zeros and values that round to 0, of either sign: in groups whose scale is 0, in groups with ordinary values, -0 itself."""
    rng = np.random.default_rng(hd + 1)
    x = rows_of(4, N, HKV, HKV, hd).reshape(N, -1, hd // 16, 16)
    sign = np.where(rng.random(x.shape) < 0.5, -1.0, 1.0).astype(np.float32)
    x[:10] = 1e-5 * sign[:10]                                      # below 6 * 2^-10: a scale of 0
    x[10:20, ..., :8] = 1e-3 * sign[10:20, ..., :8]                # below a quarter of a scale
    x[20:25] = 0.0 * sign[20:25]
    x[25:30, ..., ::2] = 0.0 * sign[25:30, ..., ::2]
    x[30:34, ..., ::5] = 1e-40 * sign[30:34, ..., ::5]             # (not normal in fp32)
    x[34] = 6 * 2.0 ** -10 * sign[34]                              # on the border to the smallest scale
    return gen.bf16_round(x.reshape(N, -1, hd))


@pytest.mark.parametrize("hd", [64, 128])
def test_codes_of_zeros(pdlib, hd):
    """The bytes themselves: a scale of 0 has codes of 0, under any other a negative value that rounds to 0 keeps its sign, and a
    zero of either sign is code 0."""
    for exps in ((0, 1), (-4, 3)):
        x = small(hd)
        x[:, HKV:] = gen.bf16_round(x[:, HKV:] * np.exp2(np.array(exps * 2))[:, None].astype(np.float32))
        for pairs, rot in ((False, 0), (True, 0), (False, hd), (True, hd // 2)):
            c, t = cache(pdlib, hd, exps), Transform(pdlib, hd, rot, N, pairs, gains=False)
            append(pdlib, c, t, x, [0], [0, N], q=False)
            expect(c, t, x, [0], [0, N])
            check_bytes(c)
        c = cache(pdlib, hd, exps)
        write(pdlib, c, x[:, HKV:2 * HKV], x[:, 2 * HKV:])
        check_bytes(c)


def check_bytes(c):
    for d, ds, h, hs in ((c.dk, c.dks, c.k, c.ks), (c.dv, c.dvs, c.v, c.vs)):
        got, scales = d.cpu().numpy(), ds.cpu().numpy()
        np.testing.assert_array_equal(scales, hs)
        zero = np.repeat(hs == 0, 8, axis=-1)
        assert zero.any() and not got[zero].any()
        live = np.repeat((hs & 0x7F) != 0x7F, 8, axis=-1)
        np.testing.assert_array_equal(got[live], h[live])

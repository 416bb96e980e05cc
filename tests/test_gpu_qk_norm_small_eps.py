"""GPU: the norm of q and k heads where eps is far below what fp32 holds, and where mean(x^2) + eps is as small as is allowed."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from kv4_util import Cache4, Transform, transform_bound
from test_gpu_kv4_append import append, expect

pytestmark = pytest.mark.gpu
HQ, HKV, HD, N = 4, 2, 64, 6


def rows(size):
    x = gen.normal_bf16(3, gen.S_X, (N, HQ + 2 * HKV, HD), 1.0)
    x[:3] = gen.bf16_round(x[:3] * np.float32(size))
    x[3] = 0                                         # (a padded row)
    x[4, ::2] = 0
    return x


@pytest.mark.parametrize("eps,size", [(1e-50, 1e-17), (1e-46, 1.0), (1e-44, 1e-17), (1e-30, 1e-20), (1e-36, 1e-25)])
def test_heads_of_zeros_stay_zero(pdlib, eps, size):
    x = rows(size)
    for pairs, rot in ((False, HD), (True, 32)):
        t = Transform(pdlib, HD, rot, 16, pairs, eps=eps)
        cfg = pdlib.LayerConfig(HQ * HD, HQ, HKV, HD, 64)
        q, k = empty_bf16(N, HQ * HD), empty_bf16(N, HKV * HD)
        width = (HQ + 2 * HKV) * HD
        pdlib.pd_qk_norm_rope(cfg, t.struct, to_dev(x.reshape(N, width)), width, q, HQ * HD, k, HKV * HD, i32_dev(np.arange(N)), N)
        for got, heads, f in ((from_dev(q), x[:, :HQ], t.q), (from_dev(k), x[:, HQ:HQ + HKV], t.k)):
            got = got.reshape(heads.shape)
            y, mag = f(heads, np.arange(N))
            assert (np.abs(got - y) <= transform_bound(y, mag)).all()
            assert not got[3].any() and not got[4, ::2].any()
        c = Cache4(pdlib, HKV, HD, 16, [N], seed=2).upload()
        q = append(pdlib, c, t, x, [0], [0, N])
        expect(c, t, x, [0], [0, N], q)
        c.assert_equal()

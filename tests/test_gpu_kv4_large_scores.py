"""GPU: decode attention over the 4-bit cache where |q| * 2^k_exp comes up to its stated bound, 2^110: scores stay finite, and the
key with the largest takes all."""
import numpy as np
import pytest

import pd_inputs as gen
from kv4_util import Cache4
from oracle import paged4
from test_gpu_kv4_attention import decode, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new", [1, 3])
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("k_exp", [(30, 0), (-30, 12)])
def test_up_to_the_bound(pdlib, hq, hkv, hd, n_new, k_exp):
    lens = [2600, 61]
    c = Cache4(pdlib, hkv, hd, 32, lens, seed=hd)
    c.k_exp = np.array(k_exp, np.int32)
    c.ke = paged4.head_exp(c.k_exp, hkv)
    c.fill(lens, np.random.default_rng(hd), 0.5)
    # some keys at the largest value that can be stored, in all features
    rng = np.random.default_rng(1)
    for s, n in enumerate(lens):
        for at in range(3, n - n_new, 17):
            x = 2688.0 * np.where(rng.random((1, hkv, hd)) < 0.5, -1, 1) * np.exp2(c.ke)[:, None]
            paged4.append(c.k, c.ks, c.table[s], at, x, c.ke)
    c.upload()
    q = queries(90, 2, n_new, hq, hd).astype(np.float64)
    q /= np.abs(q).max(axis=-1, keepdims=True)
    group = hq // hkv
    for h in range(hq):
        q[:, :, h] *= min(2.0 ** (110 - int(c.ke[h // group])) * (1 - 2.0 ** -8), 3.3895e38)
    q = gen.bf16_round(q)
    kv_len = [n - n_new for n in lens]
    for most in (lens[0], 2048, n_new):            # parts that a kernel joins, parts that meet in a cluster, and one
        got = decode(pdlib, c, hq, q, kv_len, n_new, max_kv=most)
        for s, n in enumerate(lens):
            k, v = c.kv(s, n)
            for j in range(n_new):
                for h in range(hq):
                    score = k[:kv_len[s] + j + 1, h // group] @ q[s, j, h].astype(np.float64)
                    order = np.argsort(score)
                    assert score[order[-1]] - score[order[-2]] > 1e-4 * np.abs(score).max()   # (beyond the rounding of fp32 sums)
                    np.testing.assert_array_equal(got[s, j, h], v[order[-1], h // group].astype(np.float32), err_msg=f"{most} {s} {j} {h}")

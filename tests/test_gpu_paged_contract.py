"""GPU: what the header says of the 8-bit serving calls at places that the other tests do not reach."""
import numpy as np
import pytest

from gpu_util import from_dev
from oracle import paged
from paged_util import BF16
from test_gpu_paged_append import THETA, Appender, qkv_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (13, 1, 128)])
@pytest.mark.parametrize("runs", [False, True])
def test_append_beyond_the_table_still_writes_q(pdlib, hq, hkv, hd, runs):
    """Positions within the rotation table, but behind the last page of the page table: q is written, k and v are left out."""
    p = 16
    ap = Appender(pdlib, hq, hkv, hd, 64, p, [p, p, p], seed=8, extra_cols=0)       # a table of one page each
    kv, n = [p, 63, 3 * p - 1], 1
    ap.c.upload()
    rows = qkv_rows(11, 3 * n, hq, hkv, hd)
    q = ap(rows, kv, [n] * 3 if runs else None, oracle=False)
    assert int(ap.err.item()) == 2
    ap.c.assert_equal("cache")
    ref = paged.rotate(rows[:, :hq], kv, THETA)
    half = np.abs(rows[:, :hq, :hd // 2]) + np.abs(rows[:, :hq, hd // 2:])
    bound = BF16 * np.abs(ref) + 2.0 ** -21 * np.concatenate([half, half], -1)
    assert np.all(np.abs(from_dev(q[:3]).reshape(ref.shape) - ref) <= bound)

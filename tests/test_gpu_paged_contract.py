"""GPU: what the header says of the 8-bit serving calls at places that the other tests do not reach."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import paged
from paged_util import BF16, Cache
from test_gpu_paged_append import THETA, Appender, qkv_rows
from test_gpu_paged_attention import check_decode, check_prefill, decode, prefill

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


@pytest.mark.parametrize("hq,hkv,hd,page_len,batch,max_kv,launches", [
    (16, 1, 128, 16, 130, 600, 2),      # two parts of 2080 rows: the join with a warp per row
    (64, 8, 64, 32, 33, 8192, 2),       # the same, parts cut for the length bound
    (32, 8, 128, 64, 2, 1500, 2),       # few rows: the join with a block per row
    (32, 8, 128, 64, 40, 250, 1)])      # one part
def test_decode_result_at_any_address(pdlib, hq, hkv, hd, page_len, batch, max_kv, launches):
    """`out` starts between two 4-byte words: the same bits as at an aligned address, and nothing in front of it or behind."""
    import torch
    rng = np.random.default_rng(batch)
    kv_len = [int(v) for v in rng.integers(-1, min(max_kv, 400), batch)]
    c = Cache(pdlib, hkv, hd, page_len, [n + 1 for n in kv_len], seed=batch, extra_cols=max_kv // page_len + 1)
    c.fill([n + 1 for n in kv_len], rng, 0.5)
    c.upload()
    q = gen.normal_bf16(103, gen.S_X, (batch, hq, hd), 1.0, sub=batch)
    want = decode(pdlib, c, hq, q, kv_len, max_kv=max_kv)
    check_decode(c, hq, q[:9], kv_len[:9], want)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = pdlib.pd_paged_decode_attention_workspace_bytes(cfg, batch, max_kv)
    ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    for shift in (1, 2, 3):
        buf = empty_bf16(batch * hq * hd + 8)
        out = buf[shift:shift + batch * hq * hd]
        assert out.data_ptr() % 8 == 2 * shift
        before = pdlib.pd_launch_count()
        pdlib.pd_paged_decode_attention(cfg, to_dev(q.reshape(batch, -1)), hq * hd, out, i32_dev(kv_len), batch, max_kv, c.struct, ws, need)
        torch.cuda.synchronize()
        assert pdlib.pd_launch_count() - before == launches
        np.testing.assert_array_equal(from_dev(out).reshape(want.shape), want)
        assert not buf[:shift].any() and not buf[shift + batch * hq * hd:].any()


@pytest.mark.parametrize("hq,hkv,hd,new,prefix", [(8, 2, 64, [0, 3, 0, 2], [-1, 40, -1, 0]), (32, 8, 128, [0, 70, 0, 130, 0], [-7, 100, -1, 5, 1 << 30])])
def test_prefill_of_a_padded_batch(pdlib, hq, hkv, hd, new, prefix):
    """Requests without rows may have any prefix: the others get what they get without them."""
    rng = np.random.default_rng(hd)
    total = [a + b if a else 1 for a, b in zip(new, prefix)]
    c = Cache(pdlib, hkv, hd, 32, total, seed=hd)
    c.fill(total, rng, 0.5)
    c.upload()
    q = gen.normal_bf16(104, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    got = prefill(pdlib, c, hq, q, new, prefix)
    check_prefill(c, hq, q, new, prefix, got, rows=8)
    np.testing.assert_array_equal(got, prefill(pdlib, c, hq, q, new, [b if a else 0 for a, b in zip(new, prefix)]))

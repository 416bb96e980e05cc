"""GPU: calls of the 8-bit paged cache at the edges of what is allowed: very many requests, large batches of short sequences, a
length bound far above the lengths, streams given by the caller, heads of 64 in a group of 16."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import paged
from paged_util import BF16, F16, Cache, assert_within, attention_bound
from test_gpu_paged_append import Appender, qkv_rows
from test_gpu_paged_attention import check_decode, check_prefill, decode, prefill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_req", [33, 1500])
def test_append_of_very_many_requests(pdlib, n_req):
    """More requests than one, and than two, rounds of the search take."""
    rng = np.random.default_rng(n_req)
    kv = [int(v) for v in rng.integers(0, 20, n_req)]
    new = [int(v) for v in rng.integers(0, 4, n_req)]
    new[0] = new[-1] = 0
    ap = Appender(pdlib, 2, 1, 64, 64, 16, [a + b for a, b in zip(kv, new)], seed=1)
    ap.c.fill(kv, rng)
    ap.c.upload()
    ap(qkv_rows(3, sum(new), 2, 1, 64), kv, new)
    ap.c.assert_equal()
    # and one token each
    ap2 = Appender(pdlib, 2, 1, 64, 64, 16, [a + 1 for a in kv], seed=2)
    ap2.c.fill(kv, rng)
    ap2.c.upload()
    ap2(qkv_rows(4, n_req, 2, 1, 64), kv)
    ap2.c.assert_equal()
    assert int(ap.err.item()) == 0 and int(ap2.err.item()) == 0


def test_attention_of_very_many_requests(pdlib):
    rng = np.random.default_rng(5)
    n_req = 1100
    prefix = [int(v) for v in rng.integers(0, 60, n_req)]
    new = [int(v) for v in rng.integers(0, 3, n_req)]
    c = Cache(pdlib, 1, 64, 16, [a + b for a, b in zip(prefix, new)], seed=3)
    c.fill([a + b for a, b in zip(prefix, new)], rng, 0.5)
    c.upload()
    q = gen.normal_bf16(92, gen.S_X, (sum(new), 4, 64), 1.0)
    check_prefill(c, 4, q, new, prefix, prefill(pdlib, c, 4, q, new, prefix))
    kv_len = [a + b - 1 for a, b in zip(prefix, new)]   # -1 where a sequence is empty
    qd = gen.normal_bf16(93, gen.S_X, (n_req, 4, 64), 1.0)
    check_decode(c, 4, qd, kv_len, decode(pdlib, c, 4, qd, kv_len))


def test_length_bound_far_above_the_lengths(pdlib):
    """max_kv_len of a captured program is a capacity."""
    hq, hkv, hd = 8, 2, 64
    kv_len = [5, 300, -1, 1000]
    c = Cache(pdlib, hkv, hd, 64, [n + 1 for n in kv_len], seed=4, extra_cols=2000)
    c.fill([max(0, n + 1) for n in kv_len], np.random.default_rng(4), 0.5)
    c.upload()
    q = gen.normal_bf16(94, gen.S_X, (4, hq, hd), 1.0)
    check_decode(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len, max_kv=c.width * 64))


@pytest.mark.parametrize("hq,hd", [(16, 64), (13, 128)])
def test_wide_groups_over_runs(pdlib, hq, hd):
    new, prefix = [1, 7, 40, 300], [500, 0, 100, 33]
    c = Cache(pdlib, 1, hd, 16, [a + b for a, b in zip(new, prefix)], seed=5)
    c.fill([a + b for a, b in zip(new, prefix)], np.random.default_rng(5), 0.5)
    c.upload()
    q = gen.normal_bf16(95, gen.S_X, (sum(new), hq, hd), 1.0)
    check_prefill(c, hq, q, new, prefix, prefill(pdlib, c, hq, q, new, prefix), rows=5)


def test_caller_given_streams_are_used(pdlib):
    """Work goes to the stream that is given: behind what that stream waits for, not behind the default stream."""
    import torch
    hq, hkv, hd = 8, 2, 64
    c = Cache(pdlib, hkv, hd, 16, [100, 40], seed=6)
    c.fill([100, 40], np.random.default_rng(6))
    c.upload()
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    q = gen.normal_bf16(96, gen.S_X, (2, hq, hd), 1.0)
    want = decode(pdlib, c, hq, q, [99, 39])
    s = torch.cuda.Stream()
    dq, out, kv = torch.zeros_like(to_dev(q.reshape(2, -1))), empty_bf16(2, hq * hd), i32_dev([0, 0])
    src, src_kv = to_dev(q.reshape(2, -1)), i32_dev([99, 39])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)     # the inputs arrive late, on the stream
        dq.copy_(src)
        kv.copy_(src_kv)
    need = pdlib.pd_paged_decode_attention_workspace_bytes(cfg, 2, 100)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    pdlib.pd_paged_decode_attention(cfg, dq, hq * hd, out, kv, 2, 100, c.struct, ws, need, stream=s)
    s.synchronize()
    np.testing.assert_array_equal(from_dev(out), want)


def test_gradually_growing_values_lose_nothing(pdlib):
    """A page filled token by token with sizes that double each time: what the first tokens keep is what one rounding to the
    final scale leaves, up to the subnormal codes."""
    hkv, hd, p = 2, 64, 16
    ap = Appender(pdlib, 2, hkv, hd, 32, p, [16], seed=7)
    rows = qkv_rows(8, 16, 2, hkv, hd, 0.0)
    for i in range(16):
        rows[i] *= np.float32(2.0 ** (i / 2))
    rows = gen.bf16_round(rows)
    for i in range(16):
        ap(rows[i:i + 1], [i])
    ap.c.assert_equal()
    got = paged.sequence(ap.c.v, ap.c.vs, ap.c.table[0], 16)
    want = rows[:, 2 + hkv:]
    step = ap.c.vs[ap.c.table[0, 0]][:, None] * 2.0 ** -9
    assert np.all(np.abs(got - want) <= 2.0 ** -4 * np.abs(want) + step)


@pytest.mark.parametrize("hq,hkv,hd,new,prefix", [
    (16, 8, 128, [1400], [3500]),                         # 88 blocks of rows and heads for 148 SMs: all cut
    (16, 8, 64, [2600], [1900]),                          # 168: the first three blocks of tokens cut
    (16, 8, 128, [200, 0, 1000, 1500], [3000, 5, 0, 900]),
    (12, 6, 64, [130, 1, 129, 3000], [2500, 2600, 40, 0])])
def test_key_ranges_cut_behind_the_last_full_turn(pdlib, hq, hkv, hd, new, prefix):
    total = [a + b for a, b in zip(new, prefix)]
    c = Cache(pdlib, hkv, hd, 128, total, seed=hd + len(new))
    c.fill(total, np.random.default_rng(8), 0.5, pages=1.0)
    c.upload()
    q = gen.normal_bf16(97, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    got = prefill(pdlib, c, hq, q, new, prefix)
    check_prefill(c, hq, q, new, prefix, got, rows=10)
    np.testing.assert_array_equal(got, prefill(pdlib, c, hq, q, new, prefix, pad=8))

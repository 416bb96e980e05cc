"""GPU: decode and prefill attention over the 8-bit paged KV cache against the float64 oracle on the same cached values.  Rows
without a token hold NaN codes and unused table entries are -1: neither may reach an output."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import paged
from paged_util import BF16, F16, Cache, assert_within, attention_bound

pytestmark = pytest.mark.gpu


def decode(pd, c, hq, q, kv_len, max_kv=None, pad=0, err=None, stream=None):
    import torch
    b = len(kv_len)
    cfg = pd.LayerConfig(hq * c.hd, hq, c.hkv, c.hd, 64)
    width = hq * c.hd
    flat = np.full((b, width + pad), np.nan, np.float32)
    flat[:, :width] = q.reshape(b, width)
    max_kv = max_kv or max(1, max(kv_len) + 1)
    ws_bytes = pd.pd_paged_decode_attention_workspace_bytes(cfg, b, max_kv)
    ws = torch.full((max(ws_bytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    out = empty_bf16(b + 1, width)
    pd.pd_paged_decode_attention(cfg, to_dev(flat), width + pad, out, i32_dev(kv_len), b, max_kv, c.struct, ws, ws_bytes, err_word=err)
    torch.cuda.synchronize()
    assert not out[b].any()
    return from_dev(out[:b])


def check_decode(c, hq, q, kv_len, got):
    for s, n in enumerate(kv_len):
        if n < 0:
            assert not got[s].any()
            continue
        k, v = c.kv(s, n + 1)
        o, spread, score = paged.attend(q[s:s + 1].reshape(1, hq, c.hd), k, v, [n])
        assert_within(got[s].reshape(1, hq, c.hd), o, attention_bound(o, spread, score, F16), f"sequence {s} ({n + 1} keys)")


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (64, 8, 128), (4, 4, 128), (16, 1, 128), (16, 1, 64), (9, 1, 64), (11, 1, 128),
                                       (6, 2, 64)])
@pytest.mark.parametrize("page_len", [16, 32, 64, 128])
def test_decode_lengths(pdlib, hq, hkv, hd, page_len):
    """One key to several splits, every tail of the 16-key tile and of the page, padding rows."""
    kv_len = [0, 1, 14, 15, 16, 63, 64, 65, -1, 127, 128, 300, 1111, 255]
    c = Cache(pdlib, hkv, hd, page_len, [max(0, n + 1) for n in kv_len], seed=hq + page_len)
    c.fill([max(0, n + 1) for n in kv_len], np.random.default_rng(hd + page_len), 0.5)
    c.upload()
    q = gen.normal_bf16(70, gen.S_X, (len(kv_len), hq, hd), 1.0, sub=hd)
    got = decode(pdlib, c, hq, q, kv_len, pad=8)
    check_decode(c, hq, q, kv_len, got)
    np.testing.assert_array_equal(got, decode(pdlib, c, hq, q, kv_len))               # deterministic, whatever the pitch
    whole = decode(pdlib, c, hq, q, kv_len, max_kv=1)                                 # no split: a bound that is too small
    check_decode(c, hq, q, kv_len, whole)


@pytest.mark.parametrize("hq,hkv,hd,page_len,n", [(32, 8, 128, 64, 20011), (8, 2, 64, 16, 9000), (16, 1, 128, 32, 5000)])
def test_decode_long_sequence(pdlib, hq, hkv, hd, page_len, n):
    c = Cache(pdlib, hkv, hd, page_len, [n, 40], seed=n)
    c.fill([n, 40], np.random.default_rng(n), 0.5)
    c.upload()
    q = gen.normal_bf16(71, gen.S_X, (2, hq, hd), 1.5, sub=n)
    check_decode(c, hq, q, [n - 1, 39], decode(pdlib, c, hq, q, [n - 1, 39]))


def test_decode_scales_far_apart_and_large_queries(pdlib):
    """Pages whose scales differ by many octaves, queries from 1e-20 to 1e20 (the softmax is then one-hot or flat)."""
    hq, hkv, hd = 8, 2, 64
    kv_len = [200, 333, 90, 17]
    c = Cache(pdlib, hkv, hd, 16, [n + 1 for n in kv_len], seed=12)
    c.fill([n + 1 for n in kv_len], np.random.default_rng(12), 1.0, pages=6.0)
    # K of ordinary size again (scores stay comparable), V as it is
    rng = np.random.default_rng(13)
    for s, n in enumerate(kv_len):
        paged.append(c.k, c.ks, c.table[s], 0, gen.bf16_round(rng.standard_normal((n + 1, hkv, hd))))
    c.upload()
    q = gen.normal_bf16(72, gen.S_X, (4, hq, hd), 1.0)
    q[1] = gen.bf16_round(q[1] * np.float32(1e-20))
    q[2] = gen.bf16_round(q[2] * np.float32(100.0))
    q[3] = 0.0
    check_decode(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len))


def test_decode_non_finite_values_stay_in_their_row(pdlib):
    hq, hkv, hd = 8, 2, 64
    c = Cache(pdlib, hkv, hd, 16, [50, 50, 50], seed=14)
    c.fill([50, 50, 50], np.random.default_rng(14))
    c.upload()
    q = gen.normal_bf16(73, gen.S_X, (3, hq, hd), 1.0)
    clean = decode(pdlib, c, hq, q, [49, 49, 49])
    c.v[c.table[1, 2], 1, 3, 7] = 0x7F                  # a NaN in a visible V row of the second KV head
    c.upload()
    q[2, 3, 5] = np.nan
    got = decode(pdlib, c, hq, q, [49, 49, 49])
    np.testing.assert_array_equal(got[0], clean[0])
    bad = np.zeros((hq, hd), bool)
    bad[4:, 7] = True
    np.testing.assert_array_equal(np.isnan(got[1].reshape(hq, hd)), bad)
    assert np.isnan(got[2].reshape(hq, hd)[3]).all()
    np.testing.assert_array_equal(np.delete(got[2].reshape(hq, hd), 3, 0), np.delete(clean[2].reshape(hq, hd), 3, 0))


def test_decode_bad_pages_and_lengths_are_reported(pdlib):
    import torch
    hq, hkv, hd, p = 8, 2, 64, 16
    kv_len = [79, 60, 200]
    c = Cache(pdlib, hkv, hd, p, [80, 80, 80], seed=15, extra_cols=0)
    c.fill([80, 80, 80], np.random.default_rng(15))
    full = c.table.copy()
    c.table[0, 1], c.table[1, 0] = -1, c.n_pages
    c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = gen.normal_bf16(74, gen.S_X, (3, hq, hd), 1.0)
    got = decode(pdlib, c, hq, q, kv_len, max_kv=80, err=err)
    assert int(err.item()) == 2
    c.table = full
    for s, keys in enumerate([np.r_[0:16, 32:80], np.r_[16:61], np.r_[0:80]]):   # without the bad page; the table's end
        k, v = c.kv(s, 80)
        o, spread, score = paged.attend(q[s:s + 1], k[keys], v[keys], [len(keys) - 1])
        assert_within(got[s].reshape(1, hq, hd), o, attention_bound(o, spread, score, F16), f"sequence {s}")
    # every page bad: nothing to attend to
    c.table = np.full_like(full, -7)
    c.upload()
    assert not decode(pdlib, c, hq, q, kv_len, max_kv=80, err=err).any()


def test_decode_pool_beyond_32_bit_offsets(pdlib):
    """A pool of more than 2^32 code bytes, the sequence's pages at its end."""
    import torch
    hq, hkv, hd, p, n = 32, 8, 128, 128, 700
    n_pages = (1 << 32) // (hkv * p * hd) + 200
    c = Cache(pdlib, hkv, hd, p, [n], seed=16)
    c.fill([n], np.random.default_rng(16))
    big = [torch.empty((n_pages, hkv, p, hd), dtype=torch.uint8, device="cuda") for _ in range(2)]
    sc = [torch.empty((n_pages, hkv), device="cuda") for _ in range(2)]
    table = c.table.copy()
    at = np.array([n_pages - 1 - 3 * i for i in range(c.width - 1)])
    for i, page in enumerate(at):
        for dst, src in ((big[0], c.k), (big[1], c.v), (sc[0], c.ks), (sc[1], c.vs)):
            dst[int(page)] = torch.from_numpy(src[c.table[0, i]].copy()).cuda()
        table[0, i] = page
    c.struct = pdlib.paged_kv_cache_struct(big[0], big[1], sc[0], sc[1], keep := i32_dev(table), n_pages, p, 1, c.width)
    q = gen.normal_bf16(75, gen.S_X, (1, hq, hd), 1.0)
    check_decode(c, hq, q, [n - 1], decode(pdlib, c, hq, q, [n - 1]))
    del keep


def test_decode_batch_on_a_side_stream_and_replayed(pdlib):
    import torch
    hq, hkv, hd = 32, 8, 128
    kv_len = [int(t) for t in gen.uniform_lengths(5, 48, 0, 900)]
    c = Cache(pdlib, hkv, hd, 64, [n + 1 for n in kv_len], seed=17)
    c.fill([n + 1 for n in kv_len], np.random.default_rng(17), 0.5)
    c.upload()
    q = gen.normal_bf16(76, gen.S_X, (48, hq, hd), 1.0)
    ref = decode(pdlib, c, hq, q, kv_len)
    sel = [0, 7, 47]
    for s in sel:
        k, v = c.kv(s, kv_len[s] + 1)
        o, spread, score = paged.attend(q[s:s + 1], k, v, [kv_len[s]])
        assert_within(ref[s].reshape(1, hq, hd), o, attention_bound(o, spread, score, F16), f"sequence {s}")
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    m = max(kv_len) + 1
    need = pdlib.pd_paged_decode_attention_workspace_bytes(cfg, 48, m)
    dq, dkv, out = to_dev(q.reshape(48, -1)), i32_dev([0] * 48), empty_bf16(48, hq * hd)
    ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    pdlib.pd_paged_decode_attention(cfg, dq, hq * hd, out, dkv, 48, m, c.struct, ws, need)   # (kernel attributes are set outside the capture)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pdlib.pd_paged_decode_attention(cfg, dq, hq * hd, out, dkv, 48, m, c.struct, ws, need)
    dkv.copy_(i32_dev(kv_len))       # lengths of the replay, not of the capture
    g.replay()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(from_dev(out), ref)


# ---------------------------------------------------------------------------------------------------------- prefill
def prefill(pd, c, hq, q, new, prefix, pad=0, err=None, no_prefix=False):
    import torch
    t, width = q.shape[0], hq * c.hd
    cfg = pd.LayerConfig(width, hq, c.hkv, c.hd, 64)
    cu = [0] + [int(v) for v in np.cumsum(new)]
    flat = np.full((t, width + pad), np.nan, np.float32)
    flat[:, :width] = q.reshape(t, width)
    need = pd.pd_paged_prefill_attention_workspace_bytes(cfg, len(new), max(a + b for a, b in zip(new, prefix)))
    ws = torch.full((max(256, need),), 0xFF, dtype=torch.uint8, device="cuda")     # NaN wherever it is read unwritten
    out = empty_bf16(t + 1, width)
    e = err if err is not None else torch.zeros(1, dtype=torch.int32, device="cuda")
    pd.pd_paged_prefill_attention(cfg, to_dev(flat), width + pad, out, i32_dev(cu), cu, None if no_prefix else i32_dev(prefix),
                                  None if no_prefix else prefix, c.struct, ws, need, err_word=e)
    torch.cuda.synchronize()
    assert err is not None or int(e.item()) == 0
    assert not out[t].any()
    return from_dev(out[:t])


def check_prefill(c, hq, q, new, prefix, got, rows=None):
    at = 0
    for s, (n, pre) in enumerate(zip(new, prefix)):
        if n:
            k, v = c.kv(s, pre + n)
            sel = np.arange(n) if rows is None or n <= rows else np.unique(np.r_[0, n - 1, np.random.default_rng(s).integers(0, n, rows)])
            o, spread, score = paged.attend(q[at + sel], k, v, pre + sel)
            # (weights may be held in bf16 here)
            assert_within(got[at + sel].reshape(len(sel), hq, c.hd), o, attention_bound(o, spread, score, BF16), f"request {s}")
        at += n


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (16, 1, 128), (3, 3, 64), (64, 8, 128)])
@pytest.mark.parametrize("page_len", [16, 32, 64, 128])
def test_prefill_lengths(pdlib, hq, hkv, hd, page_len):
    new = [1, 2, 0, 5, 17, 130, 1, 260]
    prefix = [0, 1, 30, 127, page_len, 0, 400, 300]
    c = Cache(pdlib, hkv, hd, page_len, [a + b for a, b in zip(new, prefix)], seed=hq + page_len)
    c.fill([a + b for a, b in zip(new, prefix)], np.random.default_rng(hd + page_len), 0.5)
    c.upload()
    q = gen.normal_bf16(80, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    check_prefill(c, hq, q, new, prefix, prefill(pdlib, c, hq, q, new, prefix, pad=8), rows=6)


@pytest.mark.parametrize("new,prefix", [([1], [0]), ([1, 1, 1], [0, 15, 16]), ([4] * 6, [0, 3, 100, 255, 256, 1000]), ([3, 1, 16, 7], [2000, 0, 17, 333])])
def test_prefill_short_runs(pdlib, new, prefix):
    hq, hkv, hd = 32, 8, 128
    c = Cache(pdlib, hkv, hd, 32, [a + b for a, b in zip(new, prefix)], seed=len(new))
    c.fill([a + b for a, b in zip(new, prefix)], np.random.default_rng(3), 0.5)
    c.upload()
    q = gen.normal_bf16(81, gen.S_X, (sum(new), hq, hd), 1.0, sub=len(new))
    got = prefill(pdlib, c, hq, q, new, prefix)
    check_prefill(c, hq, q, new, prefix, got)
    np.testing.assert_array_equal(got, prefill(pdlib, c, hq, q, new, prefix, pad=8))


def test_prefill_long_prompt_and_no_prefix(pdlib):
    hq, hkv, hd, new = 8, 2, 64, [1500, 700]
    c = Cache(pdlib, hkv, hd, 64, new, seed=21)
    c.fill(new, np.random.default_rng(21), 0.5)
    c.upload()
    q = gen.normal_bf16(82, gen.S_X, (sum(new), hq, hd), 1.0)
    got = prefill(pdlib, c, hq, q, new, [0, 0], no_prefix=True)
    check_prefill(c, hq, q, new, [0, 0], got, rows=24)


def test_prefill_of_one_row_is_decode(pdlib):
    """One fresh row per request: the same definition as the decode call."""
    hq, hkv, hd = 64, 8, 128
    kv_len = [0, 15, 200, 513]
    c = Cache(pdlib, hkv, hd, 16, [n + 1 for n in kv_len], seed=22)
    c.fill([n + 1 for n in kv_len], np.random.default_rng(22), 0.5)
    c.upload()
    q = gen.normal_bf16(83, gen.S_X, (4, hq, hd), 1.0)
    a, b = decode(pdlib, c, hq, q, kv_len), prefill(pdlib, c, hq, q, [1] * 4, kv_len)
    for s, n in enumerate(kv_len):
        k, v = c.kv(s, n + 1)
        o, spread, score = paged.attend(q[s:s + 1], k, v, [n])
        bound = attention_bound(o, spread, score, BF16)
        assert_within(a[s].reshape(o.shape), b[s].reshape(o.shape).astype(np.float64), 2 * bound, f"sequence {s}")


def test_prefill_bad_page_is_reported(pdlib):
    import torch
    c = Cache(pdlib, 2, 64, 16, [40, 40], seed=23)
    c.fill([40, 40], np.random.default_rng(23))
    c.table[1, 1] = -1
    c.upload()
    q = gen.normal_bf16(84, gen.S_X, (60, 8, 64), 1.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = prefill(pdlib, c, 8, q, [30, 30], [10, 10], err=err)
    assert int(err.item()) == 2
    check_prefill(c, 8, q[:30], [30], [10], got[:30])      # the other request is untouched


def test_prefill_replayed(pdlib):
    import torch
    hq, hkv, hd, new, prefix = 8, 2, 64, [200, 9], [33, 500]
    c = Cache(pdlib, hkv, hd, 32, [233, 509], seed=24)
    c.fill([233, 509], np.random.default_rng(24))
    c.upload()
    q = gen.normal_bf16(85, gen.S_X, (209, hq, hd), 1.0)
    ref = prefill(pdlib, c, hq, q, new, prefix)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(cfg, 2, 509)
    ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    dq, out, cu, pre = empty_bf16(209, hq * hd), empty_bf16(209, hq * hd), i32_dev([0, 200, 209]), i32_dev(prefix)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pdlib.pd_paged_prefill_attention(cfg, dq, hq * hd, out, cu, [0, 200, 209], pre, prefix, c.struct, ws, need)
    dq.copy_(to_dev(q.reshape(209, -1)))
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(from_dev(out), ref)


def test_prefill_nan_key_at_every_position(pdlib):
    """A NaN in the cached K of one key makes the rows that see it NaN and leaves the others alone, wherever the key stands in
    a tile (the weights of a tile's keys are not all computed in the same way)."""
    hq, hkv, hd, page_len, new, prefix = 8, 2, 64, 32, 40, 120
    c = Cache(pdlib, hkv, hd, page_len, [new + prefix], seed=77)
    c.fill([new + prefix], np.random.default_rng(77), 0.5)
    clean = c.k.copy()
    q = gen.normal_bf16(91, gen.S_X, (new, hq, hd), 1.0)
    for key in list(range(64)) + [prefix - 1, prefix, prefix + 7, prefix + new - 1]:
        c.k = clean.copy()
        c.k[c.table[0][key // page_len], 1, key % page_len, key % hd] = 0x7F  # the second KV head: query heads 4 .. 7
        c.upload()
        got = np.asarray(prefill(pdlib, c, hq, q, [new], [prefix]), dtype=np.float64).reshape(new, hq, hd)
        sees = np.arange(new) + prefix >= key
        assert np.isnan(got[sees][:, 4:]).all(), key
        assert np.isfinite(got[:, :4]).all() and np.isfinite(got[~sees]).all(), key


@pytest.mark.parametrize("hq,hkv,hd,new,prefix", [(8, 2, 64, [40, 3, 16], [120, 0, 37]), (32, 8, 128, [70, 1, 130], [0, 5, 300]),
                                                  (4, 4, 128, [4, 2, 1], [500, 30, 0])])
def test_prefill_nan_value_reaches_only_the_rows_that_see_it(pdlib, hq, hkv, hd, new, prefix):
    """NaN entries of V make their feature NaN in the rows that see the key; a row before it is left alone, although it shares
    a tile with the key (its weight there is 0)."""
    c = Cache(pdlib, hkv, hd, 32, [a + b for a, b in zip(new, prefix)], seed=hd + hq)
    c.fill([a + b for a, b in zip(new, prefix)], np.random.default_rng(hd), 0.5)
    clean = c.v.copy()
    q = gen.normal_bf16(92, gen.S_X, (sum(new), hq, hd), 1.0, sub=hq)
    want = np.asarray(prefill(pdlib, c.upload(), hq, q, new, prefix), dtype=np.float64).reshape(sum(new), hq, hd)
    start = np.cumsum([0] + new)
    for step in (1, 5, 29):
        c.v = clean.copy()
        bad = np.zeros((sum(new), hq, hd), bool)
        for s, (n, pre) in enumerate(zip(new, prefix)):
            for i, key in enumerate(range(pre + n - 1, max(pre - 20, -1), -step)):
                head, d = i % hkv, (7 * i + 3) % hd
                c.v[c.table[s][key // 32], head, key % 32, d] = 0xFF if i % 2 else 0x7F
                rows = start[s] + np.arange(n)[pre + np.arange(n) >= key]
                bad[np.ix_(rows, np.arange(head * hq // hkv, (head + 1) * hq // hkv), [d])] = True
        c.upload()
        got = np.asarray(prefill(pdlib, c, hq, q, new, prefix), dtype=np.float64).reshape(sum(new), hq, hd)
        np.testing.assert_array_equal(np.isnan(got), bad)
        np.testing.assert_array_equal(got[~bad], want[~bad])

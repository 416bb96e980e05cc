"""GPU: attention over pages whose V scales lie many octaves apart, by every kernel.  What a row gets must not depend on pages
that weigh nothing for it, nor on pages that only later rows see."""
import os
import subprocess
import sys

import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import paged
from paged_util import F16, Cache, assert_within, attention_bound
from test_gpu_paged_attention import decode, prefill

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def scaled_cache(pd, hkv, hd, page_len, total, octaves, rng, k_of_page=None):
    """Sequences of total[s] tokens whose V on page i is of size 2^octaves(s, i); K of page i is k_of_page(s, i) where that is
    not None."""
    c = Cache(pd, hkv, hd, page_len, total, seed=page_len + hd)
    for s, n in enumerate(total):
        for i in range(-(-n // page_len)):
            m = min(page_len, n - i * page_len)
            k = None if k_of_page is None else k_of_page(s, i)
            k = rng.standard_normal((m, hkv, hd)) if k is None else np.broadcast_to(k, (m, hkv, hd))
            v = rng.standard_normal((m, hkv, hd)) * 2.0 ** octaves(s, i)
            paged.append(c.k, c.ks, c.table[s], i * page_len, gen.bf16_round(k))
            paged.append(c.v, c.vs, c.table[s], i * page_len, gen.bf16_round(v))
    return c.upload()


def weight_floor(q, keys, vals, scale, top, pos):
    """What the smallest f16 numbers leave of softmax weights, times |v|: a weight is held as 2^7 times its share of the row's
    largest, half a step of the smallest numbers is 2^-25, so it is off by up to 2^-32 of the largest; where a page's V scale is
    folded into the weight (within 2^-10 of the largest scale) by as much more as that scale is smaller.  A weight below that may be
    lost: it is off by no more than itself.  `scale` [S, Hkv]: V's page scales, `top` [Hkv]: the largest one
    that the sequence has (other rows of a block may see it)."""
    n, hq, hd = q.shape
    g = hq // keys.shape[1]
    lost = 2.0 ** -32 * np.minimum(2.0 ** 10, top / scale)
    out = np.zeros((n, hq, hd))
    for h in range(hq):
        z = q[:, h].astype(np.float64) @ keys[:, h // g].T / np.sqrt(hd)
        z[np.arange(len(keys))[None] > np.asarray(pos)[:, None]] = -np.inf
        p = np.exp(z - z.max(axis=1, keepdims=True))
        out[:, h] = np.minimum(p, lost[:, h // g]) @ np.abs(vals[:, h // g])
    return out


def check(c, hq, q, first, n, s, got, what):
    """Rows `first` .. of sequence s (24 of them), to the bound of attention_bound and what the smallest weights lose."""
    keys, vals = c.kv(s, first + n)
    sel = np.unique(np.r_[0, n - 1, np.random.default_rng(n).integers(0, n, 22)]) if n > 24 else np.arange(n)
    pos, q, got = first + sel, q[sel], got[sel]
    o, spread, score = paged.attend(q, keys, vals, pos)
    scale = c.vs[c.table[s][np.arange(first + n) // c.page_len]].astype(np.float64)
    top = c.vs[c.table[s][c.table[s] >= 0]].max(axis=0).astype(np.float64)
    assert_within(got.reshape(len(sel), hq, c.hd), o, attention_bound(o, spread, score, F16) + weight_floor(q, keys, vals, scale, top, pos), what)


SHAPES = [(8, 2, 64, 16), (32, 8, 128, 64), (16, 1, 128, 16), (4, 4, 64, 32)]


@pytest.mark.parametrize("hq,hkv,hd,page_len", SHAPES)
@pytest.mark.parametrize("pages", [8.0, 25.0])
def test_runs_over_pages_of_random_size(pdlib, hq, hkv, hd, page_len, pages):
    rng = np.random.default_rng(int(pages) + hd)
    new, prefix = [40, 3, 150], [300, 90, 0]
    total = [a + b for a, b in zip(new, prefix)]
    size = {}
    c = scaled_cache(pdlib, hkv, hd, page_len, total, lambda s, i: size.setdefault((s, i), np.round(np.clip(pages * rng.standard_normal(), -55, 55))), rng)
    q = gen.normal_bf16(98, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    got, at = prefill(pdlib, c, hq, q, new, prefix), 0
    for s, (n, pre) in enumerate(zip(new, prefix)):
        check(c, hq, q[at:at + n], pre, n, s, got[at:at + n], f"request {s}")
        at += n


@pytest.mark.parametrize("hq,hkv,hd,page_len", SHAPES)
@pytest.mark.parametrize("octaves", [14, 17, 22, 26, 30, 90])
def test_a_large_page_without_weight_leaves_the_others_alone(pdlib, hq, hkv, hd, page_len, octaves):
    """Page 0 and page 3 are large, but their keys point away from every query (weights below 2^-60 octaves)."""
    rng = np.random.default_rng(octaves)
    new, prefix = [20, 130], [200, 77]
    sign = np.where(rng.random(hd) < 0.5, -1.0, 1.0)
    strong = np.ceil(octaves / 8 + 6)           # scores of -strong * sqrt(hd) below the others': 11 bits for each 8 octaves
    c = scaled_cache(pdlib, hkv, hd, page_len, [a + b for a, b in zip(new, prefix)], lambda s, i: octaves if i in (0, 3) else 0, rng,
                     lambda s, i: -strong * sign if i in (0, 3) else None)
    q = gen.bf16_round(sign * (1 + 0.1 * rng.standard_normal((sum(new), hq, hd))))
    got, at = prefill(pdlib, c, hq, q, new, prefix), 0
    for s, (n, pre) in enumerate(zip(new, prefix)):
        check(c, hq, q[at:at + n], pre, n, s, got[at:at + n], f"request {s}")
        at += n
    one = decode(pdlib, c, hq, q[:2], [200, 77])
    for s, k in enumerate([200, 77]):
        check(c, hq, q[s:s + 1], k, 1, s, one[s:s + 1], f"decode {s}")


@pytest.mark.parametrize("hq,hkv,hd,page_len", SHAPES)
@pytest.mark.parametrize("octaves", [10, 18, 30, 70])
def test_rows_in_front_of_a_large_page_do_not_notice_it(pdlib, hq, hkv, hd, page_len, octaves):
    """The page of the last tokens is large, in the key tile of rows in front of it or behind."""
    rng = np.random.default_rng(octaves + 1)
    for new, prefix in ((100, 0), (9, 30), (260, 1000)):
        last = (new + prefix - 1) // page_len
        c = scaled_cache(pdlib, hkv, hd, page_len, [new + prefix], lambda s, i: octaves if i == last else 0, rng)
        q = gen.normal_bf16(99, gen.S_X, (new, hq, hd), 1.0, sub=octaves)
        got = prefill(pdlib, c, hq, q, [new], [prefix])
        check(c, hq, q, prefix, new, 0, got, f"{new} rows over {prefix}")
        front = last * page_len - prefix
        if front > 0:                            # held to the pages that these rows see
            check(c, hq, q[:front], prefix, front, 0, got[:front], "rows in front")


def test_some_requests_of_many_have_such_pages(pdlib):
    """More row blocks than SMs, so that a block goes from usual requests to one with pages far apart and on."""
    hq, hkv, hd, page_len, n = 16, 8, 128, 32, 60
    rng = np.random.default_rng(9)
    new, prefix = [int(v) for v in rng.integers(20, 200, n)], [int(v) for v in rng.integers(0, 150, n)]
    far = [s % 7 == 3 for s in range(n)]
    c = scaled_cache(pdlib, hkv, hd, page_len, [a + b for a, b in zip(new, prefix)], lambda s, i: 40 if far[s] and i == 1 else 0, rng)
    q = gen.normal_bf16(101, gen.S_X, (sum(new), hq, hd), 1.0)
    got, at = prefill(pdlib, c, hq, q, new, prefix), 0
    np.testing.assert_array_equal(got, prefill(pdlib, c, hq, q, new, prefix, pad=8))
    for s, (m, pre) in enumerate(zip(new, prefix)):
        if far[s] or s % 5 == 0:
            for first, k in ((0, 1), (max(0, min(31 - pre, m - 1)), 2), (m - 1, 1)):      # the last of the first page, and behind
                k = min(k, m - first)
                check(c, hq, q[at + first:at + first + k], pre + first, k, s, got[at + first:at + first + k], f"request {s}")
        at += m


@pytest.mark.parametrize("hq,hkv,hd,page_len", SHAPES)
def test_nan_values_among_far_pages(pdlib, hq, hkv, hd, page_len):
    """NaN codes of V reach the rows that see them, of their feature, and no others; a NaN of K the rows that see its key."""
    rng = np.random.default_rng(77)
    new, prefix = [60, 5], [70, 33]
    total = [a + b for a, b in zip(new, prefix)]
    c = scaled_cache(pdlib, hkv, hd, page_len, total, lambda s, i: 50 if i == 1 else -20 if i == 3 else 0, rng)
    q = gen.normal_bf16(102, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    want = prefill(pdlib, c, hq, q, new, prefix).reshape(-1, hq, hd)
    bad, g, start = np.zeros(want.shape, bool), hq // hkv, [0, new[0]]
    for s, key, head, d in ((0, 3, 0, 5), (0, 75, hkv - 1, hd - 1), (0, 100, 0, 17), (1, 36, hkv - 1, 0)):
        c.v[c.table[s][key // page_len], head, key % page_len, d] = 0x7F
        rows = start[s] + np.arange(new[s])[prefix[s] + np.arange(new[s]) >= key]
        bad[rows, head * g:(head + 1) * g, d] = True
    c.k[c.table[0][90 // page_len], 0, 90 % page_len, 3] = 0xFF
    bad[np.arange(new[0])[prefix[0] + np.arange(new[0]) >= 90], :g] = True
    got = prefill(pdlib, c.upload(), hq, q, new, prefix).reshape(-1, hq, hd)
    np.testing.assert_array_equal(np.isnan(got), bad)
    np.testing.assert_array_equal(got[~bad], want[~bad])


def test_wait_timeout_among_far_pages(pdlib):
    """One arrival left out while the second copy of the roles is at work: the error word says so and the next call is right."""
    import torch
    hq, hkv, hd, page_len, n, pre = 32, 8, 128, 64, 128, 2000
    c = scaled_cache(pdlib, hkv, hd, page_len, [n + pre], lambda s, i: 30 if i % 9 == 0 else 0, np.random.default_rng(5))
    q = gen.normal_bf16(107, gen.S_X, (n, hq, hd), 1.0)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(cfg, 1, n + pre)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, err = empty_bf16(n, hq * hd), torch.zeros(1, dtype=torch.int32, device="cuda")
    pdlib.pd_test_inject_wait_timeout(pdlib.INJECT_ATTN_PAGED, 20_000_000)
    try:
        pdlib.pd_paged_prefill_attention(cfg, to_dev(q.reshape(n, -1)), hq * hd, out, i32_dev([0, n]), [0, n], i32_dev([pre]), [pre], c.struct,
                                         ws, need, err_word=err)
        torch.cuda.synchronize()
    finally:
        pdlib.pd_test_inject_wait_timeout(pdlib.INJECT_NONE, 0)
    if os.environ.get("PD_PAGED_PREFILL") != "0":      # (the streaming kernel waits for nothing)
        assert int(err.item()) == 1
    check(c, hq, q, pre, n, 0, prefill(pdlib, c, hq, q, [n], [pre]), "after it")


def test_far_pages_in_a_replayed_graph(pdlib):
    """Whether pages are far apart is seen on the device: a captured call follows the scales of its replay."""
    import torch
    hq, hkv, hd, page_len, n, pre = 32, 8, 128, 64, 200, 300
    c = scaled_cache(pdlib, hkv, hd, page_len, [n + pre], lambda s, i: 0, np.random.default_rng(6))
    q = gen.normal_bf16(108, gen.S_X, (n, hq, hd), 1.0)
    usual = prefill(pdlib, c, hq, q, [n], [pre])
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(cfg, 1, n + pre)
    ws, dq, out = torch.empty(need, dtype=torch.uint8, device="cuda"), to_dev(q.reshape(n, -1)), empty_bf16(n, hq * hd)
    cu, dpre, s, g = i32_dev([0, n]), i32_dev([pre]), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pdlib.pd_paged_prefill_attention(cfg, dq, hq * hd, out, cu, [0, n], dpre, [pre], c.struct, ws, need)
    for page, factor in ((2, 2.0 ** 35), (2, 2.0 ** -35), (6, 2.0 ** -50)):
        c.vs[c.table[0, page]] *= np.float32(factor)
        c.dvs.copy_(torch.from_numpy(c.vs))
        g.replay()
        torch.cuda.synchronize()
        got = from_dev(out)
        check(c, hq, q, pre, n, 0, got, f"page {page}")
        if factor == 2.0 ** -35:
            np.testing.assert_array_equal(got, usual)


@pytest.mark.parametrize("which", [0, 1])
def test_each_kernel(pdlib, which):
    """The switch is read once per process."""
    res = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_paged_spread.py", "-k", "not each_kernel", "-x", "-q", "-m", "gpu"],
                         cwd=ROOT, env={**os.environ, "PD_PAGED_PREFILL": str(which)}, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-1000:]

"""GPU: decode attention over the 4-bit paged KV cache against the float64 oracle on the same cached values.  Rows without a token
have NaN scales and unused table entries are -1: neither may reach an output."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from kv4_util import Cache4, check_attention
from oracle import paged4

pytestmark = pytest.mark.gpu


def decode(pd, c, hq, q, kv_len, n_new=1, max_kv=None, pad=0, err=None, stream=None):
    import torch
    b = len(kv_len)
    cfg = pd.LayerConfig(hq * c.hd, hq, c.hkv, c.hd, 64)
    width = hq * c.hd
    flat = np.full((b * n_new, width + pad), np.nan, np.float32)
    flat[:, :width] = q.reshape(b * n_new, width)
    max_kv = max(n_new, max_kv or max(kv_len) + n_new)
    ws_bytes = pd.pd_paged_kv4_decode_attention_workspace_bytes(cfg, b, n_new, max_kv)
    ws = torch.full((max(ws_bytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    out = empty_bf16(b * n_new + 1, width)
    pd.pd_paged_kv4_decode_attention(cfg, to_dev(flat), width + pad, out, i32_dev(kv_len), b, n_new, max_kv, c.struct, ws, ws_bytes, err_word=err)
    torch.cuda.synchronize()
    assert not out[b * n_new].any()
    return from_dev(out[:b * n_new]).reshape(b, n_new, hq, c.hd)


def check(c, hq, q, kv_len, got, n_new=1, cap=None):
    q = q.reshape(len(kv_len), n_new, hq, c.hd)
    for s, n in enumerate(kv_len):
        if n < 0:
            assert not got[s].any()
            continue
        total = min(n + n_new, cap or n + n_new)
        k, v = c.kv(s, total)
        pos = np.minimum(n + np.arange(n_new), total - 1)
        check_attention(q[s], k, v, pos, got[s], f"sequence {s} ({n} keys)")


def queries(seed, b, n_new, hq, hd, std=1.0):
    return gen.normal_bf16(seed, gen.S_X, (b, n_new, hq, hd), std, sub=hd)


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (64, 8, 128), (4, 4, 128), (16, 1, 128), (16, 1, 64), (9, 1, 64), (11, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("page_len", [16, 32, 64, 128])
def test_lengths(pdlib, hq, hkv, hd, page_len):
    """One key to several parts, every tail of a tile's halves and of the page, padding rows."""
    kv_len = [0, 1, 14, 15, 16, 31, 32, 63, 64, 65, -1, 127, 128, 300, 1111, 255]
    lens = [max(0, n + 1) for n in kv_len]
    c = Cache4(pdlib, hkv, hd, page_len, lens, seed=hq + page_len).fill(lens, np.random.default_rng(hd + page_len), 0.5).upload()
    q = queries(70, len(kv_len), 1, hq, hd)
    got = decode(pdlib, c, hq, q, kv_len, pad=8)
    check(c, hq, q, kv_len, got)
    np.testing.assert_array_equal(got, decode(pdlib, c, hq, q, kv_len))               # deterministic, whatever the pitch
    check(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len, max_kv=1))                # no split: a bound that is too small


@pytest.mark.parametrize("hq,hkv,hd,n_new", [(8, 2, 64, 2), (32, 8, 128, 3), (32, 8, 128, 4), (64, 8, 128, 2), (16, 1, 64, 3), (4, 4, 128, 8), (4, 4, 64, 17), (32, 8, 128, 9), (9, 1, 64, 2)])
@pytest.mark.parametrize("page_len", [16, 64])
def test_several_tokens(pdlib, hq, hkv, hd, n_new, page_len):
    """Each token sees the keys up to its own; blocks of all tokens, of some, of one."""
    kv_len = [0, 1, 13, 30, 31, -1, 63, 300, 1100]
    lens = [n + n_new if n >= 0 else 0 for n in kv_len]
    c = Cache4(pdlib, hkv, hd, page_len, lens, seed=n_new).fill(lens, np.random.default_rng(n_new), 0.5).upload()
    q = queries(71, len(kv_len), n_new, hq, hd)
    got = decode(pdlib, c, hq, q, kv_len, n_new)
    check(c, hq, q, kv_len, got, n_new)
    np.testing.assert_array_equal(got, decode(pdlib, c, hq, q, kv_len, n_new, pad=16))


@pytest.mark.parametrize("hq,hkv,hd,page_len,n,n_new", [(32, 8, 128, 64, 20011, 1), (8, 2, 64, 16, 9000, 1), (16, 1, 128, 32, 5000, 2), (8, 1, 64, 128, 30001, 4)])
def test_long_sequence(pdlib, hq, hkv, hd, page_len, n, n_new):
    """Page numbers in more than one batch, many parts, a short sequence beside."""
    lens = [n, 40]
    c = Cache4(pdlib, hkv, hd, page_len, lens, seed=n).fill(lens, np.random.default_rng(n), 0.5).upload()
    q = queries(72, 2, n_new, hq, hd, 1.5)
    kv_len = [n - n_new, 40 - n_new]
    check(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len, n_new), n_new)
    alone = decode(pdlib, c, hq, q, kv_len, n_new, max_kv=n_new)                      # one block for all keys
    check(c, hq, q, kv_len, alone, n_new)


@pytest.mark.parametrize("n_new", [1, 3])
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 128), (32, 8, 64)])
def test_parts_that_join_in_either_way(pdlib, n_new, hq, hkv, hd):
    """The same rows with keys cut into one part to more than ten (a bound of 256 keys each), few sequences and among many that pad:
    parts without keys, with a NaN that the last token alone sees, and a sequence that reaches past the bound."""
    lens = [2000, 60, 700, 257]
    c = Cache4(pdlib, hkv, hd, 64, lens, seed=16).fill(lens, np.random.default_rng(16), 0.5)
    c.table = np.pad(c.table, ((0, 60), (0, 64 - c.width)), constant_values=-1)
    c.width = 64
    k_nan, v_nan = (c.table[0, 1999 // 64], 0, 1999 % 64, 1), (c.table[2, 699 // 64], 1, 699 % 64, 2)
    kv_len = [n - n_new for n in lens]
    q = queries(76, 64, n_new, hq, hd)
    for broken in (False, True):
        if broken:
            c.ks[k_nan] = c.vs[v_nan] = 0x7F
        c.upload()
        bad = np.zeros((4, n_new, hq, hd), bool)
        group = hq // hkv
        if broken:
            bad[0, -1, :group] = True
            bad[2, -1, group:2 * group, 32:48] = True
        for pads in (0, 60):
            for most in (256, 512, 1100, 2000, 2048, 2300, 2560, 2817, 4096):
                got = decode(pdlib, c, hq, q[:4 + pads], kv_len + [-1] * pads, n_new, max_kv=most)
                assert not got[4:].any()
                np.testing.assert_array_equal(np.isnan(got[:4]), bad, err_msg=f"{pads} {most}")
                if not broken:
                    check(c, hq, q[:4], kv_len, got[:4], n_new)


def test_sizes_far_apart_and_large_queries(pdlib):
    """Values of V over many octaves, queries from 1e-20 to 1e20 (the softmax is then one-hot or flat), zeros."""
    hq, hkv, hd = 8, 2, 64
    kv_len = [200, 333, 90, 17, 60]
    lens = [n + 1 for n in kv_len]
    c = Cache4(pdlib, hkv, hd, 16, lens, seed=12).fill(lens, np.random.default_rng(12), 2.5)
    rng = np.random.default_rng(13)
    for s, n in enumerate(kv_len):  # K of ordinary size again (scores stay comparable), V as it is
        paged4.append(c.k, c.ks, c.table[s], 0, gen.bf16_round(rng.standard_normal((n + 1, hkv, hd))), c.ke)
    c.upload()
    q = queries(73, 5, 1, hq, hd)
    q[1] = gen.bf16_round(q[1] * np.float32(1e-20))
    q[2] = gen.bf16_round(q[2] * np.float32(100.0))
    q[3] = 0.0
    check(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len))
    # one-hot: the largest score takes all
    q[4] = gen.bf16_round(q[4] * np.float32(1e20))
    got = decode(pdlib, c, hq, q, kv_len)[4, 0]
    k, v = c.kv(4, 61)
    for h in range(hq):
        best = int((k[:, h // 4] @ q[4, 0, h].astype(np.float64)).argmax())
        np.testing.assert_array_equal(got[h], gen.bf16_round(v[best, h // 4].astype(np.float32)))


@pytest.mark.parametrize("n_new", [1, 3])
def test_non_finite_values_stay_with_the_rows_that_see_them(pdlib, n_new):
    """A stored NaN of V reaches its 16 features, one of K the whole head, of the rows at or behind it and of no other."""
    hq, hkv, hd, p = 8, 2, 64, 16
    lens = [50] * 4
    kv_len = [50 - n_new] * 4
    c = Cache4(pdlib, hkv, hd, p, lens, seed=14).fill(lens, np.random.default_rng(14)).upload()
    q = queries(74, 4, n_new, hq, hd)
    clean = decode(pdlib, c, hq, q, kv_len, n_new)
    c.vs[c.table[0, 2], 1, 3, 2] = 0x7F                    # key 35: every row sees it
    c.vs[c.table[1, 3], 0, 1, 1] = 0xFF                    # key 49: the last row alone
    c.ks[c.table[2, 3], 1, 1, 0] = 0x7F                    # key 49, K
    c.upload()
    q[3, 0, 3, 5] = np.nan
    got = decode(pdlib, c, hq, q, kv_len, n_new)
    bad = np.zeros((4, n_new, hq, hd), bool)
    bad[0, :, 4:, 32:48] = True
    bad[1, n_new - 1, :4, 16:32] = True
    bad[2, n_new - 1, 4:] = True
    bad[3, 0, 3] = True
    np.testing.assert_array_equal(np.isnan(got), bad)
    np.testing.assert_array_equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("n_new", [1, 4])
def test_bad_pages_and_lengths_are_reported(pdlib, n_new):
    import torch
    hq, hkv, hd, p = 8, 2, 64, 16
    kv_len = [80 - n_new, 60, 200, -3]
    c = Cache4(pdlib, hkv, hd, p, [80] * 4, seed=15, extra_cols=0).fill([80] * 4, np.random.default_rng(15))
    q = queries(75, 4, n_new, hq, hd)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.upload()
    got = decode(pdlib, c, hq, q, kv_len, n_new, max_kv=80, err=err)
    assert int(err.item()) == 2                            # a sequence that reaches past the table: what is there counts
    check(c, hq, q, kv_len, got, n_new, cap=80)
    err.zero_()
    kv_len[2] = 70
    check(c, hq, q, kv_len, decode(pdlib, c, hq, q, kv_len, n_new, max_kv=80, err=err), n_new)
    assert int(err.item()) == 0
    table = c.table.copy()
    c.table[1, 1] = 99                                     # keys 16 .. 31 of the second sequence are left out
    c.upload()
    got = decode(pdlib, c, hq, q, kv_len, n_new, max_kv=80, err=err)
    assert int(err.item()) == 2
    c.table = table
    for s in (0, 2):
        check(c, hq, q, [kv_len[s] if i == s else -1 for i in range(4)], np.where(np.arange(4)[:, None, None, None] == s, got, 0), n_new)
    k, v = c.kv(1, 60 + n_new)
    keep = np.r_[0:16, 32:60 + n_new]
    check_attention(q[1], k[keep], v[keep], 60 - 16 + np.arange(n_new), got[1])


def test_heads_without_exponents(pdlib):
    hq, hkv, hd = 8, 2, 128
    c = Cache4(pdlib, hkv, hd, 32, [77, 20], seed=16, exps=False).fill([77, 20], np.random.default_rng(16)).upload()
    q = queries(76, 2, 1, hq, hd)
    check(c, hq, q, [76, 19], decode(pdlib, c, hq, q, [76, 19]))
    c.k_exp, c.v_exp = np.array([100, -100], np.int32), np.array([-100, 100], np.int32)   # held to -30 .. 30
    c.ke, c.ve = np.array([30, -30]), np.array([-30, 30])
    c.upload()
    q[:, :, :4] = gen.bf16_round(q[:, :, :4] * np.float32(2.0 ** -30))
    q[:, :, 4:] = gen.bf16_round(q[:, :, 4:] * np.float32(2.0 ** 30))
    check(c, hq, q, [76, 19], decode(pdlib, c, hq, q, [76, 19]))


def test_results_at_any_alignment(pdlib):
    """out starts on any bf16, in the joined form as well."""
    import torch
    hq, hkv, hd, n = 8, 2, 64, 3000
    c = Cache4(pdlib, hkv, hd, 64, [n], seed=17).fill([n], np.random.default_rng(17)).upload()
    q = queries(77, 1, 1, hq, hd)
    want = decode(pdlib, c, hq, q, [n - 1])
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    ws_bytes = pdlib.pd_paged_kv4_decode_attention_workspace_bytes(cfg, 1, 1, n)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    out = empty_bf16(hq * hd + 8)
    pdlib.pd_paged_kv4_decode_attention(cfg, to_dev(q.reshape(1, -1)), hq * hd, out.data_ptr() + 6, i32_dev([n - 1]), 1, 1, n, c.struct, ws, ws_bytes)
    got = from_dev(out)
    np.testing.assert_array_equal(got[3:3 + hq * hd].reshape(hq, hd), want[0, 0])
    assert not got[:3].any() and not got[3 + hq * hd:].any()

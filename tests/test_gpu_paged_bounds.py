"""GPU: the 8-bit serving operators held to no more than their stated roundings: codes of the norm to half a step of the format,
prefill attention to weights in f16, and every prefill kernel on the edge cases whatever the lengths would choose."""
import os
import subprocess
import sys

import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import i32_dev
from oracle import fp8, paged
from paged_util import F16, Cache, assert_within, attention_bound
from test_gpu_norm_fp8 import REL, run
from test_gpu_paged_attention import decode, prefill

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def half_step(a):
    """Half the distance of the E4M3 numbers around magnitude a: 2^-4 of the binade's lower end, 2^-10 below 2^-6."""
    e = np.clip(np.floor(np.log2(np.maximum(a, 2.0 ** -20))), -6, 8)
    return 2.0 ** (e - 4)


@pytest.mark.parametrize("rows,d,group", [(64, 4096, 128), (33, 8192, 0), (1, 128, 128), (7, 1040, 0), (300, 512, 128)])
def test_norm_codes_are_the_nearest(pdlib, rows, d, group):
    """Against n / s with the scale that the call wrote: half a step, and what the fp32 arithmetic of n (REL), the product with the
    approximate reciprocal (2^-22 in all) move a value across the middle of two codes."""
    x, r = gen.normal_bf16(66, 1, (rows, d), 1.0, sub=d), gen.normal_bf16(66, 2, (rows, d), 2.0, sub=d)
    g = gen.normal_bf16(66, 3, (d,), 0.3, 1.0)
    _, _, codes, scales = run(pdlib, x, r, g, group)
    _, n, so = paged.add_rmsnorm(x, r, g, 1e-6, group)
    s = scales.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(s - so.reshape(s.shape)) <= REL * s)
    want = n / np.repeat(s, d // s.shape[1], axis=1)
    slack = (REL + 2.0 ** -22) * np.abs(want)
    off = np.abs(fp8.e4m3_decode(codes.cpu().numpy()) - np.clip(want, -448.0, 448.0))
    assert np.all(off <= half_step(np.abs(want) + slack) + slack), (off / half_step(np.abs(want) + slack)).max()


def f16_bound(q, keys, vals, pos, o, spread, score):
    """attention_bound with weights in f16, and what the tensor-memory kernel leaves of q: it is the sum of two E4M3 numbers,
    exact but for entries below 2^-9 of the row's largest (their last bits lie below 2^-9 where the largest is 2^7 to 2^8), which
    are off by up to 2^-17 of it.  An error of a score acts on a weight twice, as in attention_bound."""
    n, hq, hd = q.shape
    g = hq // keys.shape[1]
    a = np.abs(q.astype(np.float64))
    top = a.max(axis=-1, keepdims=True)
    small = (a < top * 2.0 ** -9) & (a > 0)
    dq = np.zeros((n, hq))
    for h in range(hq):
        dq[:, h] = (small[:, h] * (2.0 ** -17 * top[:, h])) @ np.abs(keys[:, h // g]).max(axis=0) / np.sqrt(hd)
    # weights are at most 2^-32 of the row's largest off as well (the smallest f16 numbers)
    low = 2.0 ** -32 * np.repeat(np.abs(vals).sum(axis=0)[None], n, axis=0)
    return attention_bound(o, spread, score, F16) + 2.0 * dq[..., None] * spread + np.repeat(low, g, axis=1)


def check(c, hq, q, new, prefix, got, rows):
    at = 0
    for s, (n, pre) in enumerate(zip(new, prefix)):
        if n:
            k, v = c.kv(s, pre + n)
            sel = np.arange(n) if n <= rows else np.unique(np.r_[0, n - 1, np.random.default_rng(s).integers(0, n, rows)])
            o, spread, score = paged.attend(q[at + sel], k, v, pre + sel)
            assert_within(got[at + sel].reshape(o.shape), o, f16_bound(q[at + sel], k, v, pre + sel, o, spread, score), f"request {s}")
        at += n


@pytest.mark.parametrize("hq,hkv,hd,page_len", [(8, 2, 64, 16), (32, 8, 128, 64), (16, 1, 128, 32), (3, 3, 64, 128), (9, 1, 64, 16), (64, 8, 128, 16)])
@pytest.mark.parametrize("size", [1.0, 3.0])
def test_prefill_weights_are_f16(pdlib, hq, hkv, hd, page_len, size):
    new, prefix = [1, 5, 0, 130, 1, 260], [0, 127, 30, 70, 400, 300]
    total = [a + b for a, b in zip(new, prefix)]
    c = Cache(pdlib, hkv, hd, page_len, total, seed=hq + page_len)
    c.fill(total, np.random.default_rng(hd + hq), 0.5)
    c.upload()
    q = gen.normal_bf16(105, gen.S_X, (sum(new), hq, hd), size, sub=hd)
    got = prefill(pdlib, c, hq, q, new, prefix)
    check(c, hq, q, new, prefix, got, rows=12)
    # a row for itself by the decode call: both within the bound of the same exact row
    rows, kv = [0, 1, 6, 136], [0, 127, 70, 400]
    one = decode(pdlib, c_rows(c, [0, 1, 3, 4]), hq, q[rows], kv)
    for i, (row, n) in enumerate(zip(rows, kv)):
        k, v = c.kv([0, 1, 3, 4][i], n + 1)
        o, spread, score = paged.attend(q[row:row + 1], k, v, [n])
        bound = f16_bound(q[row:row + 1], k, v, [n], o, spread, score)
        assert_within(one[i].reshape(o.shape), o, bound, f"decode {i}")
        assert_within(one[i].reshape(o.shape), got[row].reshape(o.shape).astype(np.float64), 2 * bound, f"decode and prefill {i}")


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("factor", [30.0, 1000.0, 30000.0])
def test_prefill_weights_with_an_outlier_in_q(pdlib, hq, hkv, hd, factor):
    """One channel of q is far larger than the others and meets keys that are 0 there, so that all of a score comes from the
    small entries."""
    new, prefix, page_len = [40, 200], [90, 10], 32
    total = [a + b for a, b in zip(new, prefix)]
    c, rng = Cache(pdlib, hkv, hd, page_len, total, seed=hd), np.random.default_rng(hd)
    for s, n in enumerate(total):
        k = rng.standard_normal((n, hkv, hd))
        k[..., 5] = 0.0
        paged.append(c.k, c.ks, c.table[s], 0, gen.bf16_round(k))
        paged.append(c.v, c.vs, c.table[s], 0, gen.bf16_round(rng.standard_normal((n, hkv, hd))))
    c.upload()
    q = gen.normal_bf16(106, gen.S_X, (sum(new), hq, hd), 1.0, sub=hd)
    q[..., 5] = gen.bf16_round(q[..., 5] * np.float32(factor))
    check(c, hq, q, new, prefix, prefill(pdlib, c, hq, q, new, prefix), rows=12)


def c_rows(c, rows):
    """The same pool with a page table of the given sequences."""
    import copy
    d = copy.copy(c)
    d.table = c.table[rows]
    d.dt = i32_dev(d.table)
    d.struct = c.pd.paged_kv_cache_struct(c.dk, c.dv, c.dks, c.dvs, d.dt, c.n_pages, c.page_len, len(rows), c.width)
    return d


@pytest.mark.parametrize("which", [0, 1])
def test_each_kernel_on_the_edge_cases(pdlib, which):
    """The switch is read once per process."""
    env = {**os.environ, "PD_PAGED_PREFILL": str(which)}
    for args in (["tests/test_gpu_paged_edges.py", "-k", "attention_of_very_many or wide_groups or cut_behind"],
                 ["tests/test_gpu_paged_paths.py", "-k", "odd_groups"], ["tests/test_gpu_paged_contract.py", "-k", "prefill"],
                 ["tests/test_gpu_paged_bounds.py", "-k", "weights"]):
        res = subprocess.run([sys.executable, "-m", "pytest", *args, "-x", "-q", "-m", "gpu"], cwd=ROOT, env=env, capture_output=True, text=True,
                             timeout=600)
        assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-1000:]


CUT = """
import sys; sys.path[:0] = ["tests", "."]
import numpy as np, torch
import paper_2603_04716_b200 as pd
from gpu_util import empty_bf16, i32_dev
from paged_util import Cache
hq, hkv, hd, new, prefix, want = eval(sys.argv[1])
c = Cache(pd, hkv, hd, 128, [new + prefix], seed=1)
c.fill([new + prefix], np.random.default_rng(1))
c.upload()
cfg = pd.LayerConfig(hq * hd, hq, hkv, hd, 64)
need = pd.pd_paged_prefill_attention_workspace_bytes(cfg, 1, new + prefix)
ws, q = torch.empty(need, dtype=torch.uint8, device="cuda"), empty_bf16(new, hq * hd)
before = pd.pd_launch_count()
pd.pd_paged_prefill_attention(cfg, q, hq * hd, torch.empty_like(q), i32_dev([0, new]), [0, new], i32_dev([prefix]), [prefix], c.struct, ws, need)
torch.cuda.synchronize()
assert pd.pd_launch_count() - before == want, pd.pd_launch_count() - before
"""


@pytest.mark.parametrize("case", [(16, 8, 128, 1400, 3500, 2),     # 88 items for 148 SMs
                                  (16, 8, 64, 2600, 1900, 2),      # 168: those behind the first full turn
                                  (16, 2, 128, 60, 3000, 2),       # a few
                                  (16, 8, 128, 2300, 100, 1),      # 144: fewer than SMs, more than half of them, of too few keys
                                  (16, 8, 128, 100, 20, 1)])       # one key tile: nothing to cut
def test_key_ranges_are_cut(pdlib, case):
    """On the tensor-memory kernel: a second launch joins the parts where key ranges are cut."""
    res = subprocess.run([sys.executable, "-c", CUT, repr(case)], cwd=ROOT, env={**os.environ, "PD_PAGED_PREFILL": "1"}, capture_output=True,
                         text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-1000:] + res.stderr[-2000:]

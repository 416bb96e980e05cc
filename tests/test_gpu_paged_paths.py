"""GPU: every kernel behind pd_paged_prefill_attention on every test case, whatever the lengths would choose (the switch is read
once per process), and the bounded waits of the tensor-memory kernel."""
import os
import subprocess
import sys

import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from paged_util import Cache
from test_gpu_paged_attention import check_prefill, prefill

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("which", [0, 1])
def test_each_kernel_on_all_cases(pdlib, which):
    res = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_paged_attention.py", "-k", "prefill", "-x", "-q", "-m", "gpu"],
                         cwd=ROOT, env={**os.environ, "PD_PAGED_PREFILL": str(which)}, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-1000:]


def test_many_requests_and_odd_groups(pdlib):
    """More requests than a warp has lanes, runs without rows, groups that do not divide a row tile, items taken over."""
    rng = np.random.default_rng(31)
    for hq, hkv, hd, hi in [(6, 2, 64, 40), (5, 1, 128, 90), (33, 3, 64, 25), (32, 8, 128, 300)]:
        n = 45
        new = [int(v) for v in rng.integers(0, hi, n)]
        new[3] = new[40] = 0
        prefix = [int(v) for v in rng.integers(0, 400, n)]
        c = Cache(pdlib, hkv, hd, 32, [a + b for a, b in zip(new, prefix)], seed=hq)
        c.fill([a + b for a, b in zip(new, prefix)], rng, 0.5)
        c.upload()
        q = gen.normal_bf16(90, gen.S_X, (sum(new), hq, hd), 1.0, sub=hq)
        check_prefill(c, hq, q, new, prefix, prefill(pdlib, c, hq, q, new, prefix, pad=16), rows=2)


def test_wait_timeout_is_reported_and_leaves_the_gpu_usable(pdlib):
    """One arrival left out: the waits of the blocks run into their bound, the error word says so, the next call is right."""
    import torch
    hq, hkv, hd, new, prefix = 32, 8, 128, [128], [2000]
    c = Cache(pdlib, hkv, hd, 64, [2128], seed=32)
    c.fill([2128], np.random.default_rng(32), 0.5)
    c.upload()
    q = gen.normal_bf16(91, gen.S_X, (128, hq, hd), 1.0)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(cfg, 1, 2128)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, err = empty_bf16(128, hq * hd), torch.zeros(1, dtype=torch.int32, device="cuda")
    pdlib.pd_test_inject_wait_timeout(pdlib.INJECT_ATTN_PAGED, 20_000_000)
    try:
        pdlib.pd_paged_prefill_attention(cfg, to_dev(q.reshape(128, -1)), hq * hd, out, i32_dev([0, 128]), [0, 128], i32_dev(prefix), prefix,
                                         c.struct, ws, need, err_word=err)
        torch.cuda.synchronize()
    finally:
        pdlib.pd_test_inject_wait_timeout(pdlib.INJECT_NONE, 0)
    assert int(err.item()) == 1
    check_prefill(c, hq, q, new, prefix, prefill(pdlib, c, hq, q, new, prefix), rows=8)

"""GPU: a traced serving step over the 4-bit cache accounts for every one of its kernels."""
import numpy as np
import pytest

from gpu_util import empty_bf16, i32_dev, to_dev
from kv4_util import Cache4, Transform
from test_gpu_kv4_append import rows_of

pytestmark = pytest.mark.gpu


def test_every_call_of_a_step_is_traced(pdlib):
    import torch
    hq, hkv, hd, n = 8, 2, 128, 50
    c = Cache4(pdlib, hkv, hd, 32, [n], seed=1).fill([n], np.random.default_rng(1)).upload()
    t = Transform(pdlib, hd, 64, 64)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    x, width = to_dev(rows_of(2, n, hq, hkv, hd).reshape(n, -1)), (hq + 2 * hkv) * hd
    q, k, flat = empty_bf16(n, hq * hd), empty_bf16(n, hkv * hd), empty_bf16(2, 1, hkv, n, hd)
    back, zero, end = pdlib.kv_cache_struct(flat[0], flat[1], 1, n), i32_dev([0]), i32_dev([n])
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    calls = [
        ("rmsnorm", lambda: pdlib.pd_qk_norm_rope(cfg, t.struct, x, width, q, hq * hd, k, hkv * hd, i32_dev(list(range(n))), n)),
        ("kv_append", lambda: pdlib.pd_paged_kv4_append(cfg, t.struct, x, width, q, c.struct, zero, 1, i32_dev([0, n]), [0, n])),
        ("kv_append", lambda: pdlib.pd_paged_kv4_read(cfg, c.struct, None, end, 1, n, back)),
        ("kv_append", lambda: pdlib.pd_paged_kv4_write(cfg, c.struct, None, end, 1, n, back)),
        ("attn_decode", lambda: pdlib.pd_paged_kv4_decode_attention(cfg, q, hq * hd, k.new_zeros(1, hq * hd), i32_dev([n - 1]), 1, 1, n, c.struct, ws, 0)),
    ]
    for name, call in calls:
        call()
        pdlib.pd_trace_begin()
        call()
        rep = pdlib.pd_trace_end()
        assert rep[name][1] == 1 and 0 < rep[name][0] < 0.1, (name, rep)
        assert sum(v[1] for v in rep.values()) == 1, rep

"""Argument checks of the calls around the 4-bit paged KV cache: every refusal precedes any device call, so no GPU is needed.  The
pointers are never read; they only have to be non-zero and aligned."""
import ctypes

import numpy as np
import pytest
import torch

PTR = 1 << 20


def cache(pd, **kw):
    a = dict(k_codes=PTR, v_codes=PTR, k_scales=PTR, v_scales=PTR, page_table=PTR, n_pages=8, page_len=64, n_seqs=4, table_ld=4,
             k_exp=PTR, v_exp=PTR)
    a.update(kw)
    return pd.paged_kv4_cache_struct(**a)


def cfg(pd, hq=8, hkv=2, hd=64):
    return pd.LayerConfig(hq * hd, hq, hkv, hd, 64)


def turn(pd, **kw):
    a = dict(table=PTR, n_pos=256, rot_dim=64, layout=0, q_gain=PTR, k_gain=PTR, eps=1e-6)
    a.update(kw)
    return pd.qk_transform_struct(**a)


def flat(pd, **kw):
    a = dict(k=PTR, v=PTR, batch_cap=4, len_cap=256)
    a.update(kw)
    return pd.kv_cache_struct(**a)


def refused(pd, status, f, **kw):
    with pytest.raises(pd.PdError) as e:
        f(**kw)
    assert e.value.status == status, kw


def test_struct_layouts(pdlib):
    assert ctypes.sizeof(pdlib.pd_paged_kv4_cache) == 8 + 7 * 8 + 4 * 4
    assert ctypes.sizeof(pdlib.pd_qk_transform) == 16 + 3 * 8 + 8
    assert ctypes.sizeof(pdlib.pd_rope_cfg) == 16 + 5 * 8


BAD_CACHES = [dict(k_codes=None), dict(v_codes=None), dict(k_scales=None), dict(v_scales=None), dict(page_table=None), dict(n_pages=0),
              dict(n_seqs=0), dict(table_ld=0), dict(n_pages=-1), dict(k_codes=PTR + 8), dict(v_scales=PTR + 8), dict(k_exp=PTR + 2),
              dict(v_exp=PTR + 1), dict(page_table=PTR + 2)]
BAD_PAGES = [dict(n_pages=1 << 26), dict(page_len=0), dict(page_len=24), dict(page_len=256), dict(page_len=8), dict(table_ld=1 << 25)]
BAD_TURNS = [dict(layout=2), dict(layout=-1), dict(rot_dim=0), dict(rot_dim=80), dict(n_pos=0), dict(n_pos=-4), dict(eps=-1.0),
             dict(eps=float("nan")), dict(eps=float("inf")), dict(table=PTR + 8), dict(q_gain=PTR + 2), dict(k_gain=PTR + 8)]


def calls(pd):
    """The calls as functions of (cfg, cache, transform) with otherwise valid arguments."""
    n = lambda c: (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim  # noqa: E731
    return {
        "append": lambda c, k, t, **kw: pd.pd_paged_kv4_append(**{**dict(cfg=c, transform=t, qkv=PTR, ldqkv=n(c), q_out=PTR, cache=k, kv_len_dev=PTR, n_req=2, stream=0), **kw}),
        "write": lambda c, k, t, **kw: pd.pd_paged_kv4_write(**{**dict(cfg=c, cache=k, begin_dev=PTR, end_dev=PTR, n_seqs=2, max_len=9, kv_in=flat(pd), stream=0), **kw}),
        "read": lambda c, k, t, **kw: pd.pd_paged_kv4_read(**{**dict(cfg=c, cache=k, begin_dev=PTR, end_dev=PTR, n_seqs=2, max_len=9, kv_out=flat(pd), stream=0), **kw}),
        "decode": lambda c, k, t, **kw: pd.pd_paged_kv4_decode_attention(**{**dict(cfg=c, q=PTR, ldq=c.n_q_heads * c.head_dim, out=PTR, kv_len_dev=PTR, batch=2, n_new=1, max_kv_len=100, cache=k, workspace=PTR, workspace_bytes=1 << 30, stream=0), **kw}),
        "norm": lambda c, k, t, **kw: pd.pd_qk_norm_rope(**{**dict(cfg=c, transform=t, qkv=PTR, ldqkv=n(c), q_out=PTR, ldq_out=c.n_q_heads * c.head_dim, k_out=PTR, ldk_out=c.n_kv_heads * c.head_dim, positions_dev=PTR, rows=3, stream=0), **kw}),
    }


@pytest.mark.parametrize("which", ["append", "write", "read", "decode"])
def test_cache_description(pdlib, which):
    f = calls(pdlib)[which]
    for bad in BAD_CACHES:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, c=cfg(pdlib), k=cache(pdlib, **bad), t=turn(pdlib))
    for bad in BAD_PAGES:
        refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, f, c=cfg(pdlib), k=cache(pdlib, **bad), t=turn(pdlib))
    k = cache(pdlib)
    k.struct_size = 8
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, c=cfg(pdlib), k=k, t=turn(pdlib))


@pytest.mark.parametrize("which", ["append", "write", "read", "decode", "norm"])
def test_head_shapes(pdlib, which):
    f = calls(pdlib)[which]
    for hq, hkv, hd, st in [(8, 2, 96, "UNSUPPORTED_SHAPE"), (8, 3, 64, "UNSUPPORTED_SHAPE"), (34, 2, 64, "UNSUPPORTED_SHAPE"),
                            (8, 2, 256, "UNSUPPORTED_SHAPE"), (0, 2, 64, "INVALID_ARG"), (8, 0, 64, "INVALID_ARG"), (8, -2, 64, "INVALID_ARG")]:
        refused(pdlib, getattr(pdlib, "PD_ERR_" + st), f, c=cfg(pdlib, hq, hkv, hd), k=cache(pdlib), t=turn(pdlib))


@pytest.mark.parametrize("which", ["append", "norm"])
def test_transform_description(pdlib, which):
    f = calls(pdlib)[which]
    for bad in BAD_TURNS:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, c=cfg(pdlib), k=cache(pdlib), t=turn(pdlib, **bad))
    for rot in (8, 24, 63):
        refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, f, c=cfg(pdlib), k=cache(pdlib), t=turn(pdlib, rot_dim=rot))
    t = turn(pdlib)
    t.struct_size = 4
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, c=cfg(pdlib), k=cache(pdlib), t=t)


@pytest.mark.parametrize("which,bads", [
    ("append", [dict(qkv=None), dict(kv_len_dev=None), dict(ldqkv=760), dict(ldqkv=772), dict(qkv=PTR + 2), dict(q_out=PTR + 8),
                dict(n_req=-1), dict(n_req=5), dict(n_req=2, cu_seqlens_host=[0, 1, 2]), dict(n_req=2, cu_seqlens_dev=PTR),
                dict(cu_seqlens_dev=PTR, cu_seqlens_host=[1, 1, 2]), dict(cu_seqlens_dev=PTR, cu_seqlens_host=[0, 3, 2])]),
    ("norm", [dict(qkv=None), dict(positions_dev=None), dict(ldqkv=632), dict(ldqkv=772), dict(qkv=PTR + 8), dict(q_out=PTR + 8),
              dict(k_out=PTR + 2), dict(ldq_out=504), dict(ldk_out=120), dict(ldq_out=516), dict(ldk_out=132), dict(rows=-1),
              dict(positions_dev=PTR + 2)]),
    ("decode", [dict(q=None), dict(out=None), dict(kv_len_dev=None), dict(ldq=504), dict(ldq=514), dict(q=PTR + 4), dict(out=PTR + 1),
                dict(batch=-1), dict(batch=5), dict(max_kv_len=0), dict(max_kv_len=257), dict(n_new=0), dict(n_new=-1),
                dict(n_new=3, max_kv_len=2)])])
def test_arguments(pdlib, which, bads):
    for bad in bads:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, calls(pdlib)[which], c=cfg(pdlib), k=cache(pdlib), t=turn(pdlib), **bad)


@pytest.mark.parametrize("which,name", [("write", "kv_in"), ("read", "kv_out")])
def test_copy_arguments(pdlib, which, name):
    f, base = calls(pdlib)[which], dict(c=cfg(pdlib), k=cache(pdlib), t=None)
    short = flat(pdlib)
    short.struct_size = 3
    bads = [dict(end_dev=None), dict(n_seqs=-1), dict(n_seqs=5), dict(max_len=-1), {name: short}]
    bads += [{name: flat(pdlib, **b)} for b in (dict(k=None), dict(v=None), dict(k=PTR + 8), dict(v=PTR + 2), dict(batch_cap=0), dict(len_cap=0))]
    for bad in bads:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, **base, **bad)
    refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, f, **{**base, "k": cache(pdlib, n_seqs=70000)}, n_seqs=65536)


def test_nothing_to_do_is_no_error(pdlib):
    f, base = calls(pdlib), dict(c=cfg(pdlib), k=cache(pdlib), t=turn(pdlib))
    f["append"](**base, n_req=0)
    f["append"](**base, cu_seqlens_dev=PTR, cu_seqlens_host=[0, 0, 0])
    f["write"](**base, n_seqs=0)
    f["read"](**base, max_len=0)
    f["decode"](**base, batch=0)
    f["norm"](**base, rows=0)
    f["norm"](**base, q_out=None, k_out=None)
    pdlib.pd_rope_table_scaled(pdlib.RopeConfig(64), 5, 0, None, stream=0)
    with pytest.raises(ValueError):
        f["append"](**base, cu_seqlens_dev=PTR, cu_seqlens_host=[0, 1])


def test_rope_table_arguments(pdlib):
    ok = dict(rot_dim=64, theta=1e4, scaling=pdlib.ROPE_SCALE_TURNS, factor=4.0, trained_len=4096, low=1.0, high=4.0, magnitude=1.0)
    call = lambda first=0, n=5, table=PTR, **kw: pdlib.pd_rope_table_scaled(pdlib.RopeConfig(**{**ok, **kw}), first, n, table, stream=0)  # noqa: E731
    nan, inf = float("nan"), float("inf")
    for bad in [dict(rot_dim=0), dict(rot_dim=-16), dict(scaling=-1), dict(scaling=5), dict(theta=1.0), dict(theta=nan), dict(theta=inf),
                dict(factor=0.5), dict(factor=nan), dict(factor=inf), dict(trained_len=0), dict(low=0.0), dict(low=4.0), dict(high=nan), dict(high=inf),
                dict(magnitude=0.0), dict(magnitude=nan), dict(magnitude=inf), dict(first=-1), dict(n=-1), dict(first=2 ** 31 - 3, n=5), dict(table=None),
                dict(table=PTR + 4)]:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, **bad)
    for rot in (8, 24, 144):
        refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, call, rot_dim=rot)


def test_decode_workspace_refusals(pdlib):
    c, big = cfg(pdlib), cache(pdlib, table_ld=1 << 12)
    need = pdlib.pd_paged_kv4_decode_attention_workspace_bytes(c, 1, 1, 1 << 15)
    assert need > 0 and pdlib.pd_paged_kv4_decode_attention_workspace_bytes(c, 4, 3, 256) == 0
    f = lambda **kw: calls(pdlib)["decode"](c, big, None, **{**dict(batch=1, max_kv_len=1 << 15, workspace_bytes=need), **kw})  # noqa: E731
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, workspace=None)
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, workspace=PTR + 128)
    refused(pdlib, pdlib.PD_ERR_WORKSPACE_TOO_SMALL, f, workspace_bytes=need // 2)
    wide = cache(pdlib, n_seqs=70000)
    refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, calls(pdlib)["decode"], c=c, k=wide, t=None, batch=65536)
    refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, calls(pdlib)["decode"], c=c, k=cache(pdlib, table_ld=1 << 12), t=None, batch=1, n_new=65536, max_kv_len=65536)
    refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, calls(pdlib)["decode"], c=c, k=cache(pdlib, n_seqs=70000, table_ld=1 << 12), t=None, batch=60000, n_new=10000, max_kv_len=65536)
    for bad in [(c, -1, 1, 5), (c, 1, 0, 5), (c, 1, 1, -5)]:
        with pytest.raises(pdlib.PdError):
            pdlib.pd_paged_kv4_decode_attention_workspace_bytes(*bad)


@pytest.mark.parametrize("hq,hkv,hd,most,n_new,longest", [(32, 8, 128, 256, 1, 2304), (64, 8, 128, 40, 5, 9473), (16, 1, 64, 200, 3, 70000), (64, 64, 128, 40, 16, 200000),
                                                          (9, 1, 64, 7, 2, (1 << 27) - 64)])
def test_decode_call_takes_the_workspace_of_a_larger_call(pdlib, hq, hkv, hd, most, n_new, longest):
    """One buffer sized for the largest batch, tokens and length: no smaller call refuses it, and the size does not fall as any
    of them grows.  (A call that gets past its checks here fails for want of a GPU, with another status.)"""
    if torch.cuda.is_available():
        pytest.skip("the pointers of this test are not to reach a GPU")
    rng = np.random.default_rng(most)
    c = cfg(pdlib, hq, hkv, hd)
    k = cache(pdlib, n_seqs=most, table_ld=1 << 21)
    need = lambda *a: pdlib.pd_paged_kv4_decode_attention_workspace_bytes(c, *a)  # noqa: E731
    room = need(most, n_new, longest)
    calls_ = [(b, m, n) for b in (1, 2, 18, most) for m in {1, 2, n_new} for n in (n_new, 257, 4097, longest // 2, longest)]
    calls_ += [(int(rng.integers(1, most + 1)), int(rng.integers(1, n_new + 1)), int(np.exp(rng.uniform(np.log(n_new), np.log(longest))))) for _ in range(80)]
    for b, m, n in calls_:
        if b > most or m > n_new or n > longest:
            continue
        n = max(n, m)
        assert need(b, m, n) <= room
        assert need(b, m, n) <= min(need(b + 1, m, n), need(b, m + 1, n), need(b, m, n + 1))
        refused(pdlib, pdlib.PD_ERR_CUDA, calls(pdlib)["decode"], c=c, k=k, t=None, batch=b, n_new=m, max_kv_len=n, workspace_bytes=room)

"""Argument checks of the 8-bit serving calls: every refusal precedes any device call, so no GPU is needed.  The pointers are
never read; they only have to be non-zero and aligned."""
import ctypes

import pytest

PTR = 1 << 20


def cache(pd, **kw):
    a = dict(k_codes=PTR, v_codes=PTR, k_scales=PTR, v_scales=PTR, page_table=PTR, n_pages=8, page_len=64, n_seqs=4, table_ld=4)
    a.update(kw)
    return pd.paged_kv_cache_struct(**a)


def cfg(pd, hq=8, hkv=2, hd=64, max_pos=256):
    return pd.LayerConfig(hq * hd, hq, hkv, hd, 64, max_pos=max_pos)


def refused(pd, status, f, *a, **kw):
    with pytest.raises(pd.PdError) as e:
        f(*a, stream=0, **kw)
    assert e.value.status == status, (a, kw)


def test_struct_layout(pdlib):
    assert ctypes.sizeof(pdlib.pd_paged_kv_cache) == 8 + 5 * 8 + 4 * 4


BAD_CACHES = [dict(k_codes=None), dict(v_codes=None), dict(k_scales=None), dict(v_scales=None), dict(page_table=None),
              dict(n_pages=0), dict(n_seqs=0), dict(table_ld=0), dict(k_codes=PTR + 8), dict(v_scales=PTR + 2)]
BAD_SHAPES = [dict(page_len=0), dict(page_len=24), dict(page_len=256), dict(page_len=8), dict(table_ld=1 << 25)]


def calls(pd):
    """The three cache calls as functions of (cfg, cache) with otherwise valid arguments."""
    return [lambda c, k, **kw: pd.pd_paged_kv_append(c, PTR, (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, PTR, PTR, k, PTR, 2, **kw),
            lambda c, k, **kw: pd.pd_paged_decode_attention(c, PTR, c.n_q_heads * c.head_dim, PTR, PTR, 2, 100, k, PTR, 1 << 30, **kw),
            lambda c, k, **kw: pd.pd_paged_prefill_attention(c, PTR, c.n_q_heads * c.head_dim, PTR, PTR, [0, 5], PTR, [3], k, PTR, 1 << 30, **kw)]


@pytest.mark.parametrize("which", range(3))
def test_cache_description(pdlib, which):
    f = calls(pdlib)[which]
    for bad in BAD_CACHES:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, cfg(pdlib), cache(pdlib, **bad))
    for bad in BAD_SHAPES:
        refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, f, cfg(pdlib), cache(pdlib, **bad))
    c = cache(pdlib)
    c.struct_size = 8
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, f, cfg(pdlib), c)


@pytest.mark.parametrize("which", range(3))
def test_head_shapes(pdlib, which):
    f = calls(pdlib)[which]
    for hq, hkv, hd, st in [(8, 2, 96, "UNSUPPORTED_SHAPE"), (8, 3, 64, "UNSUPPORTED_SHAPE"), (34, 2, 64, "UNSUPPORTED_SHAPE"),
                            (0, 2, 64, "INVALID_ARG"), (8, 0, 64, "INVALID_ARG"), (8, -2, 64, "INVALID_ARG")]:
        refused(pdlib, getattr(pdlib, "PD_ERR_" + st), f, cfg(pdlib, hq, hkv, hd), cache(pdlib))


def test_append_arguments(pdlib):
    c, k = cfg(pdlib), cache(pdlib)
    ok = dict(cfg=c, qkv=PTR, ldqkv=768, q_out=PTR, rope_tab=PTR, cache=k, kv_len_dev=PTR, n_req=2)
    for bad in [dict(qkv=None), dict(rope_tab=None), dict(kv_len_dev=None), dict(ldqkv=760), dict(ldqkv=772), dict(qkv=PTR + 2),
                dict(q_out=PTR + 8), dict(rope_tab=PTR + 4), dict(n_req=-1), dict(n_req=5), dict(cfg=cfg(pdlib, max_pos=0)),
                dict(n_req=2, cu_seqlens_host=[0, 1, 2]), dict(n_req=2, cu_seqlens_dev=PTR),
                dict(cu_seqlens_dev=PTR, cu_seqlens_host=[1, 1, 2]), dict(cu_seqlens_dev=PTR, cu_seqlens_host=[0, 3, 2])]:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, lambda stream, a: pdlib.pd_paged_kv_append(stream=stream, **a), a={**ok, **bad})
    with pytest.raises(ValueError):
        pdlib.pd_paged_kv_append(**{**ok, "cu_seqlens_dev": PTR, "cu_seqlens_host": [0, 1]}, stream=0)
    # nothing to do is not an error, and needs no device
    pdlib.pd_paged_kv_append(**{**ok, "n_req": 0}, stream=0)
    pdlib.pd_paged_kv_append(**{**ok, "cu_seqlens_dev": PTR, "cu_seqlens_host": [0, 0, 0]}, stream=0)


def test_decode_attention_arguments(pdlib):
    c, k = cfg(pdlib), cache(pdlib)
    need = pdlib.pd_paged_decode_attention_workspace_bytes(c, 1, 256)
    ok = dict(cfg=c, q=PTR, ldq=512, out=PTR, kv_len_dev=PTR, batch=1, max_kv_len=256, cache=k, workspace=PTR, workspace_bytes=need)
    call = lambda stream, a: pdlib.pd_paged_decode_attention(stream=stream, **a)  # noqa: E731
    for bad in [dict(q=None), dict(out=None), dict(kv_len_dev=None), dict(ldq=504), dict(ldq=514), dict(q=PTR + 4), dict(out=PTR + 1),
                dict(batch=-1), dict(batch=5), dict(max_kv_len=0), dict(max_kv_len=257)]:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, a={**ok, **bad})
    big = cache(pdlib, table_ld=1 << 12)
    split = {**ok, "cache": big, "max_kv_len": 1 << 15}
    need = pdlib.pd_paged_decode_attention_workspace_bytes(c, 1, 1 << 15)
    assert need > 0
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, a={**split, "workspace": None, "workspace_bytes": need})
    refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, a={**split, "workspace": PTR + 128, "workspace_bytes": need})
    refused(pdlib, pdlib.PD_ERR_WORKSPACE_TOO_SMALL, call, a={**split, "workspace_bytes": need - 1})
    wide = cache(pdlib, n_seqs=70000)
    refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, call, a={**ok, "cache": wide, "batch": 65536})
    call(0, {**ok, "batch": 0})


def test_prefill_attention_arguments(pdlib):
    c, k = cfg(pdlib), cache(pdlib)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(c, 2, 210)
    assert need > 0 and pdlib.pd_paged_prefill_attention_workspace_bytes(c, 0, 128) == 0
    ok = dict(cfg=c, q=PTR, ldq=512, out=PTR, cu_seqlens_dev=PTR, cu_seqlens_host=[0, 10, 15], prefix_dev=PTR, prefix_host=[200, 3],
              cache=k, workspace=PTR, workspace_bytes=need)
    call = lambda stream, a: pdlib.pd_paged_prefill_attention(stream=stream, **a)  # noqa: E731
    for bad in [dict(q=None), dict(out=None), dict(cu_seqlens_dev=None), dict(ldq=504), dict(ldq=516), dict(q=PTR + 8), dict(out=PTR + 16),
                dict(cu_seqlens_host=[1, 10, 15]), dict(cu_seqlens_host=[0, 10, 5]), dict(prefix_host=[-1, 0]), dict(prefix_dev=None),
                dict(prefix_host=[250, 0]), dict(prefix_host=[2 ** 31 - 5, 0]), dict(workspace=None), dict(workspace=PTR + 64),
                dict(cu_seqlens_host=[0, 1, 2, 3, 4, 5], prefix_host=[0] * 5)]:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, a={**ok, **bad})
    refused(pdlib, pdlib.PD_ERR_WORKSPACE_TOO_SMALL, call, a={**ok, "workspace_bytes": need - 1})
    with pytest.raises(ValueError):
        call(0, {**ok, "prefix_host": [1]})
    call(0, {**ok, "cu_seqlens_host": [0, 0, 0]})


def test_add_rmsnorm_arguments(pdlib):
    ok = dict(x=PTR, rows=4, d=256, gain=PTR, codes=PTR, scales=PTR, residual=PTR, sum_out=PTR + (1 << 16), norm_out=PTR)
    call = lambda stream, a: pdlib.pd_add_rmsnorm_fp8(stream=stream, **a)  # noqa: E731
    for bad in [dict(x=None), dict(gain=None), dict(scales=None), dict(codes=None, norm_out=None), dict(rows=-1), dict(d=0), dict(d=-128),
                dict(group=64), dict(group=-1), dict(ldx=248), dict(ldx=260), dict(ldr=252), dict(x=PTR + 2), dict(residual=PTR + 8),
                dict(gain=PTR + 4), dict(sum_out=PTR + 8), dict(norm_out=PTR + 8), dict(codes=PTR + 8), dict(scales=PTR + 2),
                dict(eps=-1.0), dict(eps=float("nan")), dict(sum_out=PTR, ldx=264), dict(x=PTR + 4096, sum_out=PTR, ldr=264)]:
        refused(pdlib, pdlib.PD_ERR_INVALID_ARG, call, a={**ok, **bad})
    for bad in [dict(d=192), dict(d=200, group=0), dict(d=16512), dict(d=16400, group=0)]:
        refused(pdlib, pdlib.PD_ERR_UNSUPPORTED_SHAPE, call, a={**ok, **bad})
    call(0, {**ok, "rows": 0})


def test_rope_table_arguments(pdlib):
    for bad in [dict(max_pos=0), dict(max_pos=-3)]:
        with pytest.raises(pdlib.PdError):
            pdlib.pd_rope_table(cfg(pdlib, **bad))
    with pytest.raises(pdlib.PdError) as e:
        pdlib.pd_rope_table(cfg(pdlib, hd=80))
    assert e.value.status == pdlib.PD_ERR_UNSUPPORTED_SHAPE

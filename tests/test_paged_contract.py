"""What the header says of the 8-bit serving calls, as far as that needs no GPU."""
import numpy as np
import pytest
import torch


@pytest.mark.parametrize("hq,hkv,hd", [(32, 8, 128), (8, 2, 64), (16, 1, 128), (64, 64, 128), (5, 5, 64), (2048, 512, 64)])
def test_decode_workspace_of_the_largest_call_serves_smaller_ones(pdlib, hq, hkv, hd):
    """The size does not fall as the batch or the length bound grows, and is enough for the parts that the call makes:
    the rows of a part hold hd sums, a maximum and a weight in fp32."""
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    need = lambda b, n: pdlib.pd_paged_decode_attention_workspace_bytes(cfg, b, n)  # noqa: E731
    rng = np.random.default_rng(hq)
    batches = sorted({0, 1, 2, 3, 8, 18, 19, 37, 74, 75, 148, 149, 256, 1000, 65535} | set(int(v) for v in rng.integers(1, 400, 20)))
    lengths = sorted({0, 1, 255, 256, 257, 2304, 4096, 4097, 8192, 9472, 9473, 32768, 65535, 65536, 65551, 1 << 20, (1 << 27) + 5, (1 << 31) - 300, (1 << 31) - 1} |
                     set(int(v) for v in np.exp(rng.uniform(3, 15, 30))))
    table = np.array([[need(b, n) for n in lengths] for b in batches], dtype=np.int64)
    assert (np.diff(table, axis=0) >= 0).all() and (np.diff(table, axis=1) >= 0).all()
    assert table[-1, -1] < 1 << 40


@pytest.mark.parametrize("hq,hkv,hd,most,longest", [(32, 8, 128, 256, 2304), (32, 8, 128, 256, 9473), (16, 1, 64, 200, 70000), (64, 64, 128, 40, 2000000)])
def test_decode_call_takes_the_workspace_of_a_larger_call(pdlib, hq, hkv, hd, most, longest):
    """One buffer sized for the largest batch: no smaller call refuses it.  (A call that gets past its checks here fails for want
    of a GPU, with another status.)"""
    if torch.cuda.is_available():
        pytest.skip("the pointers of this test are not to reach a GPU")
    ptr, rng = 1 << 20, np.random.default_rng(most)
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    k = pdlib.paged_kv_cache_struct(ptr, ptr, ptr, ptr, ptr, 8, 64, most, 1 << 15)
    room = pdlib.pd_paged_decode_attention_workspace_bytes(cfg, most, longest)
    calls = [(b, n) for b in (1, 2, 18, 19, most) for n in (1, 257, longest // 2, longest)]
    calls += [(int(rng.integers(1, most + 1)), int(np.exp(rng.uniform(0, np.log(longest))))) for _ in range(60)]
    for batch, n in calls:
        with pytest.raises(pdlib.PdError) as e:
            pdlib.pd_paged_decode_attention(cfg, ptr, hq * hd, ptr, ptr, batch, n, k, ptr, room, stream=0)
        assert e.value.status == pdlib.PD_ERR_CUDA, (batch, n)


def test_prefill_ignores_the_prefix_of_a_request_without_rows(pdlib):
    """A padded batch that shares its length array with the append (-1: left out) is no error as long as such a request brings no
    row; with rows it still is."""
    if torch.cuda.is_available():
        pytest.skip("the pointers of this test are not to reach a GPU")
    ptr = 1 << 20
    cfg = pdlib.LayerConfig(512, 8, 2, 64, 64)
    k = pdlib.paged_kv_cache_struct(ptr, ptr, ptr, ptr, ptr, 8, 64, 4, 4)
    need = pdlib.pd_paged_prefill_attention_workspace_bytes(cfg, 3, 256)
    call = lambda cu, pre: pdlib.pd_paged_prefill_attention(cfg, ptr, 512, ptr, ptr, cu, ptr, pre, k, ptr, need, stream=0)  # noqa: E731
    call([0, 0, 0], [-1, 5])                                  # no rows at all: nothing to do
    call([0, 0, 0], [1 << 20, -(1 << 31)])
    for cu, pre, status in [([0, 0, 7, 7], [-1, 3, -5], pdlib.PD_ERR_CUDA), ([0, 7, 7, 9], [0, 1000, 100], pdlib.PD_ERR_CUDA),
                            ([0, 1, 7, 9], [-1, 3, 0], pdlib.PD_ERR_INVALID_ARG), ([0, 1, 7, 7], [256, 3, 0], pdlib.PD_ERR_INVALID_ARG)]:
        with pytest.raises(pdlib.PdError) as e:
            call(cu, pre)
        assert e.value.status == status, (cu, pre)


def test_every_c_struct_is_the_callers_own(pdlib):
    """A caller may change the struct that c_struct() returns; the configuration and its later calls do not notice."""
    import copy
    import pickle
    cfg = pdlib.LayerConfig(512, 8, 2, 64, 64, max_pos=4)
    want = pdlib.pd_rope_table(cfg)                       # (a call that has used the configuration's struct)
    mine = cfg.c_struct()
    mine.max_pos, mine.head_dim = 0, 7
    assert cfg.c_struct().max_pos == 4 and cfg.c_struct().head_dim == 64
    np.testing.assert_array_equal(pdlib.pd_rope_table(cfg), want)
    for other in (copy.copy(cfg), copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg))):
        assert other == cfg and hash(other) == hash(cfg)
        np.testing.assert_array_equal(pdlib.pd_rope_table(other), want)

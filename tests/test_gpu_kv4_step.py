"""GPU: the operators around the 4-bit paged KV cache run together as the attention half of a layer is served: projection, norm and
rotation and append, prefill attention over what is read back, decode steps and drafted tokens over the pages; eager, captured,
on two streams; and with pools of more than 4 GB."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from kv4_util import Cache4, Transform, check_attention, transform_bound
from oracle import paged, paged4
from paged_util import BF16, assert_within, attention_bound
from test_gpu_kv4_append import append, expect, rows_of
from test_gpu_kv4_attention import check, decode, queries

pytestmark = pytest.mark.gpu
HQ, HKV, HD, D, PAGE = 8, 2, 128, 512, 32
N_QKV = (HQ + 2 * HKV) * HD


class Half:
    """Device weights and buffers for up to `rows` rows; the transform's table comes from the library."""

    def __init__(self, pd, cache, rows, n_req, max_kv, n_new=1):
        import torch
        self.pd, self.c, self.max_kv, self.n_req = pd, cache, max_kv, n_req
        self.cfg = pd.LayerConfig(D, HQ, HKV, HD, D)
        self.w = gen.normal_bf16(1, 1, (N_QKV, D), 0.05)
        self.t = Transform(pd, HD, 96, max_kv, pairs=True, seed=2)
        rope = pd.RopeConfig(96, scaling=pd.ROPE_SCALE_TURNS, factor=8.0, trained_len=128, low=1.0, high=4.0, magnitude=1.1)
        self.t.cs = paged4.table(paged4.frequencies(96, 1e4, "turns", 8.0, 128, 1.0, 4.0), np.arange(max_kv), 1.1).astype(np.float32)
        pd.pd_rope_table_scaled(rope, 0, max_kv, self.t.dtab)
        torch.cuda.synchronize()
        got = self.t.dtab.cpu().numpy()
        assert np.abs(got - self.t.cs).max() <= 1.1 * 2.0 ** -23
        self.t.cs = got                       # (codes are decided by the table that is there)
        z = lambda *s: torch.zeros(s, dtype=torch.int16, device="cuda")  # noqa: E731
        self.dw, self.x, self.qkv, self.q, self.o = to_dev(self.w), z(rows, D), z(rows, N_QKV), z(rows, HQ * HD), z(rows, HQ * HD)
        self.kv, self.err = i32_dev([0] * n_req), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws_bytes = pd.pd_paged_kv4_decode_attention_workspace_bytes(self.cfg, n_req, n_new, max_kv)
        self.ws = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device="cuda")

    def project_and_append(self, rows, cu=None, stream=None):
        self.pd.pd_gemm_bf16(self.x, self.dw, self.qkv, rows, N_QKV, D, err_word=self.err, stream=stream)
        self.pd.pd_paged_kv4_append(self.cfg, self.t.struct, self.qkv, N_QKV, self.q, self.c.struct, self.kv, self.n_req,
                                    cu_seqlens_dev=None if cu is None else i32_dev(cu), cu_seqlens_host=cu, err_word=self.err, stream=stream)

    def attend(self, n_new=1, stream=None):
        self.pd.pd_paged_kv4_decode_attention(self.cfg, self.q, HQ * HD, self.o, self.kv, self.n_req, n_new, self.max_kv, self.c.struct,
                                              self.ws, self.ws_bytes, err_word=self.err, stream=stream)

    def check_append(self, kv, cu):
        import torch
        torch.cuda.synchronize()
        assert int(self.err.item()) == 0
        rows = cu[-1]
        expect(self.c, self.t, from_dev(self.qkv[:rows]).reshape(rows, -1, HD), kv, cu, from_dev(self.q[:rows]).reshape(rows, HQ, HD))
        self.c.assert_equal()


def test_prompts_chunks_steps_and_drafts(pdlib):
    import torch
    new, chunk, steps, draft = [150, 33, 1], [40, 7, 65], 4, 3
    final = [a + b + steps + draft for a, b in zip(new, chunk)]
    c = Cache4(pdlib, HKV, HD, PAGE, final, seed=40).upload()
    h = Half(pdlib, c, sum(new), 3, max(final), n_new=draft)
    flat = torch.full((2, 3, HKV, max(final), HD), -1, dtype=torch.int16, device="cuda")      # NaN where nothing is read back
    back = pdlib.kv_cache_struct(flat[0], flat[1], 3, max(final))
    kv = [0, 0, 0]
    for part in (new, chunk):                                   # whole prompts, then chunks over cached prefixes
        cu = np.r_[0, np.cumsum(part)].tolist()
        after = [a + b for a, b in zip(kv, part)]
        h.x[:cu[-1]] = to_dev(gen.normal_bf16(50, 4, (cu[-1], D), 1.0, sub=cu[-1]))
        h.kv.copy_(i32_dev(kv))
        h.project_and_append(cu[-1], cu)
        h.check_append(kv, cu)
        pdlib.pd_paged_kv4_read(h.cfg, c.struct, None, i32_dev(after), 3, max(after), back, err_word=h.err)
        pdlib.pd_prefill_attention(h.cfg, h.q, HQ * HD, h.o, i32_dev(cu), cu, back, prefix_dev=h.kv, prefix_host=kv, err_word=h.err)
        q, o = (from_dev(t[:cu[-1]]).reshape(-1, HQ, HD) for t in (h.q, h.o))
        assert int(h.err.item()) == 0
        for s in range(3):
            sel = np.unique(np.r_[0, part[s] // 2, part[s] - 1])
            keys, vals = c.kv(s, after[s])
            ref, spread, score = paged.attend(q[cu[s] + sel], keys, vals, kv[s] + sel)
            # the prefill kernel's weights are bf16, in the product and in their sum
            assert_within(o[cu[s] + sel], ref, attention_bound(ref, spread, score, 2 * BF16), f"request {s}")
        kv = after
    for i in range(steps):                                      # a token each
        h.x[:3] = to_dev(gen.normal_bf16(51, 4, (3, D), 1.0, sub=i))
        h.kv.copy_(i32_dev(kv))
        h.project_and_append(3)
        h.check_append(kv, [0, 1, 2, 3])
        h.attend()
        q, o = (from_dev(t[:3]).reshape(3, 1, HQ, HD) for t in (h.q, h.o))
        check(c, HQ, q, kv, o)
        kv = [k + 1 for k in kv]
    cu = [0, draft, 2 * draft, 3 * draft]                       # several drafted tokens each, verified together
    h.x[:cu[-1]] = to_dev(gen.normal_bf16(52, 4, (cu[-1], D), 1.0))
    h.kv.copy_(i32_dev(kv))
    h.project_and_append(cu[-1], cu)
    h.check_append(kv, cu)
    h.attend(draft)
    q, o = (from_dev(t[:cu[-1]]).reshape(3, draft, HQ, HD) for t in (h.q, h.o))
    check(c, HQ, q, kv, o, draft)
    # of which one is kept: the next step appends over the others
    kv = [k + 1 for k in kv]
    h.x[:3] = to_dev(gen.normal_bf16(53, 4, (3, D), 1.0))
    h.kv.copy_(i32_dev(kv))
    h.project_and_append(3)
    h.check_append(kv, [0, 1, 2, 3])
    h.attend()
    check(c, HQ, from_dev(h.q[:3]).reshape(3, 1, HQ, HD), kv, from_dev(h.o[:3]).reshape(3, 1, HQ, HD))


def test_captured_steps_are_the_eager_ones(pdlib):
    """A graph of append, attention and the growth of the lengths, replayed; a sequence that is left out."""
    import torch
    steps, kv = 5, [30, 0, -(1 << 20), 100]
    final = [max(0, k) + steps for k in kv]
    runs = []
    for captured in (False, True):
        c = Cache4(pdlib, HKV, HD, PAGE, final, seed=41).fill([max(0, k) for k in kv], np.random.default_rng(41)).upload()
        h = Half(pdlib, c, 4, 4, max(final))
        xs = to_dev(gen.normal_bf16(54, 4, (steps, 4, D), 1.0))
        h.kv.copy_(i32_dev(kv))
        outs = []
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())

        def step():
            h.project_and_append(4, stream=s)
            h.attend(stream=s)
            h.kv.add_(1)

        with torch.cuda.stream(s):
            if captured:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    step()
            for i in range(steps):
                h.x.copy_(xs[i])
                g.replay() if captured else step()
                outs.append(h.o.clone())
        s.synchronize()
        assert int(h.err.item()) == 0
        runs.append((outs, c))
    (a, ca), (b, cb) = runs
    for x, y in zip(a, b):
        assert (x == y).all() and not x[2].any()
    for name in ("dk", "dv", "dks", "dvs"):
        assert (getattr(ca, name) == getattr(cb, name)).all()


def test_two_calls_at_once(pdlib):
    """Two captured decode attentions with a workspace each, replayed on two streams side by side, many times."""
    import torch
    c = Cache4(pdlib, HKV, HD, 64, [5000, 3000], seed=42).fill([5000, 3000], np.random.default_rng(42), 0.5).upload()
    cfg = pdlib.LayerConfig(D, HQ, HKV, HD, D)
    work = []
    for i in range(2):
        q = to_dev(queries(80 + i, 2, 1, HQ, HD).reshape(2, -1))
        need = pdlib.pd_paged_kv4_decode_attention_workspace_bytes(cfg, 2, 1, 5000)
        assert need > 0
        work.append(dict(q=q, out=empty_bf16(2, HQ * HD), ws=torch.empty(need, dtype=torch.uint8, device="cuda"), need=need,
                         kv=i32_dev([4999 - i, 2999 - 7 * i]), s=torch.cuda.Stream(), g=torch.cuda.CUDAGraph()))

    def call(w):
        pdlib.pd_paged_kv4_decode_attention(cfg, w["q"], HQ * HD, w["out"], w["kv"], 2, 1, 5000, c.struct, w["ws"], w["need"], stream=w["s"])

    want = []
    for w in work:
        call(w)
        w["s"].synchronize()
        want.append(w["out"].clone())
        with torch.cuda.stream(w["s"]):
            with torch.cuda.graph(w["g"], stream=w["s"]):
                call(w)
    for w in work:
        w["out"].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for w in work:
            with torch.cuda.stream(w["s"]):
                w["g"].replay()
    torch.cuda.synchronize()
    for w, x in zip(work, want):
        assert (w["out"] == x).all()


def test_work_goes_to_the_stream_that_is_given(pdlib):
    """Behind what that stream waits for, not behind the default stream: lengths and rows arrive late."""
    import torch
    c = Cache4(pdlib, HKV, HD, 16, [100, 40], seed=43).fill([99, 39], np.random.default_rng(43)).upload()
    ref = Cache4(pdlib, HKV, HD, 16, [100, 40], seed=43).fill([99, 39], np.random.default_rng(43)).upload()
    t = Transform(pdlib, HD, 64, 128)
    x = rows_of(44, 2, HQ, HKV, HD)
    q = append(pdlib, ref, t, x, [99, 39])
    want = decode(pdlib, ref, HQ, q, [99, 39])
    cfg = pdlib.LayerConfig(D, HQ, HKV, HD, D)
    s = torch.cuda.Stream()
    src, src_kv = to_dev(x.reshape(2, -1)), i32_dev([99, 39])
    dx, kv, dq, out = torch.zeros_like(src), i32_dev([-1, -1]), empty_bf16(2, HQ * HD), empty_bf16(2, HQ * HD)
    ws_bytes = pdlib.pd_paged_kv4_decode_attention_workspace_bytes(cfg, 2, 1, 100)
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        dx.copy_(src)
        kv.copy_(src_kv)
    pdlib.pd_paged_kv4_append(cfg, t.struct, dx, N_QKV, dq, c.struct, kv, 2, stream=s)
    pdlib.pd_paged_kv4_decode_attention(cfg, dq, HQ * HD, out, kv, 2, 1, 100, c.struct, ws, ws_bytes, stream=s)
    s.synchronize()
    np.testing.assert_array_equal(from_dev(out).reshape(2, 1, HQ, HD), want)


def test_from_a_bf16_cache(pdlib):
    """What a prefill instance left in bf16 goes into the pages; attention over the pages and bf16 attention over what is read back
    see the same values."""
    import torch
    lens = [700, 64, 3]
    k, v = gen.kv_cache(60, 3, HKV, 720, HD)
    dk, dv = to_dev(k), to_dev(v)
    c = Cache4(pdlib, HKV, HD, PAGE, lens, seed=45).upload()
    cfg = pdlib.LayerConfig(D, HQ, HKV, HD, D)
    flat = pdlib.kv_cache_struct(dk, dv, 3, 720)
    pdlib.pd_paged_kv4_write(cfg, c.struct, None, i32_dev(lens), 3, 720, flat)
    for s, n in enumerate(lens):
        paged4.append(c.k, c.ks, c.table[s], 0, k[s, :, :n].transpose(1, 0, 2), c.ke)
        paged4.append(c.v, c.vs, c.table[s], 0, v[s, :, :n].transpose(1, 0, 2), c.ve)
    c.assert_equal()
    pdlib.pd_paged_kv4_read(cfg, c.struct, None, i32_dev(lens), 3, 720, flat)
    q = queries(85, 3, 1, HQ, HD)
    kv_len = [n - 1 for n in lens]
    got = decode(pdlib, c, HQ, q, kv_len)
    check(c, HQ, q, kv_len, got)
    out = empty_bf16(3, HQ * HD)
    ws_bytes = pdlib.pd_decode_attention_workspace_bytes(cfg, 3, 720)
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device="cuda")
    pdlib.pd_decode_attention(cfg, to_dev(q.reshape(3, -1)), HQ * HD, out, i32_dev(kv_len), 3, 720, flat, ws, ws_bytes)
    bf = from_dev(out).reshape(3, HQ, HD)
    for s, n in enumerate(lens):
        o, spread, score = paged.attend(q[s], *c.kv(s, n), [n - 1])
        assert_within(bf[s:s + 1], o, attention_bound(o, spread, score, 2 * BF16), f"bf16, sequence {s}")


def test_pools_of_more_than_four_gigabytes(pdlib):
    """Pages at the end of a pool whose byte offsets pass 32 bits, for every call."""
    import torch
    hq, hkv, hd, page = 4, 2, 128, 128
    codes = hkv * page * hd // 2                                # bytes of a page
    n_pages = (1 << 32) // codes + 5000
    if torch.cuda.mem_get_info()[0] < 3 * n_pages * codes:
        pytest.skip("needs 10 GB of device memory")
    lens = [300, 130]
    small = Cache4(pdlib, hkv, hd, page, lens, seed=46)         # the same sequences in a small pool, and what the oracle expects
    far = {k: torch.empty((n_pages, hkv, page, hd // w), dtype=torch.uint8, device="cuda") for k, w in (("k", 2), ("v", 2), ("ks", 16), ("vs", 16))}
    assert far["k"].numel() > 1 << 32
    ids = n_pages - 1 - np.arange(small.n_pages) * 401
    table = np.where(small.table >= 0, ids[np.maximum(small.table, 0)], -1).astype(np.int32)
    dt, ke, ve = i32_dev(table), i32_dev(small.k_exp), i32_dev(small.v_exp)
    small.struct = pdlib.paged_kv4_cache_struct(far["k"], far["v"], far["ks"], far["vs"], dt, n_pages, page, 2, small.width, k_exp=ke, v_exp=ve)
    t = Transform(pdlib, hd, hd, 512)
    cu = [0, 300, 430]
    x = rows_of(47, 430, hq, hkv, hd)
    q = append(pdlib, small, t, x, [0, 0], cu)
    small.k[:], small.ks[:] = 0, 0x7F
    expect(small, t, x, [0, 0], cu, q)
    for s, n in enumerate(lens):
        kv_len = [n - 1 if i == s else -1 for i in range(2)]
        qq = q[[299, 429]]
        got = decode(pdlib, small, hq, qq, kv_len, max_kv=300)
        check_attention(qq[s:s + 1], *small.kv(s, n), [n - 1], got[s])
    flat = torch.zeros((2, 2, hkv, 300, hd), dtype=torch.int16, device="cuda")
    cfg = pdlib.LayerConfig(hq * hd, hq, hkv, hd, 64)
    back = pdlib.kv_cache_struct(flat[0], flat[1], 2, 300)
    pdlib.pd_paged_kv4_read(cfg, small.struct, None, i32_dev(lens), 2, 300, back)
    for s, n in enumerate(lens):
        for got, want in zip(flat, small.kv(s, n)):
            np.testing.assert_array_equal(from_dev(got[s])[:, :n].transpose(1, 0, 2), want)
    for d in far.values():
        d[ids[0]:].fill_(0x7F)
    pdlib.pd_paged_kv4_write(cfg, small.struct, None, i32_dev(lens), 2, 300, back)
    again = torch.zeros_like(flat)
    pdlib.pd_paged_kv4_read(cfg, small.struct, None, i32_dev(lens), 2, 300, pdlib.kv_cache_struct(again[0], again[1], 2, 300))
    # (values of a group whose largest code is not 6 may take another scale, and the same values)
    for i in range(2):
        a, b = from_dev(flat[i]), from_dev(again[i])
        for s, n in enumerate(lens):
            c, sc = paged4.quantise(a[s, :, :n].astype(np.float64) * np.exp2(-(small.ke, small.ve)[i].astype(np.float64))[:, None, None])
            np.testing.assert_array_equal(b[s, :, :n], paged4.values(c, sc) * np.exp2((small.ke, small.ve)[i].astype(np.float64))[:, None, None])


def test_very_many_requests_and_sequences(pdlib):
    """More requests than the search takes in two rounds, and a batch of mostly short sequences under a bound that is a capacity."""
    rng = np.random.default_rng(48)
    n = 1500
    kv, new = rng.integers(0, 20, n), rng.integers(0, 4, n)
    new[[0, 700, n - 1]] = 0
    cu = np.r_[0, np.cumsum(new)].tolist()
    lens = (kv + new).tolist()
    c = Cache4(pdlib, 1, 64, 16, lens, seed=49, extra_cols=300).fill(kv.tolist(), rng).upload()
    t = Transform(pdlib, 64, 32, 64)
    x = rows_of(50, cu[-1], 2, 1, 64)
    q = append(pdlib, c, t, x, kv.tolist(), cu)
    expect(c, t, x, kv.tolist(), cu, q)
    c.assert_equal()
    kv_len = [v - 1 for v in lens]                             # -1 where a sequence is empty
    qd = queries(86, n, 1, 2, 64)
    check(c, 2, qd, kv_len, decode(pdlib, c, 2, qd, kv_len, max_kv=c.width * 16))


def test_the_same_pages_under_two_sequences(pdlib):
    """A shared prefix: two rows of the table name the same full pages; each continues on its own."""
    c = Cache4(pdlib, HKV, HD, 16, [80, 80], seed=51).fill([64, 64], np.random.default_rng(51))
    c.table[1, :4] = c.table[0, :4]
    c.upload()
    t = Transform(pdlib, HD, 64, 128)
    x = rows_of(52, 10, HQ, HKV, HD)
    q = append(pdlib, c, t, x, [64, 64], [0, 7, 10])
    expect(c, t, x, [64, 64], [0, 7, 10], q)
    c.assert_equal()
    check(c, HQ, q[[6, 9]], [70, 66], decode(pdlib, c, HQ, q[[6, 9]], [70, 66]))

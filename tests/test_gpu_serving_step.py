"""GPU: the 8-bit serving operators run together as one attention half of a layer: residual addition with RMSNorm and codes,
block-wise FP8 projection, append to the paged cache, attention over it, quantisation, output projection.  Every stage is held
to the oracle on the values that the stage before it left on the device; the decode steps are captured in a graph as well."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import fp8, paged
from paged_util import BF16, F16, Cache, assert_within, attention_bound
from test_gpu_norm_fp8 import check as check_norm

pytestmark = pytest.mark.gpu
HQ, HKV, HD, D, PAGE, THETA, EPS = 8, 2, 128, 1024, 32, 1e4, 1e-6


class Step:
    """Device weights and buffers of one such half for up to `rows` rows."""

    def __init__(self, pd, cache, rows, n_req, max_kv, seed=0):
        import torch
        self.pd, self.c, self.max_kv, self.n_req = pd, cache, max_kv, n_req
        self.n_qkv = (HQ + 2 * HKV) * HD
        self.cfg = pd.LayerConfig(D, HQ, HKV, HD, 4 * D, rope_theta=THETA, max_pos=max_kv)
        self.w_qkv, self.w_o = gen.normal_bf16(seed, 1, (self.n_qkv, D), 0.03), gen.normal_bf16(seed, 2, (D, HQ * HD), 0.03)
        self.gain = gen.normal_bf16(seed, 3, (D,), 0.05, 1.0)
        z = lambda *s, dt=torch.uint8: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
        f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        self.wq, self.wqs, self.wo, self.wos = z(self.n_qkv, D), f(self.n_qkv // 128, D // 128), z(D, HQ * HD), f(D // 128, HQ * HD // 128)
        pd.pd_quantize_fp8_blocks(to_dev(self.w_qkv), self.n_qkv, D, self.wq, self.wqs)
        pd.pd_quantize_fp8_blocks(to_dev(self.w_o), D, HQ * HD, self.wo, self.wos)
        self.dgain = to_dev(self.gain)
        self.tab = pd.pd_rope_table(self.cfg)
        self.dtab = torch.from_numpy(self.tab).cuda()
        self.x, self.r, self.h, self.out = (empty_bf16(rows, D) for _ in range(4))
        self.codes, self.scales = z(rows, D), f(rows, D // 128)
        self.qkv, self.q, self.o = empty_bf16(rows, self.n_qkv), empty_bf16(rows, HQ * HD), empty_bf16(rows, HQ * HD)
        self.oc, self.os = z(rows, HQ * HD), f(rows, HQ * HD // 128)
        self.kv = i32_dev([0] * n_req)
        need = max(pd.pd_paged_prefill_attention_workspace_bytes(self.cfg, n_req, max_kv),
                   pd.pd_paged_decode_attention_workspace_bytes(self.cfg, n_req, max_kv))
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, rows, cu=None, kv_host=None, stream=None):
        """x, r -> h, out on the rows; cu: a prefill pass, else one row per request."""
        pd, kw = self.pd, dict(err_word=self.err, stream=stream)
        pd.pd_add_rmsnorm_fp8(self.x, rows, D, self.dgain, self.codes, self.scales, residual=self.r, sum_out=self.h, eps=EPS, stream=stream)
        pd.pd_gemm_fp8_blockwise(self.codes, self.scales, self.wq, self.wqs, self.qkv, rows, self.n_qkv, D, **kw)
        dcu = None if cu is None else i32_dev(cu)
        pd.pd_paged_kv_append(self.cfg, self.qkv, self.n_qkv, self.q, self.dtab, self.c.struct, self.kv, self.n_req, cu_seqlens_dev=dcu,
                              cu_seqlens_host=cu, **kw)
        if cu is None:
            pd.pd_paged_decode_attention(self.cfg, self.q, HQ * HD, self.o, self.kv, self.n_req, self.max_kv, self.c.struct, self.ws,
                                         self.ws.numel(), **kw)
        else:
            pd.pd_paged_prefill_attention(self.cfg, self.q, HQ * HD, self.o, dcu, cu, self.kv, kv_host, self.c.struct, self.ws,
                                          self.ws.numel(), **kw)
        pd.pd_quantize_fp8_groups(self.o, rows, HQ * HD, self.oc, self.os, stream=stream)
        pd.pd_gemm_fp8_blockwise(self.oc, self.os, self.wo, self.wos, self.out, rows, D, HQ * HD, **kw)

    def check(self, rows, kv, new, x, r):
        """Every stage against the oracle on the stage's own inputs."""
        import torch
        torch.cuda.synchronize()
        assert int(self.err.item()) == 0
        check_norm(x, r, self.gain, 128, (self.h[:rows], None, self.codes[:rows], self.scales[:rows]), EPS)
        for codes, scales, wq, ws, got in ((self.codes, self.scales, self.wq, self.wqs, self.qkv), (self.oc, self.os, self.wo, self.wos, self.out)):
            a, s = codes[:rows].cpu().numpy(), scales[:rows].cpu().numpy()
            ref = fp8.gemm_fp8_blockwise(a, s, wq.cpu().numpy(), ws.cpu().numpy())
            mag = fp8.gemm_fp8_blockwise(a & 0x7F, s, wq.cpu().numpy() & 0x7F, ws.cpu().numpy())
            # one rounding to bf16; fp32 sums of K = 1024 scaled products
            assert np.all(np.abs(from_dev(got[:rows]) - ref) <= BF16 * np.abs(ref) + 1024 * 2.0 ** -23 * mag)
        qkv = from_dev(self.qkv[:rows]).reshape(rows, -1, HD)
        q = from_dev(self.q[:rows]).reshape(rows, HQ, HD)
        o = from_dev(self.o[:rows]).reshape(rows, HQ, HD)
        at = 0
        for s, (k, n) in enumerate(zip(kv, new)):
            part = qkv[at:at + n]
            rot = paged.rotate_f32(part[:, HQ:HQ + HKV], self.tab[k:k + n])
            paged.append(self.c.k, self.c.ks, self.c.table[s], k, rot)
            paged.append(self.c.v, self.c.vs, self.c.table[s], k, part[:, HQ + HKV:])
            half = np.abs(part[:, :HQ, :HD // 2]) + np.abs(part[:, :HQ, HD // 2:])
            ref = paged.rotate(part[:, :HQ], np.arange(k, k + n), THETA)
            assert np.all(np.abs(q[at:at + n] - ref) <= BF16 * np.abs(ref) + 2.0 ** -21 * np.concatenate([half, half], -1))
            keys, vals = self.c.kv(s, k + n)
            sel = np.unique(np.r_[0, n // 2, n - 1])
            ref, spread, score = paged.attend(q[at + sel], keys, vals, k + sel)
            assert_within(o[at + sel], ref, attention_bound(ref, spread, score, BF16 if n > 1 else F16), f"request {s}")
            at += n
        self.c.assert_equal()
        oq, os = fp8.quantize_groups(o.reshape(rows, -1))
        assert np.array_equal(self.oc[:rows].cpu().numpy(), oq) and np.array_equal(self.os[:rows].cpu().numpy(), os)

    def reference(self, x, r, keys, vals, kv, new):
        """The half in float64 without any 8-bit rounding; keys, vals: lists per request, extended."""
        _, n, _ = paged.add_rmsnorm(x, r, self.gain, EPS, 128)
        qkv = (n @ self.w_qkv.astype(np.float64).T).reshape(len(x), -1, HD)
        out, at = [], 0
        for s, (k, m) in enumerate(zip(kv, new)):
            part = qkv[at:at + m]
            rot = paged.rotate(part[:, :HQ + HKV], np.arange(k, k + m), THETA)
            keys[s] = np.concatenate([keys[s], rot[:, HQ:]])
            vals[s] = np.concatenate([vals[s], part[:, HQ + HKV:]])
            out.append(paged.attend(rot[:, :HQ], keys[s], vals[s], k + np.arange(m))[0].reshape(m, -1))
            at += m
        return np.concatenate(out) @ self.w_o.astype(np.float64).T


def inputs(seed, rows):
    return gen.normal_bf16(seed, 4, (rows, D), 1.0), gen.normal_bf16(seed, 5, (rows, D), 1.0)


def test_prompt_then_decode_steps(pdlib):
    import torch
    new, steps = [70, 33, 1], 6
    final = [n + steps for n in new]
    c = Cache(pdlib, HKV, HD, PAGE, final, seed=40, fill=0xAB).upload()
    st = Step(pdlib, c, sum(new), 3, max(final))
    x, r = inputs(50, sum(new))
    st.x.copy_(to_dev(x))
    st.r.copy_(to_dev(r))
    cu = [0, 70, 103, 104]
    st.run(104, cu, [0, 0, 0])
    st.check(104, [0, 0, 0], new, x, r)
    keys, vals = [np.zeros((0, HKV, HD))] * 3, [np.zeros((0, HKV, HD))] * 3
    ref, got = [st.reference(x, r, keys, vals, [0, 0, 0], new)], [from_dev(st.out[:104])]
    for i in range(steps):
        kv = [n + i for n in new]
        x, r = inputs(60 + i, 3)
        st.x[:3].copy_(to_dev(x))
        st.r[:3].copy_(to_dev(r))
        st.kv.copy_(i32_dev(kv))
        st.run(3)
        st.check(3, kv, [1, 1, 1], x, r)
        ref.append(st.reference(x, r, keys, vals, kv, [1, 1, 1]))
        got.append(from_dev(st.out[:3]))
    # six operands are rounded to E4M3 on the way (n, W_qkv, k, v, o, W_o), each by at most 2^-4 of itself and 2^-4 / sqrt(3) in
    # the mean square; independent roundings add up to sqrt(6) of that, 9 %, and the scores' errors act once more through p
    ref, got = np.concatenate(ref), np.concatenate(got)
    assert np.linalg.norm(got - ref) <= 0.2 * np.linalg.norm(ref)


def test_captured_decode_step_equals_eager_steps(pdlib):
    """One graph of a whole step, kv_len advancing on the device, with a padding row in the batch."""
    import torch
    start, steps, n = [40, 0, -1, 17], 40, 4
    final = [max(s, 0) + steps for s in start]
    both = []
    for captured in (False, True):
        c = Cache(pdlib, HKV, HD, PAGE, final, seed=41, fill=0xAB)
        c.fill([max(s, 0) for s in start], np.random.default_rng(1))
        c.upload()
        st = Step(pdlib, c, n, n, max(final))
        st.kv.copy_(i32_dev(start))
        live = i32_dev([int(s >= 0) for s in start])
        outs = []
        if captured:
            s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            st.c.struct = c.struct
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(g, stream=s):
                st.run(n)
                st.kv += live
        for i in range(steps):
            x, r = inputs(70 + i, n)
            st.x.copy_(to_dev(x))
            st.r.copy_(to_dev(r))
            if captured:
                g.replay()
            else:
                st.run(n)
                st.kv += live
            torch.cuda.synchronize()
            outs.append(st.out.clone())
        assert int(st.err.item()) == 0
        assert not st.o[2].any()      # the padding row's attention
        both.append((outs, c.dk, c.dv, c.dks.view(torch.int32), c.dvs.view(torch.int32)))
    for a, b in zip(both[0][0], both[1][0]):
        live = [0, 1, 3]
        assert torch.equal(a[live], b[live])
    for a, b in zip(both[0][1:], both[1][1:]):
        assert torch.equal(a, b)


def test_two_streams_at_once(pdlib):
    """Independent batches on two streams, each with its own cache and workspace, give what they give alone."""
    import torch
    sets = []
    for k in range(2):
        c = Cache(pdlib, HKV, HD, PAGE, [600 + 40] * 3, seed=42 + k)
        c.fill([600] * 3, np.random.default_rng(2 + k))
        c.upload()
        st = Step(pdlib, c, 3 * 40, 3, 640, seed=k)
        st.kv.copy_(i32_dev([600] * 3))
        x, r = inputs(80 + k, 120)
        st.x.copy_(to_dev(x))
        st.r.copy_(to_dev(r))
        sets.append(st)
    cu = [0, 40, 80, 120]
    alone = []
    for st in sets:
        st.run(120, cu, [600] * 3)
        torch.cuda.synchronize()
        alone.append(st.out.clone())
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for st, s in zip(sets, streams):
            st.run(120, cu, [600] * 3, stream=s)
    torch.cuda.synchronize()
    for st, a in zip(sets, alone):
        assert torch.equal(st.out, a) and int(st.err.item()) == 0

"""GPU: appending to the 8-bit paged KV cache against the oracle: codes and scales bit for bit over the whole pool, rotated q
within one bf16 rounding."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, i32_dev, to_dev
from oracle import paged
from paged_util import BF16, Cache

pytestmark = pytest.mark.gpu
THETA = 1e4


def qkv_rows(seed, n, hq, hkv, hd, spread=0.7):
    """bf16 rows whose k channels and tokens differ in size."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, hq + 2 * hkv, hd)) * np.exp(spread * rng.standard_normal((n, hq + 2 * hkv, 1)))
    x[:, hq:hq + hkv] *= np.exp(0.8 * rng.standard_normal((1, hkv, hd)))
    return gen.bf16_round(x)


class Appender:
    def __init__(self, pd, hq, hkv, hd, max_pos, page_len, final_lengths, seed=0, **kw):
        import torch
        self.pd, self.hq, self.hkv, self.hd = pd, hq, hkv, hd
        self.cfg = pd.LayerConfig(hq * hd, hq, hkv, hd, 64, rope_theta=THETA, max_pos=max_pos)
        self.tab = pd.pd_rope_table(self.cfg)
        self.dtab = torch.from_numpy(self.tab).cuda()
        self.c = Cache(pd, hkv, hd, page_len, final_lengths, seed, fill=0xAB, **kw).upload()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def __call__(self, rows, kv, new=None, pad=0, with_q=True, oracle=True):
        """rows [T, Hq + 2 Hkv, hd]; new = None: one row per request.  Returns q_out."""
        import torch
        t, width = rows.shape[0], (self.hq + 2 * self.hkv) * self.hd
        flat = np.full((t, width + pad), np.nan, np.float32)
        flat[:, :width] = rows.reshape(t, width)
        cu = None if new is None else [0] + [int(v) for v in np.cumsum(new)]
        q = empty_bf16(t + 1, self.hq * self.hd) if with_q else None
        self.pd.pd_paged_kv_append(self.cfg, to_dev(flat), width + pad, q, self.dtab, self.c.struct, i32_dev(kv), len(kv),
                                   cu_seqlens_dev=None if cu is None else i32_dev(cu), cu_seqlens_host=cu, err_word=self.err)
        torch.cuda.synchronize()
        if oracle:
            at = 0
            for s, k in enumerate(kv):
                n = 1 if new is None else new[s]
                if n and k >= 0:
                    part = rows[at:at + n]
                    rot = paged.rotate_f32(part[:, self.hq:self.hq + self.hkv], self.tab[k:k + n])
                    paged.append(self.c.k, self.c.ks, self.c.table[s], k, rot)
                    paged.append(self.c.v, self.c.vs, self.c.table[s], k, part[:, self.hq + self.hkv:])
                    if with_q:
                        got = from_dev(q[at:at + n]).reshape(n, self.hq, self.hd)
                        ref = paged.rotate(part[:, :self.hq], np.arange(k, k + n), THETA)
                        # half a bf16 step, and the fp32 rounding of two products, a sum and the table's entries
                        half = self.hd // 2
                        size = np.abs(part[:, :self.hq, :half]) + np.abs(part[:, :self.hq, half:])
                        bound = BF16 * np.abs(ref) + 2.0 ** -21 * np.concatenate([size, size], -1)
                        assert np.all(np.abs(got - ref) <= bound), (s, np.abs(got - ref).max())
                at += n
            assert not with_q or not q[t].any()
        return q


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (32, 8, 128), (16, 1, 128), (6, 6, 64), (24, 3, 64)])
@pytest.mark.parametrize("page_len", [16, 32, 64, 128])
def test_ragged_runs(pdlib, hq, hkv, hd, page_len):
    """Prefixes and lengths around the page boundaries, twice in a row (the second call joins the first one's pages)."""
    p = page_len
    kv = [0, 0, p - 1, 5, p, 3, 0, p + 1]
    new = [1, p, 2, 0, 2 * p + 1, p - 3, 3 * p + 7, 1]
    more = [p - 1, 1, 2 * p, 3, 0, 4, p, p - 2]
    final = [a + b + c for a, b, c in zip(kv, new, more)]
    ap = Appender(pdlib, hq, hkv, hd, max(final), p, final, seed=p + hd)
    ap.c.fill(kv, np.random.default_rng(7))
    ap.c.upload()
    ap(qkv_rows(p, sum(new), hq, hkv, hd), kv, new, pad=8)
    ap.c.assert_equal("first")
    ap(qkv_rows(p + 1, sum(more), hq, hkv, hd, 1.5), [a + b for a, b in zip(kv, new)], more)
    ap.c.assert_equal("second")
    assert int(ap.err.item()) == 0


@pytest.mark.parametrize("hq,hkv,hd,page_len", [(8, 2, 64, 16), (32, 8, 128, 64), (64, 8, 128, 32), (16, 1, 128, 128), (5, 5, 64, 32)])
def test_token_by_token(pdlib, hq, hkv, hd, page_len):
    """Decode steps of a ragged batch with padding rows; sizes grow, so that scales do as well."""
    steps = page_len + 5
    kv = [0, page_len - 3, 7, -1, 2 * page_len]
    ap = Appender(pdlib, hq, hkv, hd, 4 * page_len, page_len, [max(k, 0) + steps for k in kv], seed=hd)
    ap.c.fill([max(k, 0) for k in kv], np.random.default_rng(8))
    ap.c.upload()
    for i in range(steps):
        rows = gen.bf16_round(qkv_rows(100 + i, len(kv), hq, hkv, hd) * np.float32(1.15 ** i))
        ap(rows, [k + i if k >= 0 else -1 for k in kv], pad=0 if i % 2 else 16)
        if i % 16 == 0:
            ap.c.assert_equal(f"step {i}")
    ap.c.assert_equal("end")
    assert int(ap.err.item()) == 0


@pytest.mark.parametrize("runs", [False, True])
def test_extreme_values(pdlib, runs):
    """Zeros, infinities, NaN, the smallest and largest bf16 values, and a page whose scale grows by more than E4M3's range."""
    hq, hkv, hd, p = 4, 2, 64, 16
    ap = Appender(pdlib, hq, hkv, hd, 64, p, [40], seed=3)
    rows = qkv_rows(5, 20, hq, hkv, hd)
    v = rows[:, hq + hkv:]
    rows[0] = 0.0
    v[1], v[2, 0, 0], v[3, 1, 5], v[4, 0, 7] = 2.0 ** -130, np.inf, np.nan, -np.inf
    rows[5] = gen.bf16_round(rows[5] * np.float32(1e-30))
    rows[6] = gen.bf16_round(rows[6] * np.float32(1e30))
    v[7, 0, 3] = 3.3e38
    rows[8, hq, 1] = np.inf          # an infinite k reaches both members of its pair
    rows = gen.bf16_round(rows)
    if runs:
        ap(rows, [0], [20], with_q=False)
    else:
        for i in range(20):
            ap(rows[i:i + 1], [i], with_q=False)
            ap.c.assert_equal(f"token {i}")
    ap.c.assert_equal("end")


def test_rewriting_earlier_positions(pdlib):
    """Rejected tokens are overwritten; what lies behind the last appended token stays."""
    ap = Appender(pdlib, 8, 2, 64, 128, 16, [64, 64], seed=4)
    ap(qkv_rows(1, 60, 8, 2, 64), [0, 0], [40, 20])
    ap(qkv_rows(2, 10, 8, 2, 64, 1.5), [30, 15], [7, 3])
    ap.c.assert_equal("rewritten runs")
    ap(qkv_rows(3, 2, 8, 2, 64, 1.5), [32, 16])     # the first row of a page again, and a later one
    ap.c.assert_equal("rewritten tokens")


def test_rows_without_a_place_are_reported_and_left_out(pdlib):
    hq, hkv, hd, p = 8, 2, 64, 16
    for runs in (False, True):
        ap = Appender(pdlib, hq, hkv, hd, 44, p, [16, 16, 16], seed=5, extra_cols=0)   # table of one page each
        ap.c.table[1, 0] = ap.c.n_pages      # outside the pool
        ap.c.table[2, 0] = -1
        ap.c.upload()
        rows = qkv_rows(9, 3 if not runs else 9, hq, hkv, hd)
        q = ap(rows, [0, 0, 0], None if not runs else [3, 3, 3], oracle=False)
        assert int(ap.err.item()) == 2
        ap.err.zero_()
        n = 1 if not runs else 3
        rot = paged.rotate_f32(rows[:n, hq:hq + hkv], ap.tab[:n])
        paged.append(ap.c.k, ap.c.ks, ap.c.table[0], 0, rot)
        paged.append(ap.c.v, ap.c.vs, ap.c.table[0], 0, rows[:n, hq + hkv:])
        ap.c.assert_equal("bad pages")
        ref = paged.rotate(rows[:, :hq], np.tile(np.arange(n), 3), THETA)
        assert np.allclose(from_dev(q[:3 * n]).reshape(ref.shape), ref, atol=1e-2, rtol=BF16)   # q is there all the same
        # beyond the table, and beyond the rotation table
        ap(qkv_rows(10, 3 if not runs else 6, hq, hkv, hd), [16, 44, 2 ** 31 - 1], None if not runs else [2, 2, 2], oracle=False)
        ap.c.assert_equal("positions without a page")
        assert int(ap.err.item()) == 2


def test_other_stream_and_graph_replay(pdlib):
    """A captured decode step, replayed while kv_len advances on the device, equals the eager steps."""
    import torch
    hq, hkv, hd, p = 32, 8, 128, 32
    eager, graph = (Appender(pdlib, hq, hkv, hd, 128, p, [80, 50], seed=6) for _ in range(2))
    width = (hq + 2 * hkv) * hd
    rows = [qkv_rows(200 + i, 2, hq, hkv, hd, 1.0) for i in range(40)]
    kv0 = [30, 0]
    for i, r in enumerate(rows):
        eager(r, [k + i for k in kv0], oracle=False)
    dqkv, dkv, q = empty_bf16(2, width), i32_dev(kv0), empty_bf16(2, hq * hd)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pdlib.pd_paged_kv_append(graph.cfg, dqkv, width, q, graph.dtab, graph.c.struct, dkv, 2)
        dkv += 1
    for r in rows:
        dqkv.copy_(to_dev(r.reshape(2, width)))
        g.replay()
    torch.cuda.synchronize()
    for a, b in ((eager.c.dk, graph.c.dk), (eager.c.dv, graph.c.dv), (eager.c.dks.view(torch.int32), graph.c.dks.view(torch.int32)),
                 (eager.c.dvs.view(torch.int32), graph.c.dvs.view(torch.int32))):
        assert torch.equal(a, b)

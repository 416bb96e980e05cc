"""Device buffers of the GPU tests of the 4-bit paged KV cache, and the transform of q and k heads."""
import numpy as np

import pd_inputs as gen
from gpu_util import i32_dev, to_dev
from oracle import paged, paged4
from paged_util import F16, assert_within, attention_bound


class Cache4:
    """The same cache on the device and in numpy; rows that hold no token have NaN scales, unused table entries are -1."""

    def __init__(self, pd, hkv, hd, page_len, n_tokens, seed=0, spare=2, extra_cols=1, exps=True):
        rng = np.random.default_rng(seed)
        self.pd, self.hkv, self.hd, self.page_len = pd, hkv, hd, page_len
        counts = [max(1, -(-n // page_len)) for n in n_tokens]
        self.n_pages = sum(counts) + spare
        perm = rng.permutation(self.n_pages)
        self.width = max(counts) + extra_cols
        self.table = np.full((len(n_tokens), self.width), -1, np.int32)
        at = 0
        for i, c in enumerate(counts):
            self.table[i, :c] = perm[at:at + c]
            at += c
        rows = (self.n_pages, hkv, page_len)
        self.k, self.v = (rng.integers(0, 256, (*rows, hd // 2)).astype(np.uint8) for _ in range(2))
        self.ks, self.vs = (np.full((*rows, hd // 16), 0x7F, np.uint8) for _ in range(2))
        self.k_exp, self.v_exp = (rng.integers(-3, 4, hkv).astype(np.int32) if exps else None for _ in range(2))
        self.ke, self.ve = paged4.head_exp(self.k_exp, hkv), paged4.head_exp(self.v_exp, hkv)

    def fill(self, lengths, rng, spread=1.0):
        """Tokens 0 .. lengths[s] - 1 of every sequence, through the oracle; `spread`: log-normal size of the tokens."""
        for s, n in enumerate(lengths):
            for codes, scales, exp in ((self.k, self.ks, self.ke), (self.v, self.vs, self.ve)):
                x = rng.standard_normal((n, self.hkv, self.hd)) * np.exp(spread * rng.standard_normal((n, self.hkv, 1)))
                paged4.append(codes, scales, self.table[s], 0, gen.bf16_round(x * np.exp2(exp)[:, None]), exp)
        return self

    def upload(self):
        import torch
        self.dk, self.dv, self.dks, self.dvs = (torch.from_numpy(a.copy()).cuda() for a in (self.k, self.v, self.ks, self.vs))
        self.dt = i32_dev(self.table)
        self.dke, self.dve = (None if e is None else i32_dev(e) for e in (self.k_exp, self.v_exp))
        self.struct = self.pd.paged_kv4_cache_struct(self.dk, self.dv, self.dks, self.dvs, self.dt, self.n_pages, self.page_len,
                                                     len(self.table), self.width, k_exp=self.dke, v_exp=self.dve)
        return self

    def assert_equal(self, what=""):
        """Codes and scales on the device are the oracle's, bit for bit, rows without tokens included.  (Codes under a scale of
        NaN say nothing, and -0 is 0.)"""
        for name, d, ds, h, hs in (("k", self.dk, self.dks, self.k, self.ks), ("v", self.dv, self.dvs, self.v, self.vs)):
            got, got_s = d.cpu().numpy(), ds.cpu().numpy()
            np.testing.assert_array_equal(got_s, hs, err_msg=f"{what} {name} scales")
            a, b = paged4.values(got, got_s), paged4.values(h, hs)
            same = (a == b) | (np.isnan(a) & np.isnan(b))
            assert same.all(), (what, name, np.argwhere(~same)[:5], a[~same][:5], b[~same][:5])

    def kv(self, s, total):
        return (paged4.sequence(self.k, self.ks, self.table[s], total, self.ke),
                paged4.sequence(self.v, self.vs, self.table[s], total, self.ve))


class Transform:
    """A transform on the device and in numpy."""

    def __init__(self, pd, hd, rot, n_pos, pairs=False, gains=True, theta=1e4, seed=0, eps=1e-6, magnitude=1.0):
        import torch
        self.pairs, self.eps, self.rot = pairs, eps, rot
        self.q_gain, self.k_gain = (gen.normal_bf16(seed, 90 + i, (hd,), 0.2, 1.0) if gains else None for i in range(2))
        self.cs = paged4.table(paged4.frequencies(rot, theta), np.arange(n_pos), magnitude).astype(np.float32) if rot else None
        self.dev = [None if a is None else to_dev(a) for a in (self.q_gain, self.k_gain)]
        self.dtab = None if self.cs is None else torch.from_numpy(self.cs).cuda()
        self.struct = pd.qk_transform_struct(self.dtab, n_pos if rot else 0, rot, pd.ROPE_PAIRS if pairs else pd.ROPE_HALVES,
                                             q_gain=self.dev[0], k_gain=self.dev[1], eps=eps)

    def heads(self, x, gain, positions):
        return paged4.transform(x, gain, self.eps, None if self.cs is None else self.cs[np.asarray(positions)], self.pairs)

    def q(self, x, positions):
        return self.heads(x, self.q_gain, positions)

    def k(self, x, positions):
        return self.heads(x, self.k_gain, positions)


def transform_bound(y, mag):
    """How far a transformed value may be from the exact one: rounding to bf16, half a step, 2^-8 |y|; the fp32 arithmetic in front
    of it relative to the magnitude of its terms: sum of up to 128 squares in chains of 20 additions (20 * 2^-24, halved by the root), the
    reciprocal root (2^-22), eps (2^-24), four products and a sum (5 * 2^-24): below 2^-19."""
    return 2.0 ** -8 * np.abs(y) + 2.0 ** -19 * mag * (1 + 2.0 ** -8) + 1e-37


def check_attention(q, k, v, positions, got, what=""):
    """Rows q [n, Hq, hd] at `positions` over k, v [S, Hkv, hd] against the oracle.  To the bound of the 8-bit cache's kernels comes
    what small weights lose: p is kept as 2^7 p in f16, whose smallest step is 2^-24, so it is off by up to 2^-25 * 2^-7 = 2^-32 of the
    row's largest weight (at most 1) for every key.  (Codes of 0 leave such a weight alone in a feature.)"""
    o, spread, score = paged.attend(q, k, v, positions)
    seen = np.arange(len(v)) <= np.asarray(positions)[:, None]
    small = 2.0 ** -32 * np.einsum("ns,shd->nhd", seen, np.abs(v)).repeat(q.shape[1] // v.shape[1], axis=1)
    assert_within(got, o, attention_bound(o, spread, score, F16) + small * (1 + 2.0 ** -8), what)

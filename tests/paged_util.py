"""Device buffers and tolerances of the GPU tests of the 8-bit paged KV cache."""
import numpy as np

import pd_inputs as gen
from gpu_util import i32_dev
from oracle import paged

BF16 = 2.0 ** -8     # half a step of bf16, relative to the value
F16 = 2.0 ** -11


class Cache:
    """The same cache on the device and in numpy; rows that hold no token are 0x7F (NaN codes), unused table entries -1."""

    def __init__(self, pd, hkv, hd, page_len, n_tokens, seed=0, spare=2, fill=0x7F, extra_cols=1):
        import torch
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
        shape = (self.n_pages, hkv, page_len, hd)
        self.k, self.v = np.full(shape, fill, np.uint8), np.full(shape, fill, np.uint8)
        self.ks, self.vs = np.full(shape[:2], np.nan, np.float32), np.full(shape[:2], np.nan, np.float32)
        self.torch = torch

    def fill(self, lengths, rng, spread=1.0, pages=0.0):
        """Tokens 0 .. lengths[s] - 1 of every sequence, through the oracle; `spread`: log-normal size of the tokens, `pages`:
        of whole pages in octaves."""
        for s, n in enumerate(lengths):
            for i in range(0, n, self.page_len):
                m = min(self.page_len, n - i)
                for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
                    x = rng.standard_normal((m, self.hkv, self.hd)) * np.exp(spread * rng.standard_normal((m, self.hkv, 1)))
                    x *= 2.0 ** np.round(pages * rng.standard_normal())
                    paged.append(codes, scales, self.table[s], i, gen.bf16_round(x))

    def upload(self):
        t = self.torch
        self.dk, self.dv = t.from_numpy(self.k.copy()).cuda(), t.from_numpy(self.v.copy()).cuda()
        self.dks, self.dvs = t.from_numpy(self.ks.copy()).cuda(), t.from_numpy(self.vs.copy()).cuda()
        self.dt = i32_dev(self.table)
        self.struct = self.pd.paged_kv_cache_struct(self.dk, self.dv, self.dks, self.dvs, self.dt, self.n_pages, self.page_len,
                                                    len(self.table), self.width)
        return self

    def assert_equal(self, what=""):
        """Codes and scales on the device are the oracle's, bit for bit, rows without tokens included."""
        for name, d, h in (("k", self.dk, self.k), ("v", self.dv, self.v)):
            got = d.cpu().numpy()
            # (any NaN code stands for NaN)
            same = (got == h) | (((got & 0x7F) == 0x7F) & ((h & 0x7F) == 0x7F))
            assert same.all(), (what, name, np.argwhere(~same)[:5], got[~same][:5], h[~same][:5])
        for name, d, h in (("k scale", self.dks, self.ks), ("v scale", self.dvs, self.vs)):
            np.testing.assert_array_equal(d.cpu().numpy().view(np.uint32), h.view(np.uint32), err_msg=what + name)

    def kv(self, s, total):
        return (paged.sequence(self.k, self.ks, self.table[s], total), paged.sequence(self.v, self.vs, self.table[s], total))


def attention_bound(o, spread, score, p_step):
    """How far the kernels' output may be from the exact one on the same cached values.
    Final rounding to bf16: 2^-8 |o| (half a step).  Weights: p is rounded to the operand type, p_step relative, and its
    normalisation comes from the unrounded sum; an error ds of a score changes p by ds relative, once in p and once in the
    sum.  ds: q k is exact term by term, the fp32 sum of hd <= 128 terms errs by at most 128 * 2^-23 * sum |q k|, scaling and
    2^x by some 2^-21 of the score's size and of 1."""
    ds = (2.0 ** -16 + 2.0 ** -20) * score + 2.0 ** -19
    ds = np.broadcast_to(ds[..., None], o.shape)
    return BF16 * np.abs(o) + (p_step + 2.0 * ds + 2.0 ** -18) * spread * (1 + BF16) + 1e-37


def assert_within(got, want, bound, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape
    assert np.all(np.isfinite(got)), f"{what}: {np.count_nonzero(~np.isfinite(got))} non-finite values"
    over = np.abs(got - want) / bound
    assert over.max(initial=0.0) <= 1.0, f"{what}: {over.max():.3f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"

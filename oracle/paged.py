"""CPU oracle for the 8-bit paged KV cache and the fused residual addition, RMSNorm and FP8 quantisation.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA path.  numpy, float64 unless said otherwise.

  * cache: K (or V) codes uint8 [n_pages, Hkv, page_len, hd] in E4M3, one scale per (page, head); value = code * scale;
  * scale: the smallest power of two 2^e with max|value| <= 448 * 2^e over the tokens appended since the page's first row
    was last written, e in -117 .. 120 (an all-zero page: -117); a non-finite value is stored as NaN and has no part in it;
  * a page whose scale grows: code = E4M3(value / new scale) of the values it already holds;
  * rotation: (x_i, x_{i+h}) -> (x_i c - x_{i+h} s, x_{i+h} c + x_i s), h = hd / 2, cos and sin of pos * theta^(-2i/hd).

Pins: tests/test_oracle_paged.py.
"""
from __future__ import annotations

import numpy as np

from .fp8 import E4M3_MAX, e4m3_decode, e4m3_encode

MIN_EXP, MAX_EXP = -117, 120


def page_scale(amax) -> np.ndarray:
    """Smallest admissible power of two s with amax <= 448 s (float64 in, float64 out)."""
    amax = np.asarray(amax, dtype=np.float64)
    m, e = np.frexp(amax / E4M3_MAX)          # amax / 448 = m 2^e, m in [0.5, 1); exact: 448 = 7 * 2^6 divides up to rounding
    e = np.where(m > 0.5, e, e - 1)
    # the division may round across a power of two: decide by the product, which is exact
    e = np.where(amax > E4M3_MAX * np.exp2(e.astype(np.float64)), e + 1, e)
    e = np.where(amax <= E4M3_MAX * np.exp2(e.astype(np.float64) - 1), e - 1, e)
    e = np.where(amax > 0, np.clip(e, MIN_EXP, MAX_EXP), MIN_EXP)
    return np.exp2(e.astype(np.float64))


def append(codes, scales, page_ids, pos0: int, rows) -> None:
    """Stores rows [n, Hkv, hd] at positions pos0 .. of the sequence whose pages are page_ids, in place."""
    page_len = codes.shape[2]
    rows = np.asarray(rows, dtype=np.float64)
    n = rows.shape[0]
    i = 0
    while i < n:
        page, off = page_ids[(pos0 + i) // page_len], (pos0 + i) % page_len
        k = min(n - i, page_len - off)
        part = rows[i:i + k].transpose(1, 0, 2)                     # [Hkv, k, hd]
        mag = np.where(np.isfinite(part), np.abs(part), 0.0).max(axis=(1, 2))
        new = page_scale(mag)
        if off > 0:
            old = scales[page].astype(np.float64)
            new = np.maximum(new, old)
            for h in np.nonzero(new > old)[0]:
                codes[page, h, :off] = e4m3_encode(e4m3_decode(codes[page, h, :off]) * (old[h] / new[h]))
        part = np.where(np.isfinite(part), part, np.nan)
        codes[page, :, off:off + k] = e4m3_encode(part / new[:, None, None])
        scales[page] = new.astype(np.float32)
        i += k


def sequence(codes, scales, page_ids, total: int) -> np.ndarray:
    """[total, Hkv, hd] float64: the cached values of positions 0 .. total - 1."""
    page_len = codes.shape[2]
    ids = np.asarray(page_ids[:-(-total // page_len)], dtype=np.int64)
    v = e4m3_decode(codes[ids]) * scales[ids].astype(np.float64)[:, :, None, None]
    return v.transpose(0, 2, 1, 3).reshape(-1, codes.shape[1], codes.shape[3])[:total]


def rotate(x, positions, theta: float) -> np.ndarray:
    """x [n, H, hd] rotated to its positions, float64."""
    x = np.asarray(x, dtype=np.float64)
    half = x.shape[-1] // 2
    ang = np.asarray(positions, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    return np.concatenate([x[..., :half] * c - x[..., half:] * s, x[..., half:] * c + x[..., :half] * s], axis=-1)


def rotate_f32(x, table) -> np.ndarray:
    """The same in float32 with every product and sum rounded, from (cos, sin) rows table [n, hd / 2, 2]: decides codes."""
    x = np.asarray(x, dtype=np.float32)
    half = x.shape[-1] // 2
    c, s = table[:, None, :, 0].astype(np.float32), table[:, None, :, 1].astype(np.float32)
    lo, hi = x[..., :half], x[..., half:]
    with np.errstate(over="ignore", invalid="ignore"):
        return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def attend(q, keys, vals, positions):
    """Causal attention of q [n, Hq, hd] at `positions` over keys, vals [S, Hkv, hd].
    Returns (o, spread, score): o [n, Hq, hd]; spread = sum p |v|, what a relative error of the weights multiplies;
    score [n, Hq] = max over the visible keys of sum |q k| / sqrt(hd), what an error of the scores is relative to."""
    q, keys, vals = (np.asarray(a, dtype=np.float64) for a in (q, keys, vals))
    n, hq, hd = q.shape
    g = hq // keys.shape[1]
    o, spread, score = np.zeros_like(q), np.zeros_like(q), np.zeros((n, hq))
    for i in range(n):
        s = int(positions[i]) + 1
        if s <= 0:
            continue
        for h in range(hq):
            k, v = keys[:s, h // g], vals[:s, h // g]
            z = k @ q[i, h] / np.sqrt(hd)
            p = np.exp(z - z.max())
            p /= p.sum()
            o[i, h], spread[i, h] = p @ v, p @ np.abs(v)
            score[i, h] = (np.abs(k) @ np.abs(q[i, h])).max() / np.sqrt(hd)
    return o, spread, score


def add_rmsnorm(x, r, gain, eps: float, group: int):
    """(h, n, scale): h = x + r rounded to bf16 (float64 values; r may be None), n = RMSNorm(h) * gain, scale per row and
    `group` channels (0: per row)."""
    from pd_inputs import bf16_round
    h = np.asarray(x, dtype=np.float64)
    if r is not None:
        # (bf16_round works on float32: the float64 sum of two bf16 values is rounded to odd first, so that rounding twice
        # equals rounding once)
        s = h + np.asarray(r, dtype=np.float64)
        f = s.astype(np.float32)
        bits = f.view(np.uint32).copy()
        inexact = (f.astype(np.float64) != s) & np.isfinite(f)
        toward = np.where(np.abs(f.astype(np.float64)) > np.abs(s), bits - 1, bits)
        bits = np.where(inexact, toward | 1, bits).astype(np.uint32)
        h = bf16_round(bits.view(np.float32)).astype(np.float64)
    n = h / np.sqrt((h * h).mean(axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    b = n.reshape(n.shape[0], -1, group) if group else n[:, None]
    amax = np.abs(b).max(axis=-1)
    scale = np.where(amax > 0, amax / E4M3_MAX, 1.0)
    return h, n, scale if group else scale[:, 0]

"""CPU oracle for the 4-bit paged KV cache, scaled rotary positions and the norms of q and k heads.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA path.  numpy, float64.

  * cache: K (or V) codes uint8 [n_pages, Hkv, page_len, hd / 2], two E2M1 codes a byte (feature 2 i in bits 0-3), scales uint8
    [n_pages, Hkv, page_len, hd / 16] in E4M3, one power of two per head; value = code * scale * 2^exp;
  * of 16 neighbouring values x in units of 2^exp: scale = E4M3(max|x| / 6), code = E2M1(x / scale), nearest, ties to even, both
    saturating, decided by comparing x with exact borders; 16 values of which one is not finite have a scale of NaN; a code has the
    sign of a negative x, but under a scale of 0 all codes are 0;
  * transform of a head: x * rsqrt(mean x^2 + eps) * gain, then (a, b) -> (a c - b s, b c + a s) of the pairs of its first features.

Pins: tests/test_oracle_paged4.py.
"""
from __future__ import annotations

import numpy as np

from .fp8 import E4M3_NAN, e4m3_decode

GROUP = 16
MAX_EXP = 30
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _borders(grid):
    """Midpoints of an increasing grid, and whether a value on the midpoint goes up (to an even place)."""
    return (grid[1:] + grid[:-1]) / 2, np.arange(1, len(grid)) % 2 == 0


def _place(x, unit, grid):
    """Place in `grid` that is nearest to x / unit, unit > 0; x and unit * border are compared exactly."""
    mid, up = _borders(grid)
    edge = unit[..., None] * mid
    x = x[..., None]
    return ((x > edge) | ((x == edge) & up)).sum(axis=-1)


def head_exp(exp, hkv):
    return np.zeros(hkv, np.int64) if exp is None else np.clip(np.asarray(exp, np.int64), -MAX_EXP, MAX_EXP)


def quantise(x):
    """Codes uint8 [..., hd / 2] and scales uint8 [..., hd / 16] of x [..., hd], in units of 2^exp."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, GROUP)
    fine = np.isfinite(b).all(axis=-1)
    b = np.where(fine[..., None], b, 0.0)
    amax = np.abs(b).max(axis=-1)
    scales = np.empty(amax.shape, np.int64)
    e4m3 = e4m3_decode(np.arange(0x7F, dtype=np.uint8))  # 0 .. 448, increasing
    flat, out = amax.reshape(-1), scales.reshape(-1)
    for i in range(0, flat.size, 4096):
        out[i:i + 4096] = _place(flat[i:i + 4096], np.full(flat[i:i + 4096].shape, 6.0), e4m3)
    s = e4m3[scales]
    mag = np.where(s[..., None] > 0, _place(np.abs(b), np.where(s > 0, s, 1.0)[..., None] * np.ones(GROUP), E2M1), 0)
    codes = (mag | (((b < 0) & (s[..., None] > 0)) << 3)).astype(np.uint8).reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), np.where(fine, scales, E4M3_NAN).astype(np.uint8)


def values(codes, scales):
    """[..., hd] float64 of codes [..., hd / 2] and scales [..., hd / 16], in units of 2^exp."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    return (v.reshape(*scales.shape, GROUP) * e4m3_decode(scales)[..., None]).reshape(v.shape)


def append(codes, scales, page_ids, pos0: int, rows, exp) -> None:
    """Stores rows [n, Hkv, hd] at positions pos0 .. of the sequence whose pages are page_ids, in place; exp [Hkv]."""
    page_len = codes.shape[2]
    rows = np.asarray(rows, dtype=np.float64) * np.exp2(-exp.astype(np.float64))[:, None]
    for i in range(0, len(rows), 512):
        at = pos0 + np.arange(i, min(i + 512, len(rows)))
        page, off = np.asarray(page_ids)[at // page_len], at % page_len
        codes[page, :, off], scales[page, :, off] = quantise(rows[i:i + 512])


def sequence(codes, scales, page_ids, total: int, exp) -> np.ndarray:
    """[total, Hkv, hd] float64: the cached values of positions 0 .. total - 1."""
    page_len = codes.shape[2]
    ids = np.asarray(page_ids[:-(-total // page_len)], dtype=np.int64)
    v = values(codes[ids], scales[ids]) * np.exp2(exp.astype(np.float64))[:, None, None]
    return v.transpose(0, 2, 1, 3).reshape(-1, v.shape[1], v.shape[3])[:total]


def frequencies(rot: int, theta: float, scaling: str = "none", factor: float = 1.0, trained_len: int = 4096, low: float = 1.0,
                high: float = 32.0) -> np.ndarray:
    """Radians per position of the rot / 2 pairs."""
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "turns":
        w = np.clip((trained_len * f / (2 * np.pi) - low) / (high - low), 0, 1)
        return w * f + (1 - w) * f / factor
    if scaling == "index":
        def pair(turns):
            return rot * np.log(trained_len / (2 * np.pi * turns)) / (2 * np.log(theta))
        a, b = max(np.floor(pair(high)), 0), min(np.ceil(pair(low)), rot - 1)
        w = 1 - np.clip((i - a) / max(b - a, 1e-3), 0, 1)
        return w * f + (1 - w) * f / factor
    return f


def table(freq, positions, magnitude: float = 1.0) -> np.ndarray:
    """[n, rot / 2, 2] float64: magnitude times cos and sin."""
    a = np.asarray(positions, dtype=np.float64)[:, None] * freq
    return magnitude * np.stack([np.cos(a), np.sin(a)], axis=-1)


def transform(x, gain, eps: float, cs, pairs: bool):
    """x [n, H, hd] normalised (gain None: not) and rotated by the rows cs [n, rot / 2, 2] (None: not); and the sum of the
    magnitudes of the terms of each result, what an error of the arithmetic is relative to."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    y, mag = x.copy(), np.abs(x)
    if cs is not None:
        c, s = (np.asarray(cs[..., k], dtype=np.float64)[:, None] for k in (0, 1))
        rot = 2 * cs.shape[1]
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, b * c + a * s
        mag[..., first], mag[..., second] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, mag

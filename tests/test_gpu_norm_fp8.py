"""GPU: residual addition, RMSNorm and FP8 codes in one pass against the float64 oracle.

Tolerances: h is one rounding of an exact sum of two bf16 values (fp32 holds it to 2^-24, which can only turn a tie of the
bf16 rounding; the inputs below have exponents close enough for the fp32 sum to be exact).  The fp32 sum of squares of d terms
in at most 64 + 13 sequential additions errs by 77 * 2^-24 relative, its root by half of it, rsqrt and two products by 2^-21:
3e-6 in all for n and for the scale.  A code is half an E4M3 step off, 2^-4 relative or 2^-10 scales."""
import numpy as np
import pytest

import pd_inputs as gen
from gpu_util import empty_bf16, from_dev, to_dev
from oracle import fp8, paged
from paged_util import BF16

pytestmark = pytest.mark.gpu
REL = 3e-6


def run(pd, x, r, g, group, eps=1e-6, ldx=0, ldr=0, want_sum=True, want_norm=True, want_codes=True):
    import torch
    rows, d = x.shape
    pad = lambda a, ld: to_dev(np.concatenate([a, np.full((rows, ld - d), np.nan, np.float32)], 1)) if ld else to_dev(a)  # noqa: E731
    dx, dr = pad(x, ldx), None if r is None else pad(r, ldr)
    h = empty_bf16(rows + 1, d) if want_sum else None
    n = empty_bf16(rows + 1, d) if want_norm else None
    codes = torch.full((rows + 1, d), 0xAB, dtype=torch.uint8, device="cuda") if want_codes else None
    scales = torch.full((rows + 1, d // 128 if group else 1), -1.0, device="cuda") if want_codes else None
    pd.pd_add_rmsnorm_fp8(dx, rows, d, to_dev(g), codes, scales, residual=dr, sum_out=h, norm_out=n, eps=eps, group=group, ldx=ldx,
                          ldr=ldr)
    torch.cuda.synchronize()
    if want_codes:   # the row behind the last one is as it was
        assert (codes[rows] == 0xAB).all() and (scales[rows] == -1).all()
    for t in (h, n):
        assert t is None or not t[rows].any()
    return [None if t is None else t[:rows] for t in (h, n, codes, scales)]


def check(x, r, g, group, out, eps=1e-6):
    rows, d = x.shape
    h, n, codes, scales = out
    ho, no, so = paged.add_rmsnorm(x, r, g, eps, group)
    so = so.reshape(rows, -1)
    if h is not None:
        np.testing.assert_array_equal(from_dev(h), ho.astype(np.float32))
    if n is not None:
        assert np.all(np.abs(from_dev(n) - no) <= (BF16 + REL) * np.abs(no) + 1e-40)
    if codes is not None:
        s = scales.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(s - so) <= REL * so)
        wide = np.repeat(s, d // s.shape[1], axis=1)
        got = fp8.e4m3_decode(codes.cpu().numpy()) * wide
        assert np.all(np.abs(got - no) <= (2.0 ** -4 + REL) * np.abs(no) + (2.0 ** -10 + REL) * wide)


@pytest.mark.parametrize("rows,d,group", [(1, 128, 128), (1, 16, 0), (3, 384, 128), (7, 1040, 0), (5, 2048, 128), (130, 4096, 128),
                                          (33, 4112, 0), (9, 8192, 0), (700, 8192, 128), (4, 16384, 128), (2, 16384, 0), (2, 16256, 128)])
@pytest.mark.parametrize("residual", [True, False])
def test_matches_oracle(pdlib, rows, d, group, residual):
    x = gen.normal_bf16(61, 1, (rows, d), 1.0, sub=d)
    r = gen.normal_bf16(61, 2, (rows, d), 2.0, sub=d) if residual else None
    g = gen.normal_bf16(61, 3, (d,), 0.3, 1.0)
    check(x, r, g, group, run(pdlib, x, r, g, group))


@pytest.mark.parametrize("group", [0, 128])
def test_zero_rows_zero_blocks_and_small_values(pdlib, group):
    x = gen.normal_bf16(62, 1, (6, 512), 1.0)
    x[0] = 0.0
    x[1, 128:256] = 0.0
    x[2] = gen.bf16_round(x[2] * np.float32(1e-20))     # below eps: n is tiny
    x[3] = gen.bf16_round(x[3] * np.float32(1e15))      # squares near 1e33
    x[4, 1:] = 0.0                                      # one element
    g = gen.normal_bf16(62, 3, (512,), 0.3, 1.0)
    out = run(pdlib, x, None, g, group)
    check(x, None, g, group, out)
    # (a zero times a negative gain is -0, code 0x80)
    assert (out[3].cpu().numpy()[0] == 1.0).all() and not (out[2][0] & 0x7F).any()


def test_strides_optional_outputs_and_in_place(pdlib):
    import torch
    x, r = gen.normal_bf16(63, 1, (37, 768), 1.0), gen.normal_bf16(63, 2, (37, 768), 1.0)
    g = gen.normal_bf16(63, 3, (768,), 0.3, 1.0)
    full = run(pdlib, x, r, g, 128)
    check(x, r, g, 128, run(pdlib, x, r, g, 128, ldx=776, ldr=1024))
    check(x, r, g, 128, run(pdlib, x, r, g, 128, want_sum=False, want_norm=False))
    check(x, r, g, 128, run(pdlib, x, r, g, 128, want_codes=False))
    # the residual stream updated in place, twice the same result as out of place
    for alias in ("x", "residual"):
        dx, dr = to_dev(x), to_dev(r)
        tgt = dx if alias == "x" else dr
        codes, scales = torch.zeros((37, 768), dtype=torch.uint8, device="cuda"), torch.zeros((37, 6), device="cuda")
        pdlib.pd_add_rmsnorm_fp8(dx, 37, 768, to_dev(g), codes, scales, residual=dr, sum_out=tgt)
        torch.cuda.synchronize()
        assert torch.equal(tgt, full[0]) and torch.equal(codes, full[2]) and torch.equal(scales, full[3])


def test_non_finite_rows_stay_visible_and_apart(pdlib):
    x = gen.normal_bf16(64, 1, (4, 256), 1.0)
    clean = run(pdlib, x, None, gen.normal_bf16(64, 3, (256,), 0.3, 1.0), 128)
    bad = x.copy()
    bad[1, 5], bad[2, 200] = np.nan, np.inf
    out = run(pdlib, bad, None, gen.normal_bf16(64, 3, (256,), 0.3, 1.0), 128)
    for a, b in zip(out, clean):
        assert bool((a[[0, 3]] == b[[0, 3]]).all())
    n, codes = from_dev(out[1]), out[2].cpu().numpy()
    assert np.isnan(n[1]).all() and np.isnan(n[2, 200])
    assert ((codes[1] & 0x7F) == 0x7F).all() and (codes[2, 200] & 0x7F) == 0x7F


def test_codes_feed_the_gemms(pdlib):
    """The two layouts are what the per-row and the block-wise GEMM take."""
    import torch
    m, d, n = 40, 512, 256
    x, r = gen.normal_bf16(65, 1, (m, d), 1.0), gen.normal_bf16(65, 2, (m, d), 1.0)
    g, w = gen.normal_bf16(65, 3, (d,), 0.1, 1.0), gen.normal_bf16(65, 4, (n, d), 0.05)
    _, no, _ = paged.add_rmsnorm(x, r, g, 1e-6, 128)
    ref = no @ w.astype(np.float64).T
    for group in (0, 128):
        _, _, codes, scales = run(pdlib, x, r, g, group)
        wq = torch.zeros((n, d), dtype=torch.uint8, device="cuda")
        c = empty_bf16(m, n)
        if group:
            ws = torch.zeros((n // 128, d // 128), device="cuda")
            pdlib.pd_quantize_fp8_blocks(to_dev(w), n, d, wq, ws)
            pdlib.pd_gemm_fp8_blockwise(codes, scales, wq, ws, c, m, n, d)
        else:
            ws = torch.zeros(n, device="cuda")
            pdlib.pd_quantize_fp8_rows(to_dev(w), n, d, wq, ws)
            pdlib.pd_gemm_fp8(codes, scales, wq, ws, c, m, n, d)
        torch.cuda.synchronize()
        # every factor is half an E4M3 step off at most: 2 * 2^-4 of sum |n w|, and the rounding of the result
        bound = (2.0 ** -3 + 2.0 ** -8) * (np.abs(no) @ np.abs(w.astype(np.float64)).T) + BF16 * np.abs(ref)
        assert np.all(np.abs(from_dev(c) - ref) <= bound)
        assert np.linalg.norm(from_dev(c) - ref) <= 0.06 * np.linalg.norm(ref)

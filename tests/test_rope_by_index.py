"""Rotary frequencies blended by pair index where the ramp ends behind the last pair: the slowest pair turns more often within the
trained length than frequencies that are divided whole, so it keeps part of its own."""
import math

import numpy as np
import pytest

from oracle import paged4

# rot_dim, theta, trained_len, factor, low, high
CASES = [(64, 1e4, 131072, 8.0, 1.0, 32.0), (16, 1e4, 32768, 8.0, 1.0, 32.0), (128, 1e4, 1 << 20, 16.0, 1.0, 4.0),
         (64, 10.0, 4096, 4.0, 1.0, 32.0), (32, 1e4, 4096, 8.0, 1.0, 32.0)]


def by_index(rot, theta, trained, factor, low, high):
    """Pair by pair: I(n) = rot ln(trained / (2 pi n)) / (2 ln theta) is the pair that turns n times; frequencies in front of pair
    floor(I(high)) are kept, those behind pair ceil(I(low)) divided by the factor, linearly in between; the first bound is at
    least 0, the second at most rot - 1."""
    at = [rot * math.log(trained / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (low, high)]
    end, begin = min(math.ceil(at[0]), rot - 1), max(math.floor(at[1]), 0)
    out = []
    for i in range(rot // 2):
        f = theta ** (-2 * i / rot)
        ramp = min(max((i - begin) / max(end - begin, 1e-3), 0.0), 1.0)
        out.append(f * (1 - ramp) + f / factor * ramp)
    return np.array(out)


@pytest.mark.parametrize("case", CASES)
def test_oracle(case):
    rot, theta, trained, factor, low, high = case
    f = paged4.frequencies(rot, theta, "index", factor, trained, low, high)
    np.testing.assert_allclose(f, by_index(*case), rtol=1e-13)
    plain = theta ** (-2 * (rot // 2 - 1) / rot)
    turns = trained * plain / (2 * math.pi)
    assert (f[-1] > plain / factor * (1 + 1e-9)) == (turns > low)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_table(pdlib, case):
    import torch
    rot, theta, trained, factor, low, high = case
    n = 300
    t = torch.empty((n, rot // 2, 2), device="cuda")
    pdlib.pd_rope_table_scaled(pdlib.RopeConfig(rot, theta, pdlib.ROPE_SCALE_INDEX, factor, trained, low, high), 0, n, t)
    angle = np.arange(n)[:, None] * by_index(*case)
    want = np.stack([np.cos(angle), np.sin(angle)], axis=-1)
    # one rounding to fp32, and the angle in double
    assert (np.abs(t.cpu().numpy() - want) <= 2.0 ** -24 + np.arange(n)[:, None, None] * 2.0 ** -50).all()

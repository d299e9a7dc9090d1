"""How far the fp32 errors of the 4-bit weights' scale search may be off, in numpy.

The search takes the nearest value of w / alpha from fl32(w * r), r the reciprocal of alpha within one
unit in the last place, and compares the sums of squared errors in fp32; sums closer than a window
go to fp64.  The window has to cover a square that is too large because the product fell on the
wrong side of a cell bound, and the roundings of both sums.  The first is found here by brute force:
every scale's significand (bf16: 128), every bound, every fp32 weight near it, every such r."""
import os
import re

import numpy as np

from conftest import ROOT

LEVELS = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
SUMS = 11 * 2.0 ** -24          # two roundings of a square, nine additions on its way


def windows():
    with open(os.path.join(ROOT, "paper_2109_03513_amd", "csrc", "w4.hip")) as f:
        m = re.search(r"kNear = sizeof\(T\) == 4 \? (0x1p-\d+)f : (0x1p-\d+)f;", f.read())
    return float.fromhex(m.group(1)), float.fromhex(m.group(2))


def nearest(x):
    """Nearest E2M1 value of fp32 x, ties to even significands, as the conversion rounds."""
    step = np.where(x >= 4, 2.0, np.where(x >= 2, 1.0, 0.5))
    return np.minimum(np.rint(x.astype(np.float64) / step) * step, 6.0)


def excess(weights_of):
    """The largest (square taken / least square) - 1 over weights_of(bound) for all scales."""
    worst = 0.0
    for man in range(128):
        alpha = 1 + man / 128
        r0 = np.float32(1 / alpha)
        for r in (np.nextafter(r0, np.float32(0)), r0, np.nextafter(r0, np.float32(4))):
            if abs(float(r) * alpha - 1) > 2.0 ** -23:
                continue
            for i in range(7):
                lo, hi = LEVELS[i] * alpha, LEVELS[i + 1] * alpha
                w = weights_of((lo + hi) / 2)
                q = nearest(w * r) * alpha
                w = w.astype(np.float64)
                least = np.minimum((w - lo) ** 2, (w - hi) ** 2)
                worst = max(worst, float(((w - q) ** 2 / least).max()) - 1)
    return worst


def test_window_of_32_bit_weights():
    def close(bound):
        bits = np.float32(bound).view(np.uint32).astype(np.int64) + np.arange(-64, 65)
        return bits.astype(np.uint32).view(np.float32)

    side = excess(close)
    assert 1e-6 < side < 28 * 1.5 * 2.0 ** -23 * 1.001       # the bound that the kernel's comment gives
    assert side + 2 * SUMS < windows()[0]


def test_window_of_16_bit_weights():
    def close(digits):
        def of(bound):
            e = np.floor(np.log2(bound))
            unit = 2.0 ** (e - digits + 1)
            return (np.rint(bound / unit) * unit + unit * np.arange(-8, 9)).astype(np.float32)
        return of

    for digits in (8, 11):                                   # bf16, fp16
        assert excess(close(digits)) == 0
    assert 2 * SUMS < windows()[1]

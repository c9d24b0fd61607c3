"""Checks shared by the tests of the 4-bit pool and of the block weights.

Tolerance of an attention output (per value): the weights are rounded to bf16 before the
value product (half a step, 2^-8 of each weight), so the sum is off by at most 2^-8 of
S = sum w |v|; the result is rounded once (2^-8 of it). A score is a float32 sum of D
products of magnitude |q||k| sm: off by at most (D + 2) 2^-24 sum |q k| sm, below 5e-5
for the inputs here, as is the exponential, so weights and lse are off by 2 * 5e-5
relative, 1e-4 S in the output. With 1% on top of the two roundings for their product:
    |out - ref| <= 1.01 * 2^-8 (S + |ref|) + 2e-4 S + 1e-33,    |lse - ref| <= 2e-4,
(weights below 2^-126 of a row's largest are zero in float32: n 2^-126 |v|, with up to
10^4 keys and |v| up to 8 below 1e-33)
and a block's weight, a sum of such weights, is off by at most 3e-4 of itself.
"""
from __future__ import annotations

import numpy as np

from tests.gpu_helpers import f64


def check_out(out, lse, ref, ref_lse, size, name, wide=1.0):
    """wide: how much larger the scores are than sm = 1 / sqrt(D) makes them."""
    out, lse = f64(out), f64(lse)
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(out), nan), name
    err = np.abs(out - ref)[~nan]
    tol = (1.01 * 2.0 ** -8 * (size + np.abs(ref)) + 2e-4 * wide * size + 1e-33)[~nan]
    assert (err <= tol).all(), "%s: off by %.3g where %.3g is allowed" % (
        name, (err - tol).max(), tol[(err - tol).argmax()])
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse)), name
    assert np.array_equal(np.isnan(lse), np.isnan(ref_lse)), name
    fine = np.isfinite(ref_lse)
    assert (np.abs(lse[fine] - ref_lse[fine]) <= 2e-4 * wide).all(), name


def check_weight(got, ref, name):
    assert (np.abs(got.cpu().numpy() - ref) <= 3e-4 * np.abs(ref) + 1e-12).all(), name

"""Cases over a 4-bit pool of random codes and scales: every byte pattern is a value, so a
large pool needs no rounding (which the float64 definition does group by group)."""
from __future__ import annotations

from unittest import mock

import numpy as np

from oracle import kv4
from tests.test_gpu_kv4 import Case


def random_tiles(k, v):
    """Tiles for blocks [nb][Hkv][16][D]: any codes, scales 2^-3 to 2^-1 (magnitudes up to 3)."""
    nb, hkv, _, D = k.shape
    rng = np.random.default_rng(nb * 1000 + hkv * 10 + D)
    tiles = rng.integers(0, 256, (nb, hkv, 17 * D), dtype=np.uint8)
    tiles[..., 16 * D:] = rng.integers(124, 127, (nb, hkv, D), dtype=np.uint8)
    return tiles


def quick_case(*args, **kwargs):
    """A Case whose cached blocks are random tiles."""
    with mock.patch.object(kv4, "pack", random_tiles):
        return Case(*args, **kwargs)


def check_counts(out, lse, ref, ref_lse, name):
    """Results at sm_scale = 0, where every visible key weighs 1: one key more or less shows
    in lse. The sums are of numbers below 2^20 with at most 4 bits behind the point (codes at
    scales of 2^-3 and above, weights of 1), so float32 holds them exactly, and so is what
    joins partitions (2^0). lse then has the error of a float32 logarithm and its product,
    each below 2^-21 of at most 2^4; an output that of a quotient, 2^-22 of it, and of its
    rounding, 2^-8 of it at most."""
    out = out.float().cpu().numpy().astype(np.float64)
    lse = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse)), name
    fine = np.isfinite(ref_lse)
    assert (np.abs(lse[fine] - ref_lse[fine]) <= 2.0 ** -16).all(), name
    assert (np.abs(out - ref) <= 2.0 ** -8 * (1 + 2.0 ** -10) * np.abs(ref) + 1e-12).all(), name

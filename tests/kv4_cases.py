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

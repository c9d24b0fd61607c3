"""Averages of values that agree: attention over the 4-bit pool divides by the weights that it
multiplied by, so an output of equal values is that value, whatever the weights.

The value product and the sum of the rounded weights are float32 sums of the same n positive
terms: off by less than (n + 4) 2^-24 of themselves each, as are the joins of partitions.
With n <= 9000 keys that is below 2^-9, half a step of bf16 (1/256 at most below the next
value), so the rounded output is exactly the value.
"""
from __future__ import annotations

import numpy as np
import pytest

import paper_2608_15241_amd as lk
from oracle import kv4
from tests.gpu_helpers import dev, f64, say
from tests.kv4_cases import quick_case
from tests.pool_helpers import bits_to_f64, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
BS = 16


def _case(seed, ctx, new, hq, hkv, D, peak):
    """Equal values at every token (another for each head and dim), scores `peak` times the
    usual ones: rows that one key dominates, and rows where the running maximum is behind."""
    c = quick_case(seed, ctx, hq, hkv, D, new=new, stale=0.2)
    row = c.rng.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (hkv, D)) * c.rng.choice(
        [-1.0, 1.0], (hkv, D)) * 2.0 ** np.repeat(c.rng.integers(-9, 9, (hkv, D // 32)), 32, 1)
    row[:, ::32] = 6.0 * 2.0 ** np.ceil(np.log2(np.abs(row).reshape(hkv, -1, 32).max(-1) / 6))
    one = kv4.pack(*np.broadcast_to(row[None, None, :, None], (2, 1, hkv, BS, D)))
    for part in (slice(8 * D, 16 * D), slice(16 * D + D // 2, 17 * D)):
        c.tiles[..., part] = one[..., part]
    assert (kv4.unpack(c.tiles)[1] == row[None, :, None]).all()
    c.vn = np.broadcast_to(f32_to_bf16_bits(row)[None], c.vn.shape).copy()
    c.q = f32_to_bf16_bits(bits_to_f64(c.q) * peak)
    return c, row


def _check(out, lse, row, group):
    out, lse = f64(out), lse.cpu().numpy()
    want = np.repeat(row, group, 0)[None]
    seen = np.isfinite(lse)[..., None]
    assert seen.any()
    assert np.array_equal(out, np.where(seen, want, 0.0))


# decode with four, two and one waves a partition; 16 rows and 128 rows in prefill
@pytest.mark.parametrize("peak", [1.0, 6.0, 30.0])
@pytest.mark.parametrize("ctx,hq,hkv,D", [([9000, 300], 8, 1, 64), ([700, 64, 1500], 8, 8, 128),
                                          ([300] * 40, 32, 8, 128), ([130] * 300, 8, 8, 64)])
def test_decode(ctx, hq, hkv, D, peak):
    c, row = _case(len(ctx), ctx, None, hq, hkv, D, peak)
    q, pool, meta, new = c.gpu()
    say("equal values", ctx[:3], hq, hkv, D, peak)
    out, lse = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, **new)
    _check(out, lse, row, hq // hkv)


@pytest.mark.parametrize("peak", [1.0, 6.0, 30.0])
@pytest.mark.parametrize("prefix,chunk,hq,hkv,D,wide", [
    ([2000, 5, 90], [3, 7, 1], 8, 2, 128, False), ([700, 20], [40, 90], 4, 4, 64, False),
    ([900, 0, 33], [150, 40, 64], 8, 2, 128, True), ([100, 60], [300, 70], 4, 4, 64, True)])
def test_prefill(prefix, chunk, hq, hkv, D, wide, peak):
    c, row = _case(len(prefix) + D, np.array(prefix) + np.array(chunk), chunk, hq, hkv, D, peak)
    if wide:
        c.widen()
    q, pool, meta, new = c.gpu()
    say("equal values", prefix, chunk, hq, hkv, D, wide, peak)
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    _check(out, lse, row, hq // hkv)

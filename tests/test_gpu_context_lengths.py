"""Lengths at the end of int32, which no table holds: the context counts as its whole table.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_15241_amd as lk
from tests.gpu_helpers import dev, dev_u16, say
from tests.kv4_helpers import check_out, check_weight
from tests.pool_helpers import dense_to_pool, f32_to_bf16_bits
from tests.test_gpu_kv4 import Case
from oracle import kv4

pytestmark = pytest.mark.gpu
BS = 16
LONG = [2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16]


def _case(width, hq, hkv, D):
    c = Case(width, [BS * width] * 4, hq, hkv, D, stale=0.2)
    short = BS * width - 5
    c.ctx = np.array(LONG + [short], np.int32)
    return c


@pytest.mark.parametrize("width,hq,hkv,D", [(3, 4, 2, 64), (90, 8, 2, 128), (600, 2, 2, 64)])
def test_decode_of_the_4_bit_pool(width, hq, hkv, D):
    c = _case(width, hq, hkv, D)
    q, pool, meta, new = c.gpu()
    want = c.appended()  # the long ones have no block for their new token
    ref, ref_lse, size, w = c.ref(want)
    say("lengths", width, hq, hkv, D)
    out, lse, wo = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, **new,
                                                  weight_out=torch.empty(c.table.shape,
                                                                         device="cuda"))
    check_out(out, lse, ref, ref_lse, size, "out")
    check_weight(wo, w, "weights")
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("width,hq,hkv,D", [(3, 4, 2, 64), (90, 8, 2, 128), (600, 2, 2, 64)])
def test_decode_and_version_check_of_the_bf16_pool(width, hq, hkv, D):
    c = _case(width, hq, hkv, D)
    q, _, meta, _ = c.gpu()
    K, V = kv4.unpack(c.tiles)
    ref, ref_lse, size, w = c.ref(c.tiles)
    K, V = (dev_u16(t).view(c.num, hkv, BS * D)
            for t in dense_to_pool(f32_to_bf16_bits(K), f32_to_bf16_bits(V)))
    say("lengths", width, hq, hkv, D)
    out, lse = lk.local_paged_attn_decode(q, K, V, *meta, c.sm, Hkv=hkv)
    check_out(out, lse, ref, ref_lse, size, "out")
    out, lse, wo = lk.local_paged_attn_decode_weighted(q, K, V, *meta, c.sm, Hkv=hkv)
    check_out(out, lse, ref, ref_lse, size, "out")
    check_weight(wo, w, "weights")
    table = c.table
    inside = (table >= 0) & (table < c.num)
    stale = ~inside | (c.tags[np.where(inside, table, 0)] != c.version[:, None])
    pairs, n, valid = lk.local_block_version_check(*meta, cap=stale.size)
    assert int(n) == stale.sum()
    assert np.array_equal(pairs.cpu().numpy()[:int(n)], np.argwhere(stale))
    live = np.full(table.shape, BS)
    live[3, -1] = BS - 5
    assert valid.cpu().numpy().tolist() == np.where(stale, 0, live).sum(1).tolist()

"""The 4-bit pool on the GPU: conversion bit by bit, decode and prefill attention against
float64 (tolerances: kv4_helpers.py).
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2608_15241_amd as lk
from oracle import kv4
from tests.gpu_helpers import dev, dev_u16, f64, say
from tests.kv4_helpers import check_out, check_weight
from tests.pool_helpers import bits_to_f64, dense_to_pool, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
BS = 16


class Case:
    """Requests over one 4-bit pool: random values, table and tags."""

    def __init__(self, seed, ctx, hq, hkv, D, new=None, stale=0.0, spare=3, width=None,
                 all_stale=()):
        rng = np.random.default_rng(seed)
        self.rng, self.hq, self.hkv, self.D = rng, hq, hkv, D
        self.ctx = np.asarray(ctx, np.int32)
        self.new = np.ones(len(ctx), np.int64) if new is None else np.asarray(new)
        nb = [(max(int(c), 0) + BS - 1) // BS for c in ctx]
        self.num = max(1, sum(nb)) + spare
        k, v = (bits_to_f64(f32_to_bf16_bits(rng.standard_normal((self.num, hkv, BS, D))))
                for _ in range(2))
        self.tiles = kv4.pack(k, v)
        ids = rng.permutation(self.num)
        width = max(nb + [1]) if width is None else width
        # entries past the context's end are never read: garbage
        self.table = rng.integers(-2 ** 31, 2 ** 31 - 1, (len(ctx), width)).astype(np.int32)
        self.version = rng.integers(1, 50, len(ctx)).astype(np.int32)
        self.tags = np.full(self.num, -7, np.int32)
        at = 0
        for b, n in enumerate(nb):
            n_t = min(n, width)
            self.table[b, :n_t] = ids[at:at + n_t]
            self.tags[ids[at:at + n]] = self.version[b]
            for j in range(n_t):
                last = j >= (int(ctx[b]) - int(self.new[b])) // BS
                if b in all_stale or (not last and rng.random() < stale):
                    if rng.random() < 0.3:
                        self.table[b, j] = rng.choice([-1, self.num, 2 ** 30])
                    else:
                        self.tags[self.table[b, j]] += 1
            at += n
        self.spare = ids[at:]
        T = int(self.new.sum())
        self.starts = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.q = f32_to_bf16_bits(rng.standard_normal((T, hq, D)))
        self.kn, self.vn = (f32_to_bf16_bits(rng.standard_normal((T, hkv, D))) for _ in range(2))
        self.sm = 1.0 / math.sqrt(D)

    def widen(self):
        """A table as for the longest contexts, of garbage past these: with more than 32 rows
        a request on average, attention then goes by 128 rows (the rule takes a table's width
        for its contexts)."""
        more = np.full((len(self.ctx), 17000), -3, np.int32)
        more[:, :self.table.shape[1]] = self.table
        if self.table.shape[1] < ((self.ctx + BS - 1) // BS).max():
            raise ValueError("the contexts would no longer end with the table")
        self.table = more

    def gpu(self, append=True):
        self.pool = torch.from_numpy(self.tiles.copy()).to("cuda")
        self.meta = [dev(x) for x in (self.table, self.ctx, self.tags, self.version)]
        new = dict(k_new=dev_u16(self.kn), v_new=dev_u16(self.vn)) if append else {}
        return dev_u16(self.q), self.pool, self.meta, new

    def appended(self):
        """The tiles with the new tokens written, by the definition."""
        t = self.tiles.copy()
        for b, (L, n) in enumerate(zip(self.ctx, self.new)):
            for i in range(int(n)):
                pos, row = int(L) - int(n) + i, int(self.starts[b]) + i
                if pos < 0 or pos // BS >= self.table.shape[1]:
                    continue
                p = self.table[b, pos // BS]
                if 0 <= p < self.num:
                    kv4.write(t, bits_to_f64(self.kn[row:row + 1]),
                              bits_to_f64(self.vn[row:row + 1]), [p], [pos % BS])
        return t

    def ref(self, tiles):
        K, V = kv4.unpack(tiles)
        return kv4.attention(bits_to_f64(self.q), self.starts, self.ctx, self.table, self.tags,
                             self.version, K, V, self.sm)


def special_tokens(rng, hkv, D):
    """Two blocks of values at the edges of the format."""
    x = rng.standard_normal((2, hkv, BS, D)).astype(np.float32)
    x[0, 0, 0] = 0.0
    x[0, 0, 1] = -0.0
    x[0, 0, 2, :32] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5,
                       -5, -6, 0.2490234375, 0.2509765625, 4.96875, 5.03125] + [0.0] * 12
    x[0, 0, 3, 0] = 6.03125
    x[0, 0, 4, 3] = 3.3895e38       # the largest group
    x[0, 0, 5, 3] = 1e-38
    x[0, 0, 6] = 2.0 ** -133        # the smallest bf16
    x[0, 0, 7, 1:3] = [1.6e38, -3e38]
    x[0, 0, 8, 5] = np.inf
    x[0, 0, 9, D - 1] = -np.inf
    x[0, 0, 10, 31] = np.nan
    x[0, 0, 11] *= 1e-30
    x[0, 0, 12] *= 1e30
    return f32_to_bf16_bits(x)


def to_pools(bits):
    k, v = dense_to_pool(bits, bits[:, :, ::-1])
    nb, hkv, _, D = bits.shape
    return (dev_u16(k).view(nb, hkv, BS * D), dev_u16(v).view(nb, hkv, BS * D),
            bits_to_f64(bits), bits_to_f64(bits[:, :, ::-1]))


@pytest.mark.parametrize("nb,hkv,D", [(1, 1, 64), (1, 1, 128), (7, 3, 64), (5, 8, 128),
                                      (33, 2, 128)])
def test_pool_conversion_is_exact(nb, hkv, D):
    rng = np.random.default_rng(nb * 1000 + D)
    bits = f32_to_bf16_bits(rng.standard_normal((nb, hkv, BS, D)) * 10.0 ** rng.uniform(-3, 3))
    bits[-1] = special_tokens(rng, hkv, D)[0]
    K, V, k, v = to_pools(bits)
    got = lk.local_kv4_pool_import(K, V)
    want = kv4.pack(k, v)
    assert np.array_equal(got.cpu().numpy(), want)
    K2, V2 = lk.local_kv4_pool_export(got)
    for x, y in zip((K2, V2), dense_to_pool(*(f32_to_bf16_bits(t) for t in kv4.unpack(want)))):
        x, y = f64(x).ravel(), bits_to_f64(y)
        assert np.array_equal(np.isnan(x), np.isnan(y))
        assert np.array_equal(x[~np.isnan(x)], y[~np.isnan(y)])


@pytest.mark.parametrize("D", [64, 128])
def test_pool_conversion_of_listed_blocks(D):
    rng = np.random.default_rng(D)
    bits = f32_to_bf16_bits(rng.standard_normal((9, 2, BS, D)))
    K, V, k, v = to_pools(bits)
    ids = [4, 0, 4, -1, 9, 7, 2 ** 31 - 1, -2 ** 31]
    want = np.full((9, 2, 17 * D), 0xa5, np.uint8)
    full = kv4.pack(k, v)
    for p in (4, 0, 7):
        want[p] = full[p]
    pool = torch.full((9, 2, 17 * D), 0xa5, dtype=torch.uint8, device="cuda")
    assert lk.local_kv4_pool_import(K, V, pool, block_ids=dev(np.array(ids))) is pool
    assert np.array_equal(pool.cpu().numpy(), want)
    K2, V2 = lk.local_kv4_pool_export(torch.from_numpy(full).to("cuda"),
                                      block_ids=dev(np.array(ids)))
    untouched = [1, 2, 3, 5, 6, 8]
    assert not K2[untouched].any() and not V2[untouched].any()
    K3, V3 = lk.local_kv4_pool_export(torch.from_numpy(full).to("cuda"))
    assert torch.equal(K2[[0, 4, 7]], K3[[0, 4, 7]]) and torch.equal(V2[[0, 4, 7]], V3[[0, 4, 7]])
    none = dev(np.array([], np.int32))
    assert not lk.local_kv4_pool_import(K, V, block_ids=none).any()


DECODE = [
    # (contexts, Hq, Hkv, D, options)
    ([1], 1, 1, 64, {}),
    ([1, 16, 17, 32, 33], 4, 4, 128, {}),
    ([5, 700, 64], 9, 3, 64, dict(stale=0.3)),
    ([1500, 3], 16, 1, 128, dict(stale=0.1, width=120)),
    ([40, 100, 90], 8, 2, 128, dict(all_stale=(1,))),
    ([0, 31, 0], 4, 2, 64, {}),
    ([1025, 2000, 512, 513], 8, 8, 64, dict(stale=0.05)),
    ([300] * 9, 32, 4, 128, dict(stale=0.5)),
    ([40], 3, 3, 128, dict(width=2)),  # longer than its table
    ([9000, 300], 8, 1, 64, dict(width=600, stale=0.05)),
    ([60, 20], 40, 10, 64, {}),
]


@pytest.mark.parametrize("i", range(len(DECODE)))
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("weighted", [True, False])
def test_decode(i, append, weighted):
    ctx, hq, hkv, D, more = DECODE[i]
    c = Case(100 + i, ctx, hq, hkv, D, **more)
    q, pool, meta, new = c.gpu(append)
    want = c.appended() if append else c.tiles
    ref, ref_lse, size, w = c.ref(want)
    say("decode", i, ctx[:5], hq, hkv, D, "append", append, "weighted", weighted)
    if weighted:
        w_in = c.rng.random(c.table.shape).astype(np.float32)
        out, lse, wo = lk.local_paged_attn_decode_kv4(
            q, pool, *meta, c.sm, weight_in=torch.from_numpy(w_in).to("cuda"), weight_decay=0.75,
            **new)
        owned = np.arange(c.table.shape[1]) < ((c.ctx + BS - 1) // BS)[:, None]
        check_weight(wo, np.where(owned, w + 0.75 * w_in.astype(np.float64), 0.0), "weights")
    else:
        out, lse = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("sm", [-0.3, 0.0, 1e-30, 4.0])
def test_softmax_scales(sm):
    """Negative, zero (every visible key weighs the same), vanishing and large scales."""
    c = Case(77, [100, 37], 8, 2, 128, new=[20, 37], stale=0.2)
    c.sm = sm
    q, pool, meta, new = c.gpu()
    ref, ref_lse, size, _ = c.ref(c.appended())
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, sm, **new)
    # (scores are up to 4 / 0.088 times those of the other tests, and so are their errors)
    wide = max(1.0, abs(sm) * math.sqrt(128))
    check_out(out, lse, ref, ref_lse, size, "prefill", wide)
    last = c.starts[1:] - 1
    rows = torch.from_numpy(last.astype(np.int64))
    out, lse = lk.local_paged_attn_decode_kv4(q[rows].contiguous(), pool, *meta, sm)
    check_out(out, lse, ref[last], ref_lse[last], size[last], "decode", wide)


def test_decode_of_many_requests():
    """More requests than the dispatch ranks (512)."""
    rng = np.random.default_rng(7)
    c = Case(8, rng.integers(0, 90, 530), 4, 2, 64, stale=0.1)
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, w = c.ref(want)
    wo = torch.full(c.table.shape, 9.0, device="cuda")
    out, lse, _ = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, weight_out=wo, **new)
    check_out(out, lse, ref, ref_lse, size, "out")
    check_weight(wo, w, "weights")
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128])
def test_decode_of_values_that_are_not_finite(D):
    """NaN groups: in a stale block and past the end they reach nothing, in a live token of
    one head that head's outputs only."""
    c = Case(11, [50, 30, 20], 4, 2, D, all_stale=(1,))
    nanv = np.full((1, 2, D), np.nan)
    one = np.ones((1, 2, D))
    one[0, 1] = np.nan  # KV head 1
    kv4.write(c.tiles, nanv, nanv, [c.table[0, 3]], [5])       # past request 0's end
    c.tiles[c.spare] = 255                                     # blocks of no request
    gone = [p for p in c.table[1, :2] if 0 <= p < c.num]       # request 1: all stale
    for p in gone:
        kv4.write(c.tiles, nanv.repeat(BS, 0), nanv.repeat(BS, 0), [p] * BS, range(BS))
    kv4.write(c.tiles, np.ones((1, 2, D)), one, [c.table[2, 0]], [2])
    c.vn[0, 0, 3] = 0x7f80  # the new token of request 0: an infinity in V of head 0
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    assert np.isnan(ref[2, 2:]).all() and not np.isnan(ref[2, :2]).any()
    assert np.isnan(ref[0, :2, :32]).all() and not np.isnan(ref[0, 2:]).any()
    out, lse = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")


PREFILL = [
    # (prefix, chunk, Hq, Hkv, D, options)
    ([0], [1], 1, 1, 64, {}),
    ([0, 5, 16], [1, 17, 40], 4, 4, 128, {}),
    ([100, 0, 33, 7], [3, 0, 130, 64], 8, 2, 64, dict(stale=0.3)),
    ([300], [200], 16, 1, 128, dict(stale=0.2)),
    ([64, 64], [70, 1], 9, 3, 64, dict(all_stale=(1,))),
    ([1700, 5], [2, 33], 4, 1, 128, dict(stale=0.1, width=130)),
    ([4500], [20], 2, 2, 64, {}),
    ([0], [300], 2, 1, 128, {}),
    ([20], [30], 4, 2, 64, dict(width=2)),  # longer than its table
    # few rows a request: 16 at a time
    ([1700, 5, 900, 64], [2, 5, 1, 0], 16, 4, 128, dict(stale=0.2)),
    ([700], [4], 16, 1, 64, {}),
    ([2000, 100, 0], [3, 40, 16], 8, 8, 128, dict(stale=0.1)),
    ([90, 40], [3, 2], 9, 3, 64, dict(all_stale=(1,), width=9)),
    ([30], [4], 8, 2, 128, dict(width=2)),  # longer than its table
    ([600, 3], [300, 90], 32, 32, 64, dict(stale=0.1)),
]


@pytest.mark.parametrize("i", range(len(PREFILL)))
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("wide", [True, False])
def test_prefill(i, append, wide):
    prefix, chunk, hq, hkv, D, more = PREFILL[i]
    ctx = np.array(prefix) + np.array(chunk)
    c = Case(200 + i, ctx, hq, hkv, D, new=chunk, **more)
    if wide and more.get("width") != 2:
        c.widen()
    say("prefill", i, prefix, chunk, hq, hkv, D, "append", append, "wide", wide)
    q, pool, meta, new = c.gpu(append)
    want = c.appended() if append else c.tiles
    ref, ref_lse, size, _ = c.ref(want)
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")
    assert np.array_equal(pool.cpu().numpy(), want)


# 16 rows at a time, 128 rows (one range each)
@pytest.mark.parametrize("most,hq,hkv", [(9, 32, 8), (90, 16, 16)])
def test_prefill_of_many_requests(most, hq, hkv):
    """More requests than one scan of the tile search takes, in one range (many tiles)."""
    rng = np.random.default_rng(3)
    prefix, chunk = rng.integers(0, 60, 140), rng.integers(0, most, 140)
    c = Case(4, prefix + chunk, hq, hkv, 64, new=chunk, stale=0.1)
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("prefix", [0, 700])
def test_few_rows_of_values_that_are_not_finite(D, prefix):
    """The same of 14 tokens (28 rows), and a slot past the context's end that holds NaN."""
    c = Case(22, [prefix + 14], 4, 2, D, new=[14])
    c.vn[5, 0, D - 1] = 0x7fc0    # V of token 5, KV head 0, the last group
    c.vn[9, 1, 2] = 0xff80
    c.kn[12, 1, 0] = 0x7f80       # K of token 12
    nan = np.full((1, 2, D), np.nan)
    last = prefix + 14
    kv4.write(c.tiles, nan, nan, [c.table[0, last // BS]], [last % BS])
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    assert not np.isnan(ref[:5]).any() and np.isnan(ref[5, :2, D - 32:]).all()
    assert not np.isnan(ref[5, :2, :D - 32]).any()
    assert not np.isnan(ref_lse[:12]).any() and np.isnan(ref_lse[12:, 2:]).all()
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("prefix", [0, 700])
@pytest.mark.parametrize("wide", [True, False])
def test_prefill_of_values_that_are_not_finite(D, prefix, wide):
    """A token whose K or V is not finite reaches the rows that see it and no other."""
    c = Case(21, [prefix + 60], 4, 2, D, new=[60])
    if wide:
        c.widen()
    c.vn[25, 0, D - 1] = 0x7fc0   # V of token 25, KV head 0, the last group
    c.vn[40, 1, 2] = 0xff80
    c.kn[50, 1, 0] = 0x7f80       # K of token 50: the whole rows from there on
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    assert not np.isnan(ref[:25]).any() and np.isnan(ref[25, :2, D - 32:]).all()
    assert not np.isnan(ref[25, :2, :D - 32]).any()
    assert not np.isnan(ref_lse[:50]).any() and np.isnan(ref_lse[50:, 2:]).all()
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")


@pytest.mark.parametrize("hq,wide", [(2, False), (8, False), (8, True)])
def test_prefill_skips_malformed_rows(hq, wide):
    c = Case(31, [40, 50, 20], hq, 2, 64, new=[10, 20, 5])
    if wide:  # 128 rows at a time
        c.widen()
    q, pool, meta, new = c.gpu()
    starts = c.starts.copy()
    starts[2:] = [30, 400]   # the last request's rows end past T: skipped whole
    out, lse = (torch.full(s, 7.0, dtype=t, device="cuda")
                for s, t in (((35, hq, 64), torch.bfloat16), ((35, hq), torch.float32)))
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    lk.local_paged_attn_prefill_kv4(q, dev(starts), pool, *meta, c.sm, out=out, lse=lse, **new)
    check_out(out[:30], lse[:30], ref[:30], ref_lse[:30], size[:30], "out")
    assert (out[30:] == 7).all() and (lse[30:] == 7).all()
    want[c.table[2, 1]] = c.tiles[c.table[2, 1]]
    want[c.table[2, 0]] = c.tiles[c.table[2, 0]]
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("new,width", [([30, 60], None), ([30, 60], 17000), ([3, 7], None)])
def test_blocks_past_32_bits(new, width):
    """A pool of more than 2^32 bytes: blocks at its far end."""
    hkv, D = 8, 128
    n = 2 ** 32 // (hkv * 17 * D) + 200
    c = Case(41, [90, 200], 8, hkv, D, new=new, width=width)
    far = n - 1 - np.arange(c.num)
    pool = torch.zeros((n, hkv, 17 * D), dtype=torch.uint8, device="cuda")
    pool[torch.from_numpy(far)] = torch.from_numpy(c.tiles).to("cuda")
    owned = np.arange(c.table.shape[1]) < ((c.ctx + BS - 1) // BS)[:, None]
    table = np.where(owned, n - 1 - np.where(owned, c.table, 0).astype(np.int64), -1)
    tags = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    tags[torch.from_numpy(far)] = dev(c.tags)
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    args = (pool, dev(table), dev(c.ctx), tags, dev(c.version), c.sm)
    out, lse = lk.local_paged_attn_prefill_kv4(dev_u16(c.q), dev(c.starts), *args,
                                               k_new=dev_u16(c.kn), v_new=dev_u16(c.vn))
    check_out(out, lse, ref, ref_lse, size, "prefill")
    assert np.array_equal(pool[torch.from_numpy(far)].cpu().numpy(), want)
    last = c.starts[1:] - 1
    out, lse = lk.local_paged_attn_decode_kv4(dev_u16(c.q[last]), *args)
    check_out(out, lse, ref[last], ref_lse[last], size[last], "decode")


# 16 rows at a time: a long request of few rows, several; 128 rows
@pytest.mark.parametrize("prefix,chunk,hq,hkv,D", [
    ([767, 0], [8, 4], 8, 2, 128), ([900, 30, 500], [5, 2, 20], 2, 2, 64),
    ([700, 41], [90, 300], 8, 2, 128), ([4500], [200], 4, 4, 64)])
def test_results_repeat(prefix, chunk, hq, hkv, D):
    """Calls of the same inputs return the same bits."""
    ctx = np.array(prefix) + np.array(chunk)
    c = Case(71, ctx, hq, hkv, D, new=chunk, stale=0.1)
    q, pool, meta, new = c.gpu()
    last = torch.from_numpy(c.starts[1:].astype(np.int64) - 1).to("cuda")
    w = torch.zeros(c.table.shape, device="cuda")

    def call():
        pre = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
        dec = lk.local_paged_attn_decode_kv4(q[last], pool, *meta, c.sm, weight_in=w,
                                             weight_out=torch.zeros_like(w), weight_decay=0.0)
        return pre + dec

    first = call()
    for r in range(30):
        for a, b in zip(call(), first):
            assert torch.equal(a, b), r


@pytest.mark.parametrize("wide", [True, False])
def test_replays_and_streams(wide):
    """A captured decode and prefill of one workspace, replayed between eager work, on a
    stream that is not the default one."""
    c = Case(51, [300, 41, 800], 8, 2, 128, new=[20, 1, 33], stale=0.1)
    if wide:
        c.widen()
    q, pool, meta, new = c.gpu()
    last = torch.from_numpy(c.starts[1:].astype(np.int64) - 1)
    ws = lk.Workspace()
    w = torch.zeros(c.table.shape, device="cuda")
    pre = lk.prepare_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, workspace=ws,
                                            **new)
    dec = lk.prepare_paged_attn_decode_kv4(
        q[last].contiguous(), pool, *meta, c.sm, k_new=new["k_new"][last].contiguous(),
        v_new=new["v_new"][last].contiguous(), weight_in=w, weight_out=w, weight_decay=0.5,
        workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p0, d0 = [t.clone() for t in pre()], [t.clone() for t in dec()]
        w.zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            pre()
            dec()
        for r in range(4):
            g.replay()
            s.synchronize()
            for a, b in zip(pre.outputs + dec.outputs[:2], p0 + d0[:2]):
                assert torch.equal(a, b)
            want = d0[2] * (2 - 0.5 ** r)  # weight, then 1.5, 1.75 ... of it
            assert torch.allclose(w, want, rtol=1e-6, atol=0)
            for t in pre.outputs + dec.outputs[:2]:
                t.zero_()
            torch.ones(1 << 20, device="cuda").sum().item()
    ref, ref_lse, size, _ = c.ref(c.appended())
    check_out(p0[0], p0[1], ref, ref_lse, size, "prefill")
    idx = last.numpy()
    check_out(d0[0], d0[1], ref[idx], ref_lse[idx], size[idx], "decode")


def test_calls_on_two_streams_at_once():
    """Calls over one pool with workspaces of their own: as one after the other."""
    c = Case(81, [900, 2000, 130, 64], 16, 4, 64, new=[40, 200, 1, 64], stale=0.1)
    c.widen()
    q, pool, meta, new = c.gpu()
    last = torch.from_numpy(c.starts[1:].astype(np.int64) - 1).to("cuda")
    lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)  # appends
    w = torch.rand(c.table.shape, device="cuda")
    pre = [lk.prepare_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm,
                                             workspace=lk.Workspace()) for _ in range(2)]
    dec = [lk.prepare_paged_attn_decode_kv4(q[last].contiguous(), pool, *meta, c.sm, weight_in=w,
                                            workspace=lk.Workspace()) for _ in range(2)]
    want = [t.clone() for t in pre[0]() + dec[0]()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for s, p, d in zip(streams, pre, dec[::-1]):
            with torch.cuda.stream(s):
                p()
                d()
    torch.cuda.synchronize()
    for p, d in zip(pre, dec):
        for a, b in zip(p.outputs + d.outputs, want):
            assert torch.equal(a, b)


def test_binding_refusals():
    c = Case(61, [20], 4, 2, 64)
    q, pool, meta, new = c.gpu()
    with pytest.raises(ValueError):  # another D
        lk.local_paged_attn_decode_kv4(q, pool[:, :, :17 * 32].contiguous(), *meta, c.sm)
    with pytest.raises(ValueError):
        lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, k_new=new["k_new"])
    with pytest.raises(ValueError):
        lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm,
                                       weight_in=torch.zeros((1, 9), device="cuda"))
    with pytest.raises(TypeError):
        lk.local_paged_attn_decode_kv4(q.float(), pool, *meta, c.sm)
    with pytest.raises(ValueError):  # not contiguous
        lk.local_kv4_pool_export(pool.transpose(0, 1))
    with pytest.raises(ValueError):
        lk.local_kv4_pool_import(torch.zeros(2, 2, 16 * 64, dtype=torch.bfloat16, device="cuda"),
                                 torch.zeros(2, 2, 16 * 64, dtype=torch.bfloat16, device="cuda"),
                                 pool)
    with pytest.raises(lk.LocalError):  # a view that does not start on 16 bytes
        flat = torch.zeros(pool.numel() + 8, dtype=torch.uint8, device="cuda")[8:]
        lk.local_paged_attn_decode_kv4(q, flat.view(pool.shape), *meta, c.sm)

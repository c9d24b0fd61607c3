"""The ways that 4-bit prefill calls of different sizes go: workspaces, and long partitions
of few rows against float64."""
from __future__ import annotations

import ctypes
import itertools
import os

import numpy as np
import pytest

from tests.conftest import ROOT

FAKE = ctypes.c_void_p(0x10000)


def _lib():
    return ctypes.CDLL(os.path.join(ROOT, "paper_2608_15241_amd", "liblocal.so"))


def _form(T, B, hq, hkv, width):
    return _lib().localk_prefill_kv4_form(ctypes.c_int64(T), B, hq, hkv, width)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hkv,group", [(1, 1), (1, 16), (4, 3), (8, 4), (32, 1), (128, 1)])
def test_workspace_ceiling(D, hkv, group):
    """One workspace, of the stated size, for all calls up to T rows and B requests."""
    f = _lib().local_paged_attn_prefill_kv4
    hq = hkv * group
    sizes = [1, 2, 15, 16, 33, 127, 128, 500, 1024, 1025, 4096, 4097, 32768, 1 << 18]
    for B, width in itertools.product([1, 2, 4, 31, 128, 700],
                                      [1, 16, 64, 65, 256, 511, 1024, 8192, 20000]):
        for T in sizes:
            n = ctypes.c_size_t(0)
            st = f(FAKE, FAKE, B, ctypes.c_int64(T), hq, hkv, D, FAKE, FAKE, FAKE,
                   ctypes.c_int64(100), 16, FAKE, width, FAKE, FAKE, FAKE, ctypes.c_float(0.1),
                   FAKE, FAKE, None, ctypes.byref(n), None)
            assert st == 0, (B, width, T)
            most = 2 ** 18 * (D + 2) * 4 + 64 * (T * group // 128 + B) + 49408
            assert n.value <= most, (B, width, T, n.value, most)


# Many requests of few rows, some behind contexts of more than 64 blocks for each of the
# ranges that the call's partial results leave: partitions of several groups of 64 blocks,
# which count from the context's end.
# (requests, tokens of each, first prefixes, Hq, Hkv, D, ranges)
LONG = [
    (1000, 15, [9000, 3100, 2047, 1030, 1015, 2032], 8, 8, 64, 2),
    (4000, 2, [12000, 1023, 1024, 5000], 16, 1, 128, 2),
    (600, 30, [4000, 995, 994, 2100, 0], 16, 16, 64, 1),
]


def _long_prefixes(B, first):
    return np.r_[first, np.random.default_rng(B).integers(0, 25, B - len(first))]


@pytest.mark.parametrize("B,n,first,hq,hkv,D,ranges", LONG)
def test_ranges_of_long_partitions(B, n, first, hq, hkv, D, ranges):
    width = (max(first) + n + 15) // 16
    form = _form(B * n, B, hq, hkv, width)
    assert form > 0 and form % 1000 == ranges
    assert width > form // 1000 * ranges


@pytest.mark.gpu
@pytest.mark.parametrize("B,n,first,hq,hkv,D,ranges", LONG)
def test_long_partitions(B, n, first, hq, hkv, D, ranges):
    from tests.gpu_helpers import say
    from tests.kv4_cases import quick_case
    c = quick_case(B, _long_prefixes(B, first) + n, hq, hkv, D, new=np.full(B, n), stale=0.3)
    c.tags[c.table[0, 60:200][c.table[0, 60:200] >= 0] % c.num] -= 1  # a group wholly stale
    say("long partitions", B, n, first, hq, hkv, D)
    _run(c, [*range(len(first)), len(first) + 1, B - 1], append=False)


def _check(c, b, out, lse, want, sm):
    """The rows of one request."""
    from oracle import kv4
    from tests.kv4_cases import check_counts
    from tests.kv4_helpers import check_out
    from tests.pool_helpers import bits_to_f64
    rows = slice(c.starts[b], c.starts[b + 1])
    if rows.start == rows.stop:
        return
    K, V = want
    ref, ref_lse, size, _ = kv4.attention(
        bits_to_f64(c.q[rows]), [0, c.new[b]], c.ctx[b:b + 1], c.table[b:b + 1], c.tags,
        c.version[b:b + 1], K, V, sm)
    if sm:
        check_out(out[rows], lse[rows], ref, ref_lse, size, "request %d" % b)
    else:
        check_counts(out[rows], lse[rows], ref, ref_lse, "request %d at 0" % b)


def _run(c, requests, append=True):
    import paper_2608_15241_amd as lk
    from oracle import kv4
    from tests.gpu_helpers import dev
    q, pool, meta, new = c.gpu(append)
    tiles = c.appended() if append else c.tiles
    want = kv4.unpack(tiles)
    for sm in (c.sm, 0.0):
        out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, sm, **new)
        for b in requests:
            _check(c, b, out, lse, want, sm)
    assert np.array_equal(pool.cpu().numpy(), tiles)


# A tile of 128 rows over more keys than a window lists (512 blocks): windows whose edge lies
# among stale blocks, one wholly stale, a last one of a single block.
WINDOWS = [(17600, 32, 16, 64), (8250, 32, 16, 128), (16 * 1025 - 40, 64, 8, 64)]


@pytest.mark.parametrize("prefix,B,hkv,D", WINDOWS)
def test_windows_are_of_one_range(prefix, B, hkv, D):
    assert _form(40 * B, B, hkv, hkv, (prefix + 55) // 16) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("prefix,B,hkv,D", WINDOWS)
def test_several_windows(prefix, B, hkv, D):
    from tests.gpu_helpers import say
    from tests.kv4_cases import quick_case
    chunk = np.full(B, 40)
    before = np.arange(B) * 7 % 50
    before[0] = prefix
    c = quick_case(B + D, before + chunk, hkv, hkv, D, new=chunk, stale=0.2)
    nb = (prefix + 55) // 16
    gone = np.r_[505:520, 520:1020 if nb > 1024 else 513]
    gone = gone[gone < nb - 4]
    c.table[0, gone] = np.where(gone % 3 == 0, -1, c.table[0, gone])
    inside = c.table[0, gone][(c.table[0, gone] >= 0) & (c.table[0, gone] < c.num)]
    c.tags[inside] = c.version[0] + 1
    say("windows", prefix, B, hkv, D)
    _run(c, [0, 1, B - 1])


# More requests than the planner scans at once (256), more tiles than it keeps in LDS (1024),
# both, and tiles that spill while every request's sizes are at hand.
PLANS = [(300, 9, 13, 60, 32, 8, 64), (1100, 2, 5, 130, 16, 1, 64), (200, 40, 60, 60, 16, 1, 64)]


@pytest.mark.parametrize("B,lo,hi,prefix,hq,hkv,D", PLANS)
def test_plans_are_of_128_rows(B, lo, hi, prefix, hq, hkv, D):
    chunk = _chunks(B, lo, hi)
    assert _form(chunk.sum(), B, hq, hkv, (prefix + hi + 15) // 16) < 0
    tiles = sum(-(-n * (hq // hkv) // 128) for n in chunk)
    assert B > 256 or tiles > 1024


def _chunks(B, lo, hi):
    return np.random.default_rng(B).integers(lo, hi, B)


@pytest.mark.gpu
@pytest.mark.parametrize("B,lo,hi,prefix,hq,hkv,D", PLANS)
def test_large_plans(B, lo, hi, prefix, hq, hkv, D):
    from tests.gpu_helpers import say
    from tests.kv4_cases import quick_case
    chunk = _chunks(B, lo, hi)
    before = np.random.default_rng(B + 1).integers(0, prefix, B)
    c = quick_case(B, before + chunk, hq, hkv, D, new=chunk, stale=0.1,
                   width=(prefix + hi + 15) // 16)
    say("plans", B, lo, hi, prefix, hq, hkv, D)
    some = np.unique(np.r_[0, 63, 64, 127, 128, 255, 256, 257, 511, 512, B - 2, B - 1,
                           np.random.default_rng(2).integers(0, B, 25)])
    _run(c, some[some < B])

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


# (prefixes, chunks, Hq, Hkv, D, table width, blocks of a partition): groups of 64 blocks
# that begin anywhere in a partition, which count from the context's end
LONG = [
    ([9000] + [3] * 19, [1] * 20, 8, 8, 64, 17000, 192),
    ([3100, 2047, 5] + [30] * 29, [6, 1, 40] + [1] * 29, 8, 8, 128, 17000, 320),
    ([1500] + [0] * 69, [2] * 70, 64, 4, 64, 17000, 896),
]


@pytest.mark.parametrize("i", range(len(LONG)))
def test_long_partitions_are_the_named_ones(i):
    prefix, chunk, hq, hkv, _, width, blocks = LONG[i]
    assert _form(sum(chunk), len(chunk), hq, hkv, width) == blocks


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(LONG)))
def test_long_partitions(i):
    import paper_2608_15241_amd as lk
    from tests.gpu_helpers import dev, say
    from tests.kv4_helpers import check_out
    from tests.kv4_cases import quick_case
    prefix, chunk, hq, hkv, D, width, _ = LONG[i]
    c = quick_case(300 + i, np.array(prefix) + np.array(chunk), hq, hkv, D, new=chunk, stale=0.3)
    c.tags[c.table[0, 60:200][c.table[0, 60:200] >= 0] % c.num] -= 1  # a group wholly stale
    c.widen()
    assert c.table.shape[1] == width
    say("long partitions", i, prefix[:3], chunk[:3], hq, hkv, D)
    q, pool, meta, new = c.gpu()
    want = c.appended()
    ref, ref_lse, size, _ = c.ref(want)
    out, lse = lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)
    check_out(out, lse, ref, ref_lse, size, "out")
    assert np.array_equal(pool.cpu().numpy(), want)

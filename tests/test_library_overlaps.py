"""Outputs that overlap what they must not are refused (host checks: no GPU)."""
import ctypes

import pytest

import paper_2608_15241_amd as lk

ERR_SHAPE = 2
B, MB, NB = 3, 40, 50
ROWS, EACH = B * MB * 4, B * 4


@pytest.fixture(scope="module")
def lib():
    return lk.load_library()


def _refused(lib, status, what):
    assert status == ERR_SHAPE, what
    assert b"overlap" in lib.local_last_error(), what


NAMES = ("table", "ctx", "weight", "keep", "version", "rv", "table_out", "ctx_out", "weight_out",
         "evicted", "n_evicted")
SIZES = dict(table=ROWS, weight=ROWS, table_out=ROWS, weight_out=ROWS, evicted=ROWS,
             version=NB * 4)


def _evict(lib, **over):
    p = {n: 0x100000 * (i + 1) for i, n in enumerate(NAMES)}
    p.update(over)
    v = {n: ctypes.c_void_p(a) for n, a in p.items()}
    return lib.local_kv_evict(v["table"], B, MB, v["ctx"], 16, v["weight"], v["keep"], 1, 2,
                              v["version"], NB, v["rv"], v["table_out"], v["ctx_out"],
                              v["weight_out"], v["evicted"], v["n_evicted"], None)


@pytest.mark.parametrize("out", NAMES[6:])
@pytest.mark.parametrize("other", NAMES)
def test_evict_outputs(lib, out, other):
    if out == other:
        return
    at = 0x100000 * (1 + NAMES.index(other))
    size, other_size = SIZES.get(out, EACH), SIZES.get(other, EACH)
    for shift in (0, other_size - 4, 4 - size):  # the whole, the last word, the first word
        if shift == 0 and out == other + "_out":
            continue  # in place: allowed
        _refused(lib, _evict(lib, **{out: at + shift}), (out, other, shift))

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


@pytest.mark.parametrize("shift", [4, -4, ROWS - 4, 4 - ROWS])
@pytest.mark.parametrize("name", ["local_paged_attn_decode_weighted",
                                  "local_paged_attn_decode_kv4"])
def test_weights_in_part(lib, name, shift):
    a = lambda i: ctypes.c_void_p(0x100000 * i)  # noqa: E731
    pools = [a(4)] if name.endswith("kv4") else [a(4), a(5)]
    n = ctypes.c_size_t(1 << 40)
    status = getattr(lib, name)(a(1), B, 8, 4, 64, a(2), a(3), *pools, NB, 16, a(6), MB, a(7),
                                a(8), a(9), 0.1, a(10), a(11), a(12), 1.0,
                                ctypes.c_void_p(0x100000 * 12 + shift), a(13), ctypes.byref(n),
                                None)
    _refused(lib, status, (name, shift))

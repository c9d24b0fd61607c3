"""4-bit decode without block weights takes what the bf16 decode takes (host checks: no GPU)."""
import ctypes

import pytest

import paper_2608_15241_amd as lk

FAKE = ctypes.c_void_p(0x10000)


def _status(Hq, Hkv, decay, weights):
    lib = lk.load_library()
    w = FAKE if weights else None
    n = ctypes.c_size_t(0)
    st = lib.local_paged_attn_decode_kv4(FAKE, 2, Hq, Hkv, 64, FAKE, FAKE, FAKE, 100, 16, FAKE, 8,
                                         FAKE, FAKE, FAKE, 0.1, FAKE, FAKE, w, decay, w, None,
                                         ctypes.byref(n), None)
    assert st != 0 or n.value > 0
    return st


@pytest.mark.parametrize("Hq,Hkv,decay", [(16400, 2050, 1.0), (8, 2, float("nan")), (8, 2, -1.0)])
def test_limits_of_the_weights_hold_with_weights_only(Hq, Hkv, decay):
    assert _status(Hq, Hkv, decay, False) == 0
    assert _status(Hq, Hkv, decay, True) == 3

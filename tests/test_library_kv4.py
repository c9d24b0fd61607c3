"""Refusals and workspace sizes of the 4-bit pool's entry points, the weighted decode and
the eviction (host checks: no GPU)."""
import ctypes

import pytest

import paper_2608_15241_amd as lk

OK, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE = 0, 1, 2, 3, 4
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10008)


@pytest.fixture(scope="module")
def lib():
    return lk.load_library()


def _args(base, **over):
    return [over.get(k, v) for k, v in base.items()]


DECODE4 = dict(q=FAKE, B=4, Hq=32, Hkv=8, D=128, kn=FAKE, vn=FAKE, kv4=FAKE, nb=100, bs=16,
               bt=FAKE, mb=64, ctx=FAKE, bv=FAKE, rv=FAKE, sm=0.1, out=FAKE, lse=FAKE, wi=FAKE,
               decay=1.0, wo=FAKE)
WEIGHTED = dict(q=FAKE, B=4, Hq=32, Hkv=8, D=128, kn=FAKE, vn=FAKE, kc=FAKE, vc=FAKE, nb=100,
                bs=16, bt=FAKE, mb=64, ctx=FAKE, bv=FAKE, rv=FAKE, sm=0.1, out=FAKE, lse=FAKE,
                wi=FAKE, decay=1.0, wo=FAKE)
PREFILL4 = dict(q=FAKE, ip=FAKE, B=4, T=100, Hq=32, Hkv=8, D=128, kn=FAKE, vn=FAKE, kv4=FAKE,
                nb=100, bs=16, bt=FAKE, mb=64, ctx=FAKE, bv=FAKE, rv=FAKE, sm=0.1, out=FAKE,
                lse=FAKE)
BIG = ctypes.c_size_t(1 << 40)


@pytest.mark.parametrize("name,base", [("local_paged_attn_decode_kv4", DECODE4),
                                       ("local_paged_attn_decode_weighted", WEIGHTED),
                                       ("local_paged_attn_prefill_kv4", PREFILL4)])
def test_attention_refusals(lib, name, base):
    f = getattr(lib, name)

    def call(ws=FAKE, n=BIG, **over):
        return f(*_args(base, **over), ws, ctypes.byref(n) if n is not None else None, None)

    assert call(n=None) == ERR_WORKSPACE
    assert call(B=0) == OK  # nothing to do, nothing launched
    for bad in (dict(B=-1), dict(Hq=0), dict(Hkv=0), dict(mb=0), dict(nb=0), dict(Hq=31)):
        assert call(**bad) == ERR_SHAPE, bad
    for bad in (dict(D=96), dict(bs=8), dict(Hq=136, Hkv=8)):
        assert call(**bad) == ERR_UNSUPPORTED, bad
    for bad in ("kn", "vn", "q", "bt", "ctx", "bv", "rv", "out"):
        assert call(**{bad: None}) == ERR_NULL, bad
    n = ctypes.c_size_t(0)
    assert call(ws=None, n=n) == OK and n.value > 0
    assert call(n=ctypes.c_size_t(n.value - 1)) == ERR_WORKSPACE
    assert name[6:].encode() in lib.local_last_error()
    if "kv4" in base:
        assert call(kv4=None) == ERR_NULL
        for bad in ("q", "kn", "vn", "kv4", "out"):
            assert call(**{bad: ODD}) == ERR_UNSUPPORTED, bad
        assert call(ws=ODD) == ERR_UNSUPPORTED
        assert b"16 bytes" in lib.local_last_error()
    if "decay" in base:
        for bad in (-0.1, 1.5, float("nan"), float("inf")):
            assert call(decay=bad) == ERR_UNSUPPORTED
        assert call(wo=None) == ERR_NULL
        assert call(Hq=16400, Hkv=2050) == ERR_UNSUPPORTED


def test_workspace_sizes(lib):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    # partials as the unweighted call's, then 4 bytes for each (request, block, query head)
    assert lib.local_paged_attn_decode_weighted(*_args(WEIGHTED), None, ctypes.byref(n),
                                                None) == OK
    plain = [v for k, v in WEIGHTED.items() if k not in ("wi", "decay", "wo")]
    assert lib.local_paged_attn_decode(*plain, None, ctypes.byref(m), None) == OK
    assert n.value == (m.value + 255) // 256 * 256 + 4 * 64 * 32 * 4
    # few tiles of 128 rows (1200 / 128 + 4 requests, 8 heads): key ranges of at least
    # 104 / 4 = 26 blocks, so 2 of 64; (D + 2) floats a row and range, behind 48 bytes a unit
    # and 16 a tile
    a = lambda v: (v + 255) // 256 * 256  # noqa: E731
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=300), None, ctypes.byref(n),
                                            None) == OK
    assert n.value == a(48 * 13 * 2 + 16 * 13) + 300 * 32 * 2 * 130 * 4
    # little work in all: partitions of 64 blocks, halved to 16, no plan
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4), None, ctypes.byref(n), None) == OK
    assert n.value == 100 * 32 * 4 * 130 * 4
    # one block a request: one partition, written as it is
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, mb=1), None, ctypes.byref(n),
                                            None) == OK
    assert n.value == 256
    # few rows a request: partitions of 16 blocks, no plan
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=4), None, ctypes.byref(n),
                                            None) == OK
    assert n.value == 4 * 32 * 4 * 130 * 4
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=1 << 20), None, ctypes.byref(n),
                                            None) == OK
    assert n.value == a(64 * ((1 << 15) + 4))
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=1 << 30), None, ctypes.byref(n),
                                            None) == ERR_UNSUPPORTED
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=-1), None, ctypes.byref(n),
                                            None) == ERR_SHAPE
    assert lib.local_paged_attn_prefill_kv4(*_args(PREFILL4, T=0), FAKE, ctypes.byref(BIG),
                                            None) == OK


def test_weights_need_an_output(lib):
    call = lambda **o: lib.local_paged_attn_decode_kv4(*_args(DECODE4, **o), FAKE,  # noqa: E731
                                                       ctypes.byref(BIG), None)
    assert call(wo=None) == ERR_NULL
    assert call(B=0, wi=None, wo=None) == OK


def test_pool_conversion_refusals(lib):
    P = ctypes.c_void_p
    A, B, C = P(0x100000), P(0x200000), P(0x300000)
    imp = lambda k=A, v=B, nb=4, h=8, d=128, bs=16, ids=None, n=-1, o=C: (  # noqa: E731
        lib.local_kv4_pool_import(k, v, nb, h, d, bs, ids, n, o, None))
    exp = lambda k=A, v=B, nb=4, h=8, d=128, bs=16, ids=None, n=-1, o=C: (  # noqa: E731
        lib.local_kv4_pool_export(o, nb, h, d, bs, ids, n, k, v, None))
    for f in (imp, exp):
        assert f(k=None, v=None, o=None, nb=0) == OK
        assert f(ids=FAKE, n=0) == OK and f(ids=None, n=0) == OK
        assert f(ids=None, n=2) == ERR_NULL
        assert f(k=None) == ERR_NULL and f(v=None) == ERR_NULL and f(o=None) == ERR_NULL
        assert f(nb=-1) == ERR_SHAPE and f(h=0) == ERR_SHAPE and f(ids=FAKE, n=-2) == ERR_SHAPE
        assert f(d=96) == ERR_UNSUPPORTED and f(bs=8) == ERR_UNSUPPORTED
        assert f(o=P(0x300004)) == ERR_UNSUPPORTED and f(k=P(0x100002)) == ERR_UNSUPPORTED
        # 4 blocks x 8 heads: 128 KB of K and of V, 68 KB of 4-bit tiles
        assert f(v=P(0x110000)) == ERR_SHAPE and f(o=P(0x1f0000)) == ERR_SHAPE
        assert b"overlap" in lib.local_last_error()
        assert f(ids=FAKE, n=1 << 41) == ERR_UNSUPPORTED


def test_evict_refusals(lib):
    base = dict(bt=FAKE, B=2, mb=8, ctx=FAKE, bs=16, w=FAKE, keep=FAKE, sink=1, recent=2, bv=FAKE,
                nb=10, rv=FAKE, to=FAKE, co=FAKE, wo=FAKE, ev=FAKE, ne=FAKE)
    call = lambda **o: lib.local_kv_evict(*_args(base, **o), None)  # noqa: E731
    assert call(B=0) == OK
    for bad in (dict(B=-1), dict(mb=0), dict(nb=0), dict(sink=-1), dict(recent=0)):
        assert call(**bad) == ERR_SHAPE, bad
    assert call(bs=32) == ERR_UNSUPPORTED
    for k in ("bt", "ctx", "w", "keep", "bv", "rv", "to", "co", "wo", "ev", "ne"):
        assert call(**{k: None}) == ERR_NULL, k
    assert b"kv_evict" in lib.local_last_error()

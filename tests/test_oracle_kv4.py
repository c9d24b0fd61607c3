"""Pins of oracle/kv4.py by hand-worked values (CPU)."""
import math

import numpy as np
import pytest

from oracle import kv4


def test_rounding_by_hand():
    # amax = 6 -> 2^0: the magnitudes stand for themselves, halfway goes to the even code
    x = np.zeros(32)
    x[:16] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.7, -5, 0.3, 4.9, 5.1, -6, 0.2]
    c, s = kv4.quantise(x)
    assert s.tolist() == [127]
    assert c[:16].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 9, 14, 1, 6, 7, 15, 0]
    assert c[16:].tolist() == [0] * 16
    v = kv4.values(c, s)
    assert v[:8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4] and v[9] == -0.5


@pytest.mark.parametrize("amax,byte", [(6.0, 127), (6.03125, 128), (12.0, 128), (1.0, 125),
                                       (0.75, 124), (0.0, 2), (2.0 ** -133, 2),
                                       (2.0 ** 127 * 1.9921875, 252), (math.inf, 255),
                                       (math.nan, 255)])
def test_scale_byte(amax, byte):
    x = np.zeros(32)
    x[7] = -amax
    c, s = kv4.quantise(x)
    assert s.tolist() == [byte]
    if byte == 255:
        assert not c.any() and np.isnan(kv4.values(c, s)).all()


@pytest.mark.parametrize("D", [64, 128])
def test_every_byte_has_one_place(D):
    ck, cv, sk, sv = kv4.places(D)
    for at in (ck, cv):  # two values a byte: dims 2i and 2i + 1 of one slot
        assert (at[:, 0::2] == at[:, 1::2]).all()
    codes = np.concatenate([ck[:, ::2].ravel(), cv[:, ::2].ravel()])
    scales = np.concatenate([sk[:, ::32].ravel(), sv[:, ::32].ravel()])
    assert sorted(np.concatenate([codes, scales]).tolist()) == list(range(17 * D))


@pytest.mark.parametrize("D", [64, 128])
def test_pack_and_unpack(D):
    rng = np.random.default_rng(D)
    k, v = rng.standard_normal((2, 3, 2, 16, D))
    tiles = kv4.pack(k, v)
    for got, x in zip(kv4.unpack(tiles), (k, v)):
        c, s = kv4.quantise(x)
        assert np.array_equal(got, kv4.values(c, s))
        # half a step of the widest spacing (2 scale units) of each group's scale
        unit = np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=-1)
        assert (np.abs(got - x) <= unit).all()
    again = kv4.pack(*kv4.unpack(tiles))
    assert np.array_equal(kv4.unpack(again)[0], kv4.unpack(tiles)[0])


def test_attention_by_hand():
    # two keys of scores 0 and ln 3: weights 1/4, 3/4; the second block is stale
    D = 64
    K, V = np.zeros((3, 1, 16, D)), np.zeros((3, 1, 16, D))
    K[2, 0, 1, 0], V[2, 0, 0, 5], V[2, 0, 1, 5] = math.log(3), 8.0, 4.0
    K[1], V[1] = np.nan, np.nan
    table = np.array([[2, 1, -5]], np.int32)
    q = np.zeros((1, 1, D))
    q[0, 0, 0] = 1.0
    out, lse, size, w = kv4.attention(q, [0, 1], [2], table, np.array([7, 6, 7]), [7], K, V, 1.0)
    assert out[0, 0, 5] == pytest.approx(5.0) and lse[0, 0] == pytest.approx(math.log(4))
    assert w[0].tolist() == pytest.approx([1.0, 0, 0])
    out, lse, _, w = kv4.attention(q, [0, 1], [40], table, np.array([7, 6, 6]), [7], K, V, 1.0)
    assert lse[0, 0] == -np.inf and not out.any() and not w.any()


def test_evict_by_hand():
    table = np.array([[10, 11, 12, 13, 14, 15, 99]], np.int32)
    tags = np.full(16, 1)
    tags[12] = 0  # stale
    w = np.array([[0.0, 5.0, 9.0, 1.0, 1.0, 0.0, 3.0]])
    t, c, wo, e, n = kv4.evict(table, np.array([16 * 5 + 3]), w, [4], tags, [1], 1, 1)
    # block 0 and the last one (5) are safe; 11 and the first of the two weights 1 stay
    assert t[0].tolist() == [10, 11, 13, 15, -1, -1, -1] and c[0] == 16 * 3 + 3
    assert wo[0].tolist() == [0, 5, 1, 0, 0, 0, 0]
    assert e[0].tolist() == [12, 14, -1, -1, -1, -1, -1] and n[0] == 2

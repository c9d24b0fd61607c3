"""The 4-bit KV pool, block weights and block eviction, in float64 (test infrastructure).

Written from the definitions in include/local.h with explicit index arithmetic and
loops over requests; it shares no code with the kernels.
"""
from __future__ import annotations

import math

import numpy as np

BS = 16
MAGS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """[..., D] float64 -> (codes uint8 [..., D], scale bytes uint8 [..., D/32])."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    codes = np.zeros(g.shape, np.uint8)
    scales = np.zeros(g.shape[:-1], np.uint8)
    flat, fc, fs = g.reshape(-1, 32), codes.reshape(-1, 32), scales.reshape(-1)
    for i, row in enumerate(flat):
        amax = np.abs(row).max()
        if not np.isfinite(amax):
            fs[i] = 255
            continue
        e = -125
        while e < 125 and amax > 6.0 * 2.0 ** e:
            e += 1
        y = np.abs(row) / 2.0 ** e
        far = np.abs(y[:, None] - MAGS[None, :])
        near = far.min(axis=1, keepdims=True)
        tied = far == near  # one index, or two neighbours: the even one
        idx = np.where(tied.sum(1) == 1, tied.argmax(1),
                       np.where(tied.argmax(1) % 2 == 0, tied.argmax(1), tied.argmax(1) + 1))
        fc[i] = idx + 8 * np.signbit(row)
        fs[i] = e + 127
    return codes.reshape(x.shape), scales


def values(codes, scales):
    """What codes and scale bytes stand for, in float64."""
    v = MAGS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def places(D):
    """Byte of each value's code and scale in a tile, [16][D]: (K code, V code, K scale,
    V scale)."""
    slot, d = np.arange(BS)[:, None], np.arange(D)[None, :]
    return ((d // (D // 4) * 16 + slot) * (D // 8) + d % (D // 4) // 2,
            8 * D + ((slot // 4 * 16 + d // (D // 16)) * 4 + slot % 4) * (D // 32)
            + d % (D // 16) // 2,
            16 * D + d // 32 * 16 + slot,
            16 * D + D // 2 + (slot // 4 * (D // 32) + d // 32) * 4 + slot % 4)


def write(tiles, k, v, blocks, slots):
    """Rounds tokens k, v [n][Hkv][D] and writes them at (blocks[i], slots[i])."""
    D = k.shape[-1]
    at = places(D)
    shift = (4 * (np.arange(D) % 2)).astype(np.uint8)
    for x, code_at, scale_at in ((k, at[0], at[2]), (v, at[1], at[3])):
        codes, scales = quantise(x)
        for i, (p, s) in enumerate(zip(blocks, slots)):
            t = tiles[p]  # [Hkv][17 D]
            t[:, code_at[s]] = 0
            for half in (0, 1):
                sel = np.arange(half, D, 2)
                t[:, code_at[s][sel]] |= codes[i][:, sel] << shift[sel]
            t[:, scale_at[s]] = np.repeat(scales[i], 32, axis=-1)
    return tiles


def pack(k, v):
    """Token-major [nb][Hkv][16][D] float64 -> tiles uint8 [nb][Hkv][17 D]."""
    nb, hkv, _, D = k.shape
    tiles = np.zeros((nb, hkv, 17 * D), np.uint8)
    blocks, slots = np.repeat(np.arange(nb), BS), np.tile(np.arange(BS), nb)
    return write(tiles, k.transpose(0, 2, 1, 3).reshape(-1, hkv, D),
                 v.transpose(0, 2, 1, 3).reshape(-1, hkv, D), blocks, slots)


def unpack(tiles):
    """Tiles -> token-major float64 (K, V) [nb][Hkv][16][D]."""
    D = tiles.shape[-1] // 17
    ck, cv, sk, sv = places(D)
    shift = 4 * (np.arange(D) % 2)
    out = []
    for c, s in ((ck, sk), (cv, sv)):
        codes = (tiles[:, :, c] >> shift) & 15
        out.append(values(codes, tiles[:, :, s][..., ::32]))
    return out


def attention(q, starts, ctx, table, tags, version, K, V, sm):
    """Rows q [T][Hq][D] of request b: starts[b] .. starts[b+1], its last positions.
    K, V token-major [nb][Hkv][16][D] float64. Returns (out, lse, sum of w|v| per out
    value, weight of each block [B][max_blocks])."""
    T, hq, D = q.shape
    hkv = K.shape[1]
    group = hq // hkv
    out, size = np.zeros((T, hq, D)), np.zeros((T, hq, D))
    lse = np.full((T, hq), -np.inf)
    weight = np.zeros(table.shape)
    for b in range(len(ctx)):
        L, n = int(ctx[b]), int(starts[b + 1] - starts[b])
        nb = min((L + BS - 1) // BS, table.shape[1])
        ok = [j for j in range(nb) if 0 <= table[b, j] < len(tags)
              and tags[table[b, j]] == version[b]]
        if not ok or n == 0:
            continue
        key = np.concatenate([np.arange(j * BS, (j + 1) * BS) for j in ok])
        k = K[table[b, ok]].transpose(0, 2, 1, 3).reshape(-1, hkv, D)
        v = V[table[b, ok]].transpose(0, 2, 1, 3).reshape(-1, hkv, D)
        for i in range(n):
            t, pos = int(starts[b]) + i, L - n + i
            see = key <= pos
            if not see.any():
                continue
            for h in range(hq):
                s = sm * (k[see, h // group] @ q[t, h])
                top = s.max()
                w = np.exp(s - top)
                lse[t, h] = top + math.log(w.sum()) if w.sum() == w.sum() else np.nan
                w = w / w.sum()
                out[t, h] = w @ v[see, h // group]
                size[t, h] = w @ np.abs(v[see, h // group])
                np.add.at(weight[b], key[see] // BS, w)
    return out, lse, size, weight


def evict(table, ctx, weight, keep, tags, version, sink, recent):
    """(table_out, ctx_out, weight_out, evicted, n_evicted) of the definition."""
    B, width = table.shape
    t_out, e_out = np.full_like(table, -1), np.full_like(table, -1)
    w_out, c_out, n_out = np.zeros_like(weight), ctx.copy(), np.zeros(B, np.int32)
    for b in range(B):
        nb = min((max(int(ctx[b]), 0) + BS - 1) // BS, width)
        safe = {j for j in range(nb) if j < sink or j >= nb - recent}

        def rank(j):
            p = table[b, j]
            stale = not (0 <= p < len(tags)) or tags[p] != version[b]
            w = weight[b, j]
            return (stale, -(w if w > 0 else 0.0) if not stale else 0.0, j)

        rest = sorted((j for j in range(nb) if j not in safe), key=rank)
        kept = sorted(safe) + rest[:max(0, int(keep[b]) - len(safe))]
        kept.sort()
        gone = [j for j in range(nb) if j not in set(kept)]
        t_out[b, :len(kept)], w_out[b, :len(kept)] = table[b, kept], weight[b, kept]
        e_out[b, :len(gone)] = table[b, gone]
        n_out[b] = len(gone)
        c_out[b] = ctx[b] - BS * len(gone)
    return t_out, c_out, w_out, e_out, n_out

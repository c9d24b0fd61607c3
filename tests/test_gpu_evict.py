"""Block weights of bf16 decode, eviction, and a run of everything together (tolerances:
kv4_helpers.py).
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
from tests.pool_helpers import bits_to_f64, dense_to_pool, f32_to_bf16_bits, make_table

pytestmark = pytest.mark.gpu
BS = 16


def bf16_case(seed, ctx, hq, hkv, D, stale):
    rng = np.random.default_rng(seed)
    table, num = make_table(rng, ctx, extra_blocks=2)
    kd, vd = (f32_to_bf16_bits(rng.standard_normal((num, hkv, BS, D))) for _ in range(2))
    tags, version = np.full(num, 3, np.int32), np.full(len(ctx), 3, np.int32)
    for b, L in enumerate(ctx):
        for j in range((L - 1) // BS):
            if rng.random() < stale:
                tags[table[b, j]] = 2
    q = f32_to_bf16_bits(rng.standard_normal((len(ctx), hq, D)))
    return rng, table, kd, vd, tags, version, q


@pytest.mark.parametrize("ctx,hq,hkv,D,stale", [
    ([1], 1, 1, 64, 0.0), ([17, 600, 16, 33], 8, 2, 128, 0.2), ([900, 4], 16, 1, 64, 0.1),
    ([1200] * 5, 4, 4, 128, 0.0), (list(range(1, 540)), 2, 1, 64, 0.3)])
@pytest.mark.parametrize("append", [True, False])
def test_decode_weighted(ctx, hq, hkv, D, stale, append):
    rng, table, kd, vd, tags, version, q = bf16_case(len(ctx), ctx, hq, hkv, D, stale)
    say("weighted", len(ctx), ctx[:4], hq, hkv, D, append)
    sm = 1.0 / math.sqrt(D)
    ctx = np.array(ctx, np.int32)
    K, V = (dev_u16(t) for t in dense_to_pool(kd, vd))
    meta = [dev(t) for t in (table, ctx, tags, version)]
    new = {}
    if append:
        kn, vn = (f32_to_bf16_bits(rng.standard_normal((len(ctx), hkv, D))) for _ in range(2))
        new = dict(k_new=dev_u16(kn), v_new=dev_u16(vn))
        at = (table[np.arange(len(ctx)), (ctx - 1) // BS], (ctx - 1) % BS)
        kd[at[0], :, at[1]], vd[at[0], :, at[1]] = kn, vn
    w_in = rng.random(table.shape).astype(np.float32)
    w = torch.from_numpy(w_in).to("cuda")
    K1, V1 = K.clone(), V.clone()
    o1, l1 = lk.local_paged_attn_decode(dev_u16(q), K1, V1, *meta, sm, Hkv=hkv, **new)
    out, lse, wo = lk.local_paged_attn_decode_weighted(
        dev_u16(q), K, V, *meta, sm, Hkv=hkv, weight_in=w, weight_out=w, weight_decay=0.5, **new)
    assert wo is w
    assert torch.equal(out, o1) and torch.equal(lse, l1)
    assert torch.equal(K, K1) and torch.equal(V, V1)
    ref, ref_lse, size, wr = kv4.attention(bits_to_f64(q), np.arange(len(ctx) + 1), ctx, table,
                                           tags, version, bits_to_f64(kd), bits_to_f64(vd), sm)
    check_out(out, lse, ref, ref_lse, size, "out")
    owned = np.arange(table.shape[1]) < ((ctx + BS - 1) // BS)[:, None]
    check_weight(wo, np.where(owned, wr + 0.5 * w_in.astype(np.float64), 0.0), "weights")


def test_weights_of_requests_without_keys():
    """ctx 0 and wholly stale contexts: no weight, what was there decays."""
    _, table, kd, vd, tags, version, q = bf16_case(5, [40, 40, 40], 4, 2, 64, 0.0)
    tags[table[1]] = 9
    ctx = np.array([40, 40, 0], np.int32)
    K, V = (dev_u16(t) for t in dense_to_pool(kd, vd))
    w = torch.ones(table.shape, device="cuda")
    out, lse, wo = lk.local_paged_attn_decode_weighted(
        dev_u16(q), K, V, *[dev(t) for t in (table, ctx, tags, version)], 0.125, Hkv=2,
        weight_in=w, weight_decay=0.25)
    wo = wo.cpu().numpy()
    assert (wo[1] == 0.25).all() and (wo[2] == 0).all()
    assert wo[0].sum() == pytest.approx(4 + 3 * 0.25, rel=1e-5)  # one softmax a query head
    assert not out[1:].any() and np.isneginf(f64(lse)[1:]).all()


def evict_case(seed, ctx, width, keep, stale=0.2, ties=True):
    rng = np.random.default_rng(seed)
    B = len(ctx)
    nb = np.minimum((np.maximum(ctx, 0) + BS - 1) // BS, width)
    num = int(nb.sum()) + 4
    table = rng.integers(-2 ** 31, 2 ** 31 - 1, (B, width)).astype(np.int32)
    tags, version = np.full(num, 5, np.int32), np.full(B, 5, np.int32)
    ids, at = rng.permutation(num), 0
    for b in range(B):
        table[b, :nb[b]] = ids[at:at + nb[b]]
        at += nb[b]
    for b in range(B):
        for j in range(nb[b]):
            if rng.random() < stale:
                if rng.random() < 0.5:
                    tags[table[b, j]] = 4
                else:
                    table[b, j] = rng.choice([-1, num, -2 ** 31])
    w = rng.random((B, width)).astype(np.float32) ** 8
    if ties:
        w = np.where(rng.random(w.shape) < 0.4, np.float32(0.25), w)
        w = np.where(rng.random(w.shape) < 0.1, rng.choice(
            [0.0, -0.0, -3.0, np.inf, np.nan, 1e-42], w.shape), w).astype(np.float32)
    return table, np.array(ctx, np.int32), w, np.array(keep, np.int32), tags, version


@pytest.mark.parametrize("ctx,width,keep,sink,recent", [
    ([1], 1, [1], 0, 1),
    ([0, 16, 17, 400, 33], 30, [0, 0, 1, 12, -5], 1, 2),
    ([4000, 1600, 77, 2560], 250, [100, 99, 3, 160], 4, 8),
    ([4096] * 3, 256, [256, 255, 1], 0, 1),
    ([5000, 5000], 400, [200, 5], 500, 1),      # everything protected
    ([5000, 4999], 400, [200, 5], 3, 2 ** 31 - 1),
    ([16 * 9000 - 3, 16 * 8193], 9100, [4000, 8000], 2, 3),  # more keys than LDS holds
    ([1000], 20, [6], 1, 1),                     # longer than its table
])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(ctx, width, keep, sink, recent, in_place):
    table, ctx, w, keep, tags, version = evict_case(width + len(ctx), ctx, width, keep)
    say("evict", ctx, width, keep, sink, recent, in_place)
    t, c, wt = dev(table), dev(ctx), torch.from_numpy(w).to("cuda")
    more = dict(table_out=t, ctx_out=c, weight_out=wt) if in_place else {}
    got = lk.local_kv_evict(t, c, wt, dev(keep), dev(tags), dev(version), sink_blocks=sink,
                            recent_blocks=recent, **more)
    ctx_ref = np.minimum(ctx, BS * width) if (ctx > BS * width).all() else ctx
    want = kv4.evict(table, ctx_ref, w, keep, tags, version, sink, recent)
    for name, x, y in zip(("table", "ctx", "weight", "evicted", "n"), got, want):
        assert np.array_equal(x.cpu().numpy(), y, equal_nan=name == "weight"), name
    if not in_place:
        assert torch.equal(t, dev(table)) and torch.equal(c, dev(ctx))


def test_evict_replayed_in_place():
    """Captured and replayed on new rows: each replay acts on what the buffers hold."""
    table, ctx, w, keep, tags, version = evict_case(3, [800, 500, 16], 60, [10, 20, 5])
    t, c, wt = dev(table), dev(ctx), torch.from_numpy(w).to("cuda")
    call = lk.prepare_kv_evict(t, c, wt, dev(keep), dev(tags), dev(version), table_out=t, ctx_out=c,
                               weight_out=wt)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for r in range(3):
            t.copy_(dev(table)), c.copy_(dev(ctx))
            wt.copy_(torch.from_numpy(w).to("cuda") * (r + 1))
            g.replay()
            s.synchronize()
            want = kv4.evict(table, ctx, w * np.float32(r + 1), keep, tags, version, 1, 2)
            for x, y in zip(call.outputs, want):
                assert np.array_equal(x.cpu().numpy(), y, equal_nan=True)


@pytest.mark.parametrize("D,hq,hkv", [(128, 8, 2), (64, 4, 4)])
def test_a_context_that_is_rounded_decoded_evicted_and_continued(D, hq, hkv):
    """A bf16 pool put into 4 bits, decode steps that append and add up weights, an eviction,
    further steps on what is left and a prefill chunk behind it, each against the definition
    on the same state."""
    rng = np.random.default_rng(D)
    ctx = np.array([150, 400, 31], np.int32)
    width = 40
    nb = (ctx + 20 + 40 + BS - 1) // BS + 1
    num = int(nb.sum())
    ids = rng.permutation(num).astype(np.int32)
    table = np.full((3, width), -1, np.int32)
    at = 0
    for b in range(3):
        table[b, :nb[b]] = ids[at:at + nb[b]]
        at += nb[b]
    tags, version = np.zeros(num, np.int32), np.array([4, 5, 6], np.int32)
    for b in range(3):
        tags[table[b, :nb[b]]] = version[b]
    tags[table[1, 3]] = 1  # stale
    kd, vd = (f32_to_bf16_bits(rng.standard_normal((num, hkv, BS, D))) for _ in range(2))
    K, V = (dev_u16(x).view(num, hkv, BS * D) for x in dense_to_pool(kd, vd))
    pool = lk.local_kv4_pool_import(K, V)
    tiles = kv4.pack(bits_to_f64(kd), bits_to_f64(vd))
    assert np.array_equal(pool.cpu().numpy(), tiles)
    sm = 1.0 / math.sqrt(D)
    t, c, w = dev(table), dev(ctx), torch.zeros((3, width), device="cuda")
    meta = (dev(tags), dev(version))
    ref_w = np.zeros((3, width))

    def step():
        nonlocal ctx, ref_w
        ctx = ctx + 1
        c.copy_(dev(ctx))
        q, kn, vn = (f32_to_bf16_bits(rng.standard_normal((3, h, D))) for h in (hq, hkv, hkv))
        out, lse, _ = lk.local_paged_attn_decode_kv4(
            dev_u16(q), pool, t, c, *meta, sm, k_new=dev_u16(kn), v_new=dev_u16(vn), weight_in=w,
            weight_out=w, weight_decay=0.9)
        kv4.write(tiles, bits_to_f64(kn), bits_to_f64(vn), table[np.arange(3), (ctx - 1) // BS],
                  (ctx - 1) % BS)
        assert np.array_equal(pool.cpu().numpy(), tiles)
        ref, ref_lse, size, more = kv4.attention(bits_to_f64(q), np.arange(4), ctx, table, tags,
                                                 version, *kv4.unpack(tiles), sm)
        check_out(out, lse, ref, ref_lse, size, "step")
        ref_w = 0.9 * ref_w + more
        check_weight(w, ref_w, "weights")

    for _ in range(5):
        step()
    keep = np.array([5, 12, 9], np.int32)
    before = w.cpu().numpy()
    want = kv4.evict(table, ctx, before, keep, tags, version, 1, 2)
    got = lk.local_kv_evict(t, c, w, dev(keep), *meta, table_out=t, ctx_out=c, weight_out=w)
    for x, y in zip(got, want):
        assert np.array_equal(x.cpu().numpy(), y)
    assert want[4].tolist() == [5, 14, 0]
    assert table[1, 3] in want[3][1]  # the stale block went
    table, ctx, ref_w = want[0].copy(), want[1].copy(), want[2].astype(np.float64)
    # the freed blocks serve the rows' growth again
    for b in range(3):
        free = want[3][b, :want[4][b]] if want[4][b] else ids[at - 1 - b:at - b]
        n = (ctx[b] + BS - 1) // BS
        if want[4][b]:
            table[b, n:n + 4] = free[-4:]
            tags[table[b, n:n + 4]] = version[b]
        else:
            n0 = int(nb[:b].sum())
            table[b, :nb[b]] = ids[n0:n0 + nb[b]]
    t.copy_(dev(table))
    meta = (dev(tags), dev(version))
    for _ in range(3):
        step()
    chunk = np.array([20, 33, 1])
    ctx = (ctx + chunk).astype(np.int32)
    starts = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
    q, kn, vn = (f32_to_bf16_bits(rng.standard_normal((54, h, D))) for h in (hq, hkv, hkv))
    out, lse = lk.local_paged_attn_prefill_kv4(dev_u16(q), dev(starts), pool, t, dev(ctx), *meta,
                                               sm, k_new=dev_u16(kn), v_new=dev_u16(vn))
    for b in range(3):
        pos = np.arange(ctx[b] - chunk[b], ctx[b])
        kv4.write(tiles, bits_to_f64(kn[starts[b]:starts[b + 1]]),
                  bits_to_f64(vn[starts[b]:starts[b + 1]]), table[b, pos // BS], pos % BS)
    assert np.array_equal(pool.cpu().numpy(), tiles)
    ref, ref_lse, size, _ = kv4.attention(bits_to_f64(q), starts, ctx, table, tags, version,
                                          *kv4.unpack(tiles), sm)
    check_out(out, lse, ref, ref_lse, size, "prefill")


@pytest.mark.parametrize("four_bit", [True, False])
def test_step_with_weights(four_bit):
    """Two chained decode layers through Step, over a 4-bit pool and a bf16 one: each
    layer's attention against the definition on the step's own q, k and v, the weights of
    both layers in one array, the version check beside, replayed from a graph."""
    from paper_2608_15241_amd.step import Step, StepMeta
    rng = np.random.default_rng(9)
    B, hq, hkv, D, H, layers = 3, 4, 2, 64, 256, 2
    ctx = np.array([70, 33, 200], np.int32)
    table, num = make_table(rng, ctx, extra_blocks=1, max_blocks=16)
    tags, version = np.full(num, 8, np.int32), np.full(B, 8, np.int32)
    tags[table[2, 4]] = 7
    kd, vd = (f32_to_bf16_bits(rng.standard_normal((layers, num, hkv, BS, D))) for _ in range(2))
    bf = lambda *s, std=1.0: dev_u16(f32_to_bf16_bits(rng.standard_normal(s) * std))  # noqa: E731
    weights = [{"W_q": bf(hq * D, H, std=0.05), "W_k": bf(hkv * D, H, std=0.05),
                "W_v": bf(hkv * D, H, std=0.05), "W_o": bf(H, hq * D, std=0.05)}
               for _ in range(layers)]
    pool = torch.stack([torch.stack([dev_u16(x).view(num, hkv, BS * D)
                                     for x in dense_to_pool(kd[l], vd[l])])
                        for l in range(layers)])
    if four_bit:
        pool = torch.stack([lk.local_kv4_pool_import(pool[l, 0], pool[l, 1])
                            for l in range(layers)])
    meta = StepMeta(block_table=dev(table), ctx_lens=dev(ctx), block_version=dev(tags),
                    req_version=dev(version), q_indptr=dev(np.arange(B + 1)),
                    token_adapter=dev(np.full(B, -1)),
                    token_scale=torch.zeros(B, device="cuda"), T=B, B=B)
    w = torch.ones((B, 16), device="cuda")
    step = Step("decode", bf(B, H), weights, meta, pool, hq, hkv, D, residual=False,
                block_weight=w, weight_decay=0.5)
    step()
    first = w.clone()
    total = np.where(np.arange(16) < ((ctx + 15) // 16)[:, None], 0.5, 0.0)
    at = (table[np.arange(B), (ctx - 1) // BS], (ctx - 1) % BS)
    for l in range(layers):
        buf = step.buffers[l]
        kn, vn = (f64(buf[n]).reshape(B, hkv, D) for n in "kv")
        if four_bit:
            tiles = kv4.write(kv4.pack(bits_to_f64(kd[l]), bits_to_f64(vd[l])), kn, vn, *at)
            assert np.array_equal(pool[l].cpu().numpy(), tiles)
            k, v = kv4.unpack(tiles)
        else:
            k, v = bits_to_f64(kd[l]), bits_to_f64(vd[l])
            k[at[0], :, at[1]], v[at[0], :, at[1]] = kn, vn
        ref, ref_lse, size, more = kv4.attention(f64(buf["q"]).reshape(B, hq, D), np.arange(B + 1),
                                                 ctx, table, tags, version, k, v,
                                                 1.0 / math.sqrt(D))
        check_out(buf["o"].view(B, hq, D), buf["lse"], ref, ref_lse, size, "layer %d" % l)
        total = total + more
    check_weight(first, total, "weights")
    assert int(step.version_outputs[1]) == 1
    assert step.version_outputs[0][0].tolist() == [2, 4]
    out = step.out.clone()
    g = step.capture()
    for r in range(3):
        w.fill_(1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(step.out, out) and torch.equal(w, first)
    with pytest.raises(ValueError):
        Step("prefill", bf(B, H), weights, meta, pool, hq, hkv, D, residual=False, block_weight=w)


def test_prefill_step_over_the_4_bit_pool():
    """A chunked-prefill step whose projections feed the 4-bit append and attention."""
    from paper_2608_15241_amd.step import Step, StepMeta
    rng = np.random.default_rng(10)
    chunk, prefix, hq, hkv, D, H = np.array([40, 7]), np.array([25, 90]), 8, 2, 128, 256
    ctx = (chunk + prefix).astype(np.int32)
    table, num = make_table(rng, ctx)
    tags, version = np.full(num, 1, np.int32), np.ones(2, np.int32)
    starts = np.concatenate([[0], np.cumsum(chunk)])
    tiles = kv4.pack(*rng.standard_normal((2, num, hkv, BS, D)))
    pool = torch.from_numpy(tiles[None].copy()).to("cuda")
    bf = lambda *s, std=1.0: dev_u16(f32_to_bf16_bits(rng.standard_normal(s) * std))  # noqa: E731
    weights = [{"W_q": bf(hq * D, H, std=0.05), "W_k": bf(hkv * D, H, std=0.05),
                "W_v": bf(hkv * D, H, std=0.05), "W_o": bf(H, hq * D, std=0.05)}]
    T = int(chunk.sum())
    meta = StepMeta(block_table=dev(table), ctx_lens=dev(ctx), block_version=dev(tags),
                    req_version=dev(version), q_indptr=dev(starts),
                    token_adapter=dev(np.full(T, -1)), token_scale=torch.zeros(T, device="cuda"),
                    T=T, B=2)
    step = Step("prefill", bf(T, H), weights, meta, pool, hq, hkv, D, residual=False)
    step()
    buf = step.buffers[0]
    row = np.repeat(np.arange(2), chunk)
    pos = np.concatenate([np.arange(p, p + n) for p, n in zip(prefix, chunk)])
    kv4.write(tiles, *(f64(buf[n]).reshape(T, hkv, D) for n in "kv"), table[row, pos // BS],
              pos % BS)
    assert np.array_equal(pool[0].cpu().numpy(), tiles)
    ref, ref_lse, size, _ = kv4.attention(f64(buf["q"]).reshape(T, hq, D), starts, ctx, table, tags,
                                          version, *kv4.unpack(tiles), 1.0 / math.sqrt(D))
    check_out(buf["o"].view(T, hq, D), buf["lse"], ref, ref_lse, size, "out")
    assert int(step.version_outputs[1]) == 0

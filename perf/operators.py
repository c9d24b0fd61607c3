"""Timed cases of the 4-bit KV pool and of block eviction by attention weight.

`listed()` holds twelve cases that stand for what a program asks of them that keeps
more context on one GPU than bf16 blocks would leave room for: the conversion of
blocks to 4 bits and back, decode and prefill attention over the 4-bit pool, decode
attention that adds up how much weight each block gets, and the eviction of the
blocks that got least. `draw(rng)` gives further cases of the same ranges. `prepare`
makes a case's inputs on the GPU from a seed, `run` does one pass (in plain torch,
or where `own` is true through the framework's calls), `work` states the bytes and
operations that one pass cannot do without, and `exact` computes the outputs in
float64.

The 4-bit pool is uint8 [num_blocks][Hkv][17*D]: per block of 16 tokens and KV head
the codes of K (8 D bytes), the codes of V (8 D bytes), the scales of K and of V (D/2
bytes each). A code is a sign and a magnitude out of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a
scale is the byte E + 127 of 2^E, shared by 32 neighbouring dims of one token. E is
the least with amax <= 6 * 2^E, at least -125 and at most 125; values are rounded to
the nearest magnitude, ties to the even code, beyond 6 to 6; a group that holds an
infinity or a NaN has scale byte 255 and codes 0 and stands for NaN.

Sizes that a case draws from are the evenly spaced quantiles of the stated range, so
that a case's work does not depend on the seed.
"""
import math
import random

import numpy as np
import torch

own = False

BS = 16  # tokens of a KV block
MAGS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ the cases

def listed():
    mha = dict(hq=32, hkv=32, d=128)
    gqa = dict(hq=32, hkv=8, d=128)
    small = dict(hq=4, hkv=4, d=64)
    return [
        # One agent's short context put into 4 bits and read back: every other block of a
        # small pool, by a list of ids.
        dict(name="pool_small_ids", kind="pool", blocks=74, listed=37, **small),
        # A whole layer's pool of grouped KV heads converted at once (512K tokens), as
        # when a server moves its cold cache into 4 bits.
        dict(name="pool_gqa_32k", kind="pool", blocks=32768, listed=0, **gqa),
        # Decode attention of four short requests, the new token appended in 4 bits; the
        # blocks that it went into are read back.
        dict(name="decode4_tiny_b4", kind="decode", bits=4, batch=4, ctx_lo=17, ctx_hi=128,
             ctx_log=False, stale=0.0, append=True, weighted=False, decay=1.0, **small),
        # Decode attention of a few long agent contexts, the weight of each block added up.
        dict(name="decode4_gqa_b5", kind="decode", bits=4, batch=5, ctx_lo=1500, ctx_hi=16384,
             ctx_log=False, stale=0.0, append=False, weighted=True, decay=0.95, **gqa),
        # Decode attention of an ordinary batch, one KV head per query head.
        dict(name="decode4_mha_b32", kind="decode", bits=4, batch=32, ctx_lo=256, ctx_hi=4096,
             ctx_log=False, stale=0.0, append=False, weighted=False, decay=1.0, **mha),
        # Decode attention of one layer of a large batch of long contexts after adapter
        # updates, a tenth of the cached blocks stale.
        dict(name="decode4_gqa_b128", kind="decode", bits=4, batch=128, ctx_lo=1024,
             ctx_hi=16384, ctx_log=False, stale=0.1, append=False, weighted=True, decay=1.0,
             **gqa),
        # Four 512-token chunks of prompts on 4-bit prefixes of 0 to 2048 tokens.
        dict(name="prefill4_4x512", kind="prefill", batch=4, chunk_lo=512, chunk_hi=512,
             prefix_lo=0, prefix_hi=2048, stale=0.0, **mha),
        # Prompts' ragged chunks with grouped KV heads, part of the cached prefix stale.
        dict(name="prefill4_gqa_ragged", kind="prefill", batch=7, chunk_lo=19, chunk_hi=411,
             prefix_lo=0, prefix_hi=3000, stale=0.05, **gqa),
        # Decode attention over a small bf16 pool with the weight of each block.
        dict(name="decode16_weighted_b3", kind="decode", bits=16, batch=3, ctx_lo=40, ctx_hi=700,
             ctx_log=False, stale=0.0, append=False, weighted=True, decay=0.9, hq=16, hkv=4,
             d=64),
        # The same of a skewed batch with grouped KV heads at 7B width.
        dict(name="decode16_weighted_gqa_b64", kind="decode", bits=16, batch=64, ctx_lo=512,
             ctx_hi=8192, ctx_log=True, stale=0.0, append=False, weighted=True, decay=1.0, **gqa),
        # Four short requests cut down to half of their blocks.
        dict(name="evict_b4", kind="evict", batch=4, ctx_lo=100, ctx_hi=1000, keep=0.5, sink=1,
             recent=2, stale=0.0),
        # A large batch of long contexts cut down to a quarter, some blocks stale.
        dict(name="evict_b128", kind="evict", batch=128, ctx_lo=1024, ctx_hi=16384, keep=0.25,
             sink=4, recent=8, stale=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["pool", "decode", "decode", "decode", "prefill", "prefill", "evict"])
    hq, hkv, d = rng.choice([(32, 32, 128), (32, 8, 128), (32, 4, 128), (16, 16, 128),
                             (16, 1, 128), (32, 8, 64), (16, 4, 64), (9, 3, 64)])
    stale = rng.choice([0.0, 0.0, 0.05, 0.1, 0.3])
    c = dict(kind=kind)
    if kind == "pool":
        blocks = _log_int(rng, 1, 32768 * 8 * 128 // (hkv * d))
        c.update(blocks=blocks, listed=rng.choice([0, max(1, blocks // 3)]))
    elif kind == "decode":
        bits = rng.choice([4, 4, 16])
        batch = _log_int(rng, 1, 128)
        most = min(16384, 2 ** 28 // (batch * hkv * d) * (2 if bits == 4 else 1))
        hi = _log_int(rng, 2, most)
        c.update(bits=bits, batch=batch, ctx_lo=rng.randint(1, max(1, hi // 4)), ctx_hi=hi,
                 ctx_log=rng.random() < 0.4, append=rng.random() < 0.4,
                 weighted=bits == 16 or rng.random() < 0.5, decay=rng.choice([1.0, 0.95, 0.5]))
    elif kind == "prefill":
        batch = _log_int(rng, 1, 8)
        hi = _log_int(rng, 1, 2048 // batch)
        c.update(batch=batch, chunk_lo=rng.randint(max(1, hi // 16), hi), chunk_hi=hi,
                 prefix_lo=0, prefix_hi=_log_int(rng, 16, 4096 if hq * d > 2048 else 8192))
    else:
        hi = _log_int(rng, 16, 16384)
        c.update(batch=_log_int(rng, 1, 128), ctx_lo=rng.randint(1, hi), ctx_hi=hi,
                 keep=rng.choice([0.1, 0.25, 0.5, 0.9]), sink=rng.randint(0, 4),
                 recent=rng.randint(1, 8))
    if kind != "pool":
        c.update(stale=stale)
    if kind != "evict":
        c.update(hq=hq, hkv=hkv, d=d)
    return c


# ------------------------------------------------------------------- the inputs

def _spread(lo, hi, n, log=False):
    """n lengths: the evenly spaced quantiles of [lo, hi]."""
    at = (np.arange(n) + 0.5) / n
    if log:
        return np.rint(np.exp(math.log(lo) + at * (math.log(hi) - math.log(lo)))).astype(np.int64)
    return np.rint(lo + at * (hi - lo)).astype(np.int64)


def _lengths(c):
    """(cached prefix, new tokens) of each request, in a fixed order."""
    n = c["batch"]
    if c["kind"] == "prefill":
        prefix = _spread(c["prefix_lo"], c["prefix_hi"], n)
        return np.random.default_rng(n).permutation(prefix), _spread(c["chunk_lo"], c["chunk_hi"],
                                                                     n, log=True)
    ctx = _spread(c["ctx_lo"], c["ctx_hi"], n, c.get("ctx_log", False))
    return ctx - 1, np.ones(n, np.int64)


class _Make:
    """Seeded values of one case."""

    def __init__(self, seed):
        self.rng = np.random.default_rng([seed, 23])
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").bfloat16()

    def i32(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to("cuda")

    def channels(self, hkv, d):
        """Spread of the dims of K: some of them are several times as large as others."""
        return torch.exp(0.5 * torch.randn((hkv, 1, d), generator=self.gen, device="cuda"))

    def kv(self, blocks, hkv, d, spread):
        """Token-major [blocks][Hkv][16][D] K and V of some blocks."""
        k, v = (torch.randn((blocks, hkv, BS, d), generator=self.gen, device="cuda")
                for _ in range(2))
        return (k * spread).bfloat16(), v.bfloat16()

    def requests(self, c):
        """Block table, tags, versions and lengths; the blocks that hold new tokens are
        never stale, the others with the stated share."""
        prefix, new = _lengths(c)
        if c["kind"] == "prefill":
            order = self.rng.permutation(len(new))
            prefix, new = prefix[order], new[order]
        else:
            prefix = self.rng.permutation(prefix)
        ctx = prefix + new
        nb = (ctx + BS - 1) // BS
        total = int(nb.sum())
        first = np.cumsum(nb) - nb
        ids = self.rng.permutation(total)
        table = np.zeros((len(ctx), int(nb.max())), np.int32)
        row = np.repeat(np.arange(len(ctx)), nb)
        at = np.arange(total) - first[row]
        table[row, at] = ids
        version = 1000 * (1 + self.rng.integers(0, 8, len(ctx)))
        tags = np.zeros(total, np.int32)
        tags[ids] = version[row]
        old = ids[at < prefix[row] // BS]
        tags[self.rng.permutation(old)[:int(round(c["stale"] * len(old)))]] -= 1
        return dict(table=self.i32(table), ctx=self.i32(ctx), tags=self.i32(tags),
                    version=self.i32(version), blocks=total, new=new, nb=nb,
                    indptr=self.i32(np.concatenate([[0], np.cumsum(new)])))


CHUNK = 1 << 25  # values of K that are made at a time


def _pool_parts(c, m, blocks):
    spread = m.channels(c["hkv"], c["d"])
    step = max(1, CHUNK // (c["hkv"] * BS * c["d"]))
    for at in range(0, blocks, step):
        n = min(step, blocks - at)
        yield slice(at, at + n), m.kv(n, c["hkv"], c["d"], spread)


def _inputs(c, seed):
    m = _Make(seed)
    s = {"case": c}
    if c["kind"] == "evict":
        s.update(m.requests(c))
        shape = tuple(s["table"].shape)
        w = torch.rand(shape, generator=m.gen, device="cuda")
        w = torch.where(w < 0.3, 0.0, torch.exp(8 * w - 8))  # some blocks never got any
        inside = torch.arange(shape[1], device="cuda") < m.i32(s["nb"])[:, None]
        s["weight"] = torch.where(inside, w, 0.0)
        s["keep"] = m.i32(np.maximum(1, (c["keep"] * s["nb"]).astype(np.int64)))
        return s
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "pool":
        s["blocks"] = c["blocks"]
        s["ids"] = m.i32(m.rng.permutation(c["blocks"])[:c["listed"]]) if c["listed"] else None
        s["K"], s["V"] = (torch.empty((c["blocks"], hkv, BS * d), dtype=torch.bfloat16,
                                      device="cuda") for _ in range(2))
        for at, (k, v) in _pool_parts(c, m, c["blocks"]):
            s["K"][at], s["V"][at] = _to_layout(k, v)
        return s
    s.update(m.requests(c))
    rows = int(s["new"].sum())
    s["q"] = m.normal(rows, hq, d)
    if c["kind"] == "prefill" or c["append"]:
        s["k_new"], s["v_new"] = m.normal(rows, hkv, d), m.normal(rows, hkv, d)
    if c.get("bits", 4) == 4:
        s["kv4"] = torch.empty((s["blocks"], hkv, 17 * d), dtype=torch.uint8, device="cuda")
        for at, (k, v) in _pool_parts(c, m, s["blocks"]):
            s["kv4"][at] = _pack(k, v)
    else:
        s["K"], s["V"] = (torch.empty((s["blocks"], hkv, BS * d), dtype=torch.bfloat16,
                                      device="cuda") for _ in range(2))
        for at, (k, v) in _pool_parts(c, m, s["blocks"]):
            s["K"][at], s["V"][at] = _to_layout(k, v)
    if c.get("weighted"):
        w = torch.rand(tuple(s["table"].shape), generator=m.gen, device="cuda") * 4
        inside = torch.arange(w.shape[1], device="cuda") < m.i32(s["nb"])[:, None]
        s["weight"] = torch.where(inside, w, 0.0)
    if "k_new" in s:  # the blocks that receive new tokens
        row = np.repeat(np.arange(c["batch"]), s["new"])
        pos = np.concatenate([np.arange(n) for n in s["new"]])
        pos += (s["ctx"].cpu().numpy().astype(np.int64) - s["new"])[row]
        s["touched"] = torch.unique(s["table"][torch.from_numpy(row), torch.from_numpy(pos // BS)])
        s["row"], s["pos"] = torch.from_numpy(row).to("cuda"), torch.from_numpy(pos).to("cuda")
        if "kv4" in s:
            s["Kt"], s["Vt"] = (torch.zeros((s["blocks"], hkv, BS * d), dtype=torch.bfloat16,
                                            device="cuda") for _ in range(2))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the prepared calls that a program keeps
        s["calls"] = _own_calls(case, s)
    return s


# ----------------------------------------------------------- the framework's calls

def _own_calls(c, s):
    import paper_2608_15241_amd as local

    if c["kind"] == "pool":
        hkv, d = c["hkv"], c["d"]
        kv4 = torch.zeros((c["blocks"], hkv, 17 * d), dtype=torch.uint8, device="cuda")
        K, V = (torch.zeros((c["blocks"], hkv, BS * d), dtype=torch.bfloat16, device="cuda")
                for _ in range(2))
        return [local.prepare_kv4_pool_import(s["K"], s["V"], kv4, block_ids=s["ids"]),
                local.prepare_kv4_pool_export(kv4, K, V, block_ids=s["ids"])]
    meta = (s["table"], s["ctx"], s["tags"], s["version"])
    if c["kind"] == "evict":
        return [local.prepare_kv_evict(s["table"], s["ctx"], s["weight"], s["keep"], s["tags"],
                                       s["version"], sink_blocks=c["sink"],
                                       recent_blocks=c["recent"])]
    sm = 1.0 / math.sqrt(c["d"])
    new = dict(k_new=s.get("k_new"), v_new=s.get("v_new"))
    weights = dict(weight_in=s["weight"], weight_decay=c["decay"]) if c.get("weighted") else {}
    if c["kind"] == "prefill":
        calls = [local.prepare_paged_attn_prefill_kv4(s["q"], s["indptr"], s["kv4"], *meta, sm,
                                                      **new)]
    elif c["bits"] == 4:
        if weights:
            weights["weight_out"] = torch.empty_like(s["weight"])
        calls = [local.prepare_paged_attn_decode_kv4(s["q"], s["kv4"], *meta, sm, **new,
                                                     **weights)]
    else:
        calls = [local.prepare_paged_attn_decode_weighted(
            s["q"], s["K"], s["V"], *meta, sm, Hkv=c["hkv"], **new, **weights)]
    if "Kt" in s:
        calls.append(local.prepare_kv4_pool_export(s["kv4"], s["Kt"], s["Vt"],
                                                   block_ids=s["touched"]))
    return calls


def run(state):
    s, c = state, state["case"]
    if own:
        outs = [call() for call in s["calls"]]
        if c["kind"] == "pool":
            return {"values": outs[1]}
        if c["kind"] == "evict":
            return outs[0]
        return _state_of(c, s, {"attn": outs[0]}, outs[-1])
    return _plain(c, s)


def _state_of(c, s, got, touched):
    """The outputs with the state that the call changed: the blocks of a 4-bit pool that
    received tokens, as values, or the bf16 pool."""
    if "Kt" in s:
        got["appended"] = touched
    elif "k_new" in s:
        got["pool"] = (s["K"], s["V"])
    return got


# ---------------------------------------------------------------- the plain forms

def _to_layout(k, v):
    """Token-major [n][Hkv][16][D] -> the bf16 pool's K and V layouts [n][Hkv][16*D]."""
    n, h, _, d = k.shape
    return (k.view(n, h, BS, d // 8, 8).transpose(2, 3).reshape(n, h, -1),
            v.transpose(2, 3).reshape(n, h, -1))


def _from_layout(k, v, d):
    n, h = k.shape[:2]
    return (k.view(n, h, d // 8, BS, 8).transpose(2, 3).reshape(n, h, BS, d),
            v.view(n, h, d, BS).transpose(2, 3))


def _quantise(x):
    """(codes, scale bytes) of [..., D] values: uint8 [..., D] and [..., D/32]."""
    g = x.float().view(x.shape[:-1] + (x.shape[-1] // 32, 32))
    amax = g.abs().amax(-1, keepdim=True)
    fine = amax < math.inf
    f, e = torch.frexp(torch.where(fine, amax, 1.0))  # amax = f * 2^e with 0.5 <= f < 1
    e = torch.where(f > 0.75, e - 2, e - 3).clamp(-125, 125)
    e = torch.where(amax == 0, -125, e)
    y = torch.ldexp(torch.where(fine, g, 0.0), -e)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5))
    code += torch.signbit(y).to(torch.uint8) << 3
    scale = torch.where(fine, e + 127, 255).to(torch.uint8).squeeze(-1)
    return code.view(x.shape), scale


def _pack(k, v):
    """Token-major K and V [n][Hkv][16][D] -> 4-bit tiles [n][Hkv][17*D]."""
    n, h, _, d = k.shape
    ck, sk = _quantise(k)
    cv, sv = _quantise(v)
    ck, cv = (t[..., 0::2] | (t[..., 1::2] << 4) for t in (ck, cv))  # [n][h][16][D/2]
    ck = ck.view(n, h, BS, 4, d // 8).transpose(2, 3).reshape(n, h, -1)
    cv = cv.view(n, h, 4, 4, 16, d // 32).transpose(3, 4).reshape(n, h, -1)
    sk = sk.transpose(2, 3).reshape(n, h, -1)
    sv = sv.view(n, h, 4, 4, d // 32).transpose(3, 4).reshape(n, h, -1)
    return torch.cat([ck, cv, sk, sv], -1)


def _codes(c):
    """Values of packed codes [..., n] -> float32 [..., 2 n]."""
    table = torch.tensor(MAGS + tuple(-m for m in MAGS), device=c.device)
    both = torch.stack([table.repeat(16), table.repeat_interleave(16)], -1)  # per byte: low, high
    return both[c.int()].flatten(-2)


def _unpack(t, d):
    """4-bit tiles [n][Hkv][17*D] -> token-major float32 K and V [n][Hkv][16][D]."""
    n, h = t.shape[:2]
    ck = t[..., :8 * d].view(n, h, 4, BS, d // 8).transpose(2, 3).reshape(n, h, BS, d // 2)
    cv = t[..., 8 * d:16 * d].view(n, h, 4, 16, 4, d // 32).transpose(3, 4)
    cv = cv.reshape(n, h, BS, d // 2)
    s = torch.ldexp(torch.ones((), device=t.device), t[..., 16 * d:].int() - 127)
    s = torch.where(t[..., 16 * d:] == 255, math.nan, s)
    sk = s[..., :d // 2].view(n, h, d // 32, BS).transpose(2, 3)
    sv = s[..., d // 2:].view(n, h, 4, d // 32, 4).transpose(3, 4).reshape(n, h, BS, d // 32)
    k, v = ((_codes(c).view(n, h, BS, d // 32, 32) * x[..., None]).view(n, h, BS, d)
            for c, x in ((ck, sk), (cv, sv)))
    return k, v


def _plain(c, s):
    if c["kind"] == "pool":
        return {"values": _plain_pool(c, s)}
    if c["kind"] == "evict":
        return _plain_evict(c, s)
    if "k_new" in s:
        _plain_append(c, s)
    got = {"attn": _plain_attention(c, s)}
    touched = None
    if "Kt" in s:
        ids = s["touched"].long()
        k, v = _unpack(s["kv4"][ids], c["d"])
        s["Kt"][ids], s["Vt"][ids] = _to_layout(k.bfloat16(), v.bfloat16())
        touched = (s["Kt"], s["Vt"])
    return _state_of(c, s, got, touched)


def _plain_pool(c, s):
    """The listed blocks rounded to 4 bits and back; the others are zero."""
    d, ids = c["d"], None if s["ids"] is None else s["ids"].long()
    k, v = _from_layout(s["K"] if ids is None else s["K"][ids],
                        s["V"] if ids is None else s["V"][ids], d)
    k, v = _unpack(_pack(k, v), d)
    k, v = _to_layout(k.bfloat16(), v.bfloat16())
    if ids is None:
        return k, v
    K, V = torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
    K[ids], V[ids] = k, v
    return K, V


def _plain_append(c, s):
    """Writes the new tokens at their positions."""
    hkv, d = c["hkv"], c["d"]
    blk, slot = s["table"][s["row"], s["pos"] // BS].long(), s["pos"] % BS
    heads = torch.arange(hkv, device="cuda")[None, :, None]
    if "kv4" not in s:
        n = s["blocks"]
        s["K"].view(n, hkv, d // 8, BS, 8)[blk, :, :, slot] = s["k_new"].view(-1, hkv, d // 8, 8)
        s["V"].view(n, hkv, d, BS)[blk, :, :, slot] = s["v_new"]
        return
    ck, sk = _quantise(s["k_new"])
    cv, sv = _quantise(s["v_new"])
    ck, cv = (t[..., 0::2] | (t[..., 1::2] << 4) for t in (ck, cv))  # [T][Hkv][D/2]
    slot = slot[:, None, None]
    i, g = torch.arange(d // 2, device="cuda"), torch.arange(d // 32, device="cuda")
    at = (blk[:, None, None], heads)
    s["kv4"][at + ((i // (d // 8) * BS + slot) * (d // 8) + i % (d // 8),)] = ck
    s["kv4"][at + (8 * d + ((slot // 4 * 16 + i // (d // 32)) * 4 + slot % 4) * (d // 32)
                   + i % (d // 32),)] = cv
    s["kv4"][at + (16 * d + g * BS + slot,)] = sk
    s["kv4"][at + (16 * d + d // 2 + (slot // 4 * (d // 32) + g) * 4 + slot % 4,)] = sv


def _plain_attention(c, s):
    """Every request padded to the longest: [B][Hkv][new * group][keys] in float32."""
    hq, hkv, d, b = c["hq"], c["hkv"], c["d"], c["batch"]
    group, width = hq // hkv, s["table"].shape[1]
    new = int(s["new"].max())
    starts, ctx = s["indptr"].long(), s["ctx"].long()
    table = s["table"].long()
    owned = torch.arange(width, device="cuda") < ((ctx + BS - 1) // BS)[:, None]
    table = torch.where(owned, table, 0)
    ok = (owned & (s["tags"][table] == s["version"][:, None])).repeat_interleave(BS, 1)
    at = torch.arange(width * BS, device="cuda")
    if "kv4" in s:
        k, v = _unpack(s["kv4"][table.view(-1)], d)
    else:
        k, v = _from_layout(s["K"][table.view(-1)], s["V"][table.view(-1)], d)
    rows = torch.arange(new, device="cuda")
    pos = ctx[:, None] - (starts[1:] - starts[:-1])[:, None] + rows  # [B][new]
    see = ok[:, None] & (at <= pos[..., None])  # [B][new][keys]
    inside = (at < ctx[:, None])[:, None, :, None] & ok[:, None, :, None]
    k, v = (t.view(b, width, hkv, BS, d).transpose(1, 2).reshape(b, hkv, width * BS, d).float()
            for t in (k, v))
    k, v = torch.where(inside, k, 0.0), torch.where(inside, v, 0.0)
    live = rows < (starts[1:] - starts[:-1])[:, None]
    take = torch.where(live, starts[:-1, None] + rows, 0)
    q = s["q"][take].float().view(b, new, hkv, group, d).transpose(1, 2)
    q = q.reshape(b, hkv, new * group, d)
    p = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    p = p.view(b, hkv, new, group, -1).masked_fill(~see[:, None, :, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(p - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).squeeze(-1)  # [B][Hkv][new][group]
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p.view(b, hkv, new * group, -1), v).view(b, hkv, new, group, d)
    out = torch.empty_like(s["q"])
    out[take[live]] = o.permute(0, 2, 1, 3, 4).reshape(b, new, hq, d)[live].to(out.dtype)
    full = torch.empty(s["q"].shape[:2], device="cuda")
    full[take[live]] = lse.permute(0, 2, 1, 3).reshape(b, new, hq)[live]
    if not c.get("weighted"):
        return out, full
    w = p.sum((1, 2, 3)).view(b, width, BS).sum(-1)
    return out, full, torch.where(owned, c["decay"] * s["weight"] + w, 0.0)


def _plain_evict(c, s):
    table, ctx, weight = s["table"], s["ctx"].long(), s["weight"]
    width = table.shape[1]
    j = torch.arange(width, device="cuda")
    nb = ((ctx + BS - 1) // BS)[:, None]
    owned = j < nb
    stale = s["tags"][torch.where(owned, table, 0).long()] != s["version"][:, None]
    held = (j < c["sink"]) | (j >= nb - c["recent"])
    kept_n = torch.maximum(s["keep"].long()[:, None], (held & owned).sum(1, keepdim=True))
    kept_n = torch.minimum(kept_n, nb)
    # rank: protected blocks, the others by weight, stale ones, none
    key = torch.where(stale, -1.0, torch.where(weight > 0, weight, 0.0))
    key = torch.where(held, math.inf, key)
    key = torch.where(owned, key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    kept = torch.zeros_like(owned)
    kept.scatter_(1, order, j < kept_n)
    gone = owned & ~kept
    to_front = torch.sort((~kept).int(), dim=1, stable=True).indices
    first = j < kept_n
    table_out = torch.where(first, table.gather(1, to_front), -1)
    weight_out = torch.where(first, weight.gather(1, to_front), 0.0)
    lost = nb - kept_n
    gone_first = torch.sort((~gone).int(), dim=1, stable=True).indices
    evicted = torch.where(j < lost, table.gather(1, gone_first), -1)
    ctx_out = (ctx - BS * lost[:, 0]).int()
    return table_out, ctx_out, weight_out, evicted, lost[:, 0].int()


# ---------------------------------------------------------- what a pass must do

def work(case):
    c = case
    if c["kind"] == "pool":
        n = float((c["listed"] or c["blocks"]) * c["hkv"] * BS * c["d"] * 2)
        return {"bytes": n * (2 + 2 * 17 / 32 + 2), "flops": 4 * n}
    prefix, new = _lengths(c)
    ctx = prefix + new
    nb = (ctx + BS - 1) // BS
    if c["kind"] == "evict":
        n, blocks = float(c["batch"]), float(c["batch"] * nb.max())
        # ids, weights and tags of the owned blocks, lengths; three full rows of outputs
        return {"bytes": 12.0 * float(nb.sum()) + 12.0 * n + 12.0 * blocks + 8.0 * n,
                "flops": 0.0}
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    rows = float(new.sum())
    held = float((prefix // BS * BS * (1 - c["stale"]) + prefix % BS + new).sum())
    fresh = c["kind"] == "prefill" or c["append"]
    per_token = d * 17 / 16 if c.get("bits", 4) == 4 else 4.0 * d  # K and V of one head
    by = held * hkv * per_token + rows * hq * (4 * d + 4) + 8.0 * float(nb.sum())
    if fresh:  # new tokens read, and read back from the blocks that they went into
        by += rows * hkv * (4 * d + per_token)
        if c.get("bits", 4) == 4:
            touched = float((nb - prefix // BS).sum()) * BS
            by += touched * hkv * (per_token + 4 * d)
    if c.get("weighted"):
        by += 8.0 * c["batch"] * float(nb.max())
    pairs = float((new * prefix * (1 - c["stale"]) + new * (new + 1) / 2).sum())
    return {"bytes": by, "flops": 4.0 * pairs * hq * d}


# --------------------------------------------------------------- the same in 64 bits

def _q64(x):
    """[..., D] values rounded to 4 bits and back, in float64: the nearest of the eight
    magnitudes, found by their distances."""
    x = x.double()
    g = x.reshape(x.shape[:-1] + (-1, 32))
    amax = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / 6) - 1e-12)
    e = torch.where(amax > 0, e, -125.0).clamp(-125, 125)
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), e)
    mags = torch.tensor(MAGS, dtype=torch.float64, device=x.device)
    odd = 1e-9 * (torch.arange(8, device=x.device) % 2)  # ties go to the even code
    y = (g / scale).abs()
    best, near = torch.full_like(y, math.inf), torch.zeros_like(y)
    for m, o in zip(mags, odd):
        far = (y - m).abs() + o
        near = torch.where(far < best, m, near)
        best = torch.minimum(best, far)
    return (torch.copysign(near, g) * scale).reshape(x.shape)


def _kv64(tiles, d):
    """4-bit tiles [n][Hkv][17*D] -> [n * 16][Hkv][D] float64 K and V, by each value's
    place in its tile."""
    dev = tiles.device
    tok, dim = torch.arange(BS, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    places = (((dim // (d // 4)) * 16 + tok) * (d // 8) + dim % (d // 4) // 2,
              8 * d + (((tok // 4) * 16 + dim // (d // 16)) * 4 + tok % 4) * (d // 32)
              + dim % (d // 16) // 2)
    scales = (16 * d + dim // 32 * 16 + tok,
              16 * d + d // 2 + (tok // 4 * (d // 32) + dim // 32) * 4 + tok % 4)
    mags = torch.tensor(MAGS, dtype=torch.float64, device=dev)
    both = []
    for at, sc in zip(places, scales):
        code = tiles[:, :, at.reshape(-1)].long() >> (4 * (dim % 2)).expand(BS, d).reshape(-1)
        value = mags[code & 7] * (1 - 2 * (code >> 3 & 1)).double()
        value = value * torch.exp2(tiles[:, :, sc.reshape(-1)].double() - 127)
        both.append(value.view(-1, tiles.shape[1], BS, d).transpose(1, 2).flatten(0, 1))
    return both


def _bf64(k, v, d):
    n, h = k.shape[:2]
    return (k.view(n, h, d // 8, BS, 8).permute(0, 3, 1, 2, 4).reshape(n * BS, h, d).double(),
            v.view(n, h, d, BS).permute(0, 3, 1, 2).reshape(n * BS, h, d).double())


def _exact_attention(c, s):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    group = hq // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    weight = torch.zeros(s["table"].shape, dtype=torch.float64, device="cuda")
    four = "kv4" in s
    touched = {}
    start = 0
    for b in range(c["batch"]):
        n, new = int(s["ctx"][b]), int(s["new"][b])
        nb = (n + BS - 1) // BS
        ids = s["table"][b, :nb].long()
        k, v = _kv64(s["kv4"][ids], d) if four else _bf64(s["K"][ids], s["V"][ids], d)
        rows = slice(start, start + new)
        start += new
        if "k_new" in s:
            k[n - new:n] = _q64(s["k_new"][rows]) if four else s["k_new"][rows].double()
            v[n - new:n] = _q64(s["v_new"][rows]) if four else s["v_new"][rows].double()
            for j in range((n - new) // BS, nb):
                touched[int(ids[j])] = (k[j * BS:(j + 1) * BS].clone(),
                                        v[j * BS:(j + 1) * BS].clone())
        fine = (s["tags"][ids] == s["version"][b]).repeat_interleave(BS)[:n]
        at = fine.nonzero().view(-1)
        k, v = (t[at].transpose(0, 1).contiguous() for t in (k, v))  # [Hkv][keys][D]
        q = s["q"][rows].double().view(new, hkv, group, d).permute(1, 0, 2, 3)
        q = q.reshape(hkv, new * group, d).contiguous()
        p = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        hide = at[None, :] > torch.arange(n - new, n, device="cuda")[:, None]
        p = p.view(hkv, new, group, -1).masked_fill(hide[None, :, None], -math.inf)
        l = torch.logsumexp(p, -1)
        lse[rows] = l.transpose(0, 1).reshape(new, hq)
        p = torch.exp(p - torch.where(l == -math.inf, 0.0, l)[..., None])
        if "weight" in s:
            weight[b].index_add_(0, at // BS, p.sum((0, 1, 2)))
            weight[b, :nb] += c["decay"] * s["weight"][b, :nb].double()
        o = torch.bmm(p.view(hkv, new * group, -1), v).view(hkv, new, group, d)
        out[rows] = o.transpose(0, 1).reshape(new, hq, d)
    got = {"attn": (out, lse, weight) if "weight" in s else (out, lse)}
    if "k_new" in s:
        K, V = ((torch.zeros_like(s["Kt"]), torch.zeros_like(s["Vt"])) if four
                else (s["K"].clone(), s["V"].clone()))
        for p, (k, v) in touched.items():
            K[p] = k.view(BS, hkv, d // 8, 8).permute(1, 2, 0, 3).reshape(hkv, -1).to(K.dtype)
            V[p] = v.permute(1, 2, 0).reshape(hkv, -1).to(V.dtype)
        got["appended" if four else "pool"] = (K, V)
    return got


def _exact_evict(c, s):
    table, ctx = s["table"].cpu().numpy(), s["ctx"].cpu().numpy()
    weight, tags = s["weight"].cpu().numpy(), s["tags"].cpu().numpy()
    version, keep = s["version"].cpu().numpy(), s["keep"].cpu().numpy()
    t_out, e_out = np.full_like(table, -1), np.full_like(table, -1)
    w_out, c_out = np.zeros(weight.shape), ctx.copy()
    lost = np.zeros(len(ctx), np.int32)
    for b, n in enumerate(ctx):
        nb = -(-int(n) // BS)
        safe = [j for j in range(nb) if j < c["sink"] or j >= nb - c["recent"]]
        rest = sorted((j for j in range(nb) if c["sink"] <= j < nb - c["recent"]),
                      key=lambda j: (bool(tags[table[b, j]] != version[b]), -weight[b, j], j))
        kept = sorted(safe + rest[:max(0, int(keep[b]) - len(safe))])
        gone = sorted(set(range(nb)) - set(kept))
        t_out[b, :len(kept)], w_out[b, :len(kept)] = table[b, kept], weight[b, kept]
        e_out[b, :len(gone)], lost[b] = table[b, gone], len(gone)
        c_out[b] = n - BS * len(gone)
    return tuple(torch.from_numpy(x) for x in (t_out, c_out, w_out, e_out, lost))


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "evict":
        return _exact_evict(c, s)
    if c["kind"] != "pool":
        return _exact_attention(c, s)
    K, V = torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
    k, v = _bf64(s["K"], s["V"], c["d"])
    k, v = (_q64(t).view(-1, BS, c["hkv"], c["d"]) for t in (k, v))
    ids = torch.arange(c["blocks"], device="cuda") if s["ids"] is None else s["ids"].long()
    K[ids] = k[ids].unflatten(-1, (-1, 8)).permute(0, 2, 3, 1, 4).flatten(2).to(K.dtype)
    V[ids] = v[ids].permute(0, 2, 3, 1).flatten(2).to(V.dtype)
    return {"values": (K, V)}

"""Every form of 4-bit decode (partition length, waves that share one, dispatch order) against
float64: with block weights at the usual scale, without them at 0, where each key counts the
same."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest

from tests.conftest import ROOT

# (batch, Hq, Hkv, D, longest context, table width, blocks of a partition, waves, longest
# units first)
CASES = [
    (20, 64, 32, 128, 300, 256, 32, 1, True),      # eight partitions, most not there
    (40, 16, 16, 64, 1400, 256, 32, 1, True),      # ... and several of a request
    (300, 8, 8, 64, 130, 9, 32, 1, True),          # one partition, five registers of requests
    (15, 32, 32, 64, 1700, 500, 48, 1, True),
    (10, 16, 8, 128, 2000, 500, 48, 4, False),
    (3, 32, 8, 128, 5000, 17000, 64, 1, True),
    (31, 4, 4, 64, 2500, 1024, 64, 2, True),
    (8, 16, 8, 128, 2500, 1024, 64, 4, True),
    (1, 4, 1, 128, 9000, 3000, 64, 4, False),
    (700, 4, 4, 64, 200, 64, 32, 1, False),        # too many requests to rank
    (520, 2, 1, 128, 600, 57, 32, 4, False),       # ... four waves, two partitions
    (520, 8, 4, 64, 300, 40, 32, 2, False),        # ... two waves
    (40, 32, 32, 64, 200, 16, 32, 2, True),
    (20, 32, 32, 64, 200, 16, 16, 2, False),
    (2, 8208, 513, 64, 40, 4, 32, 2, True),       # more query heads than weights go with
]


def _contexts(rng, B, longest):
    ctx = rng.integers(0 if B > 2 else 1, longest + 1, size=B)
    ctx[0] = longest
    if B > 9:  # ends of partitions and of blocks
        ctx[1:8] = [min(longest, n) for n in (256, 257, 255, 512, 768, 1024, 1025)]
    return ctx


@pytest.mark.parametrize("B,Hq,Hkv,D,longest,width,blocks,waves,ranked", CASES)
def test_forms_are_the_named_ones(B, Hq, Hkv, D, longest, width, blocks, waves, ranked):
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2608_15241_amd", "liblocal.so"))
    form = lib.localk_decode_kv4_form(B, Hq, Hkv, width)
    assert (form % 256, form // 256 % 16, form // 4096) == (blocks, waves, int(ranked))


@pytest.mark.gpu
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forms(i, weighted):
    import torch
    import paper_2608_15241_amd as lk
    from tests.gpu_helpers import say
    from tests.kv4_cases import check_counts, quick_case
    from tests.kv4_helpers import check_out, check_weight
    B, hq, hkv, D, longest, width = CASES[i][:6]
    weighted = weighted and hq <= 8192
    rng = np.random.default_rng(i)
    c = quick_case(400 + i, _contexts(rng, B, longest), hq, hkv, D, width=width, stale=0.3)
    say("decode forms", i, B, hq, hkv, D, longest, width, weighted)
    q, pool, meta, new = c.gpu()
    want = c.appended()
    more = {}
    if weighted:
        w_in = c.rng.random(c.table.shape).astype(np.float32)
        more = dict(weight_in=torch.from_numpy(w_in).to("cuda"), weight_decay=0.5)
    c.sm = c.sm if weighted else 0.0
    ref, ref_lse, size, w = c.ref(want)
    got = lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm, **new, **more)
    if weighted:
        check_out(*got[:2], ref, ref_lse, size, "out")
        owned = np.arange(width) < ((c.ctx + 15) // 16)[:, None]
        check_weight(got[2], np.where(owned, w + 0.5 * w_in.astype(np.float64), 0.0), "weights")
    else:
        check_counts(*got, ref, ref_lse, "out")
    assert np.array_equal(pool.cpu().numpy(), want)

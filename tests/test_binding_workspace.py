"""Workspaces of prepared calls: one of its own where none is given, a shared one where the
caller says so."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_15241_amd as lk
from paper_2608_15241_amd import binding as bd


def _asks_for(nbytes):
    """An entry point that asks for nbytes."""
    def fn(ws, n, stream):
        if ws is None:
            n._obj.value = nbytes
        return 0
    return fn


@pytest.fixture
def on_cpu(monkeypatch):
    monkeypatch.setattr(bd, "_stream", lambda: None)


def _span(call):
    return call.ws.data_ptr(), call.ws.data_ptr() + call.ws.numel()


def test_calls_without_a_workspace_share_none(on_cpu):
    calls = [lk.Call(_asks_for(n), (), None, "cpu") for n in (4096, 100, 0, 9000, 4096)]
    spans = sorted(_span(c) for c in calls)
    assert all(c.ws_bytes.value >= n for c, n in zip(calls, (4096, 100, 0, 9000, 4096)))
    assert all(end <= start for (_, end), (start, _) in zip(spans, spans[1:]))


def test_calls_share_the_workspace_that_they_were_given(on_cpu):
    ws = lk.Workspace("cpu")
    a, b = (lk.Call(_asks_for(n), (), ws, "cpu") for n in (4096, 100))
    assert _span(a) == _span(b)


@pytest.mark.gpu
def test_calls_without_a_workspace_on_two_streams():
    """Prefill and decode calls of different requests, side by side on two streams: what each
    gives alone."""
    from tests.gpu_helpers import dev, dev_u16
    from tests.test_gpu_kv4 import Case
    sides = []
    for seed, ctx, new in ((91, [900, 2000, 130], [40, 200, 1]), (92, [4000, 70], [150, 64])):
        c = Case(seed, ctx, 16, 4, 64, new=new, stale=0.1)
        c.widen()
        q, pool, meta, new = c.gpu()
        lk.local_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm, **new)  # appends
        last = torch.from_numpy(c.starts[1:].astype(np.int64) - 1)
        sides.append([lk.prepare_paged_attn_prefill_kv4(q, dev(c.starts), pool, *meta, c.sm),
                      lk.prepare_paged_attn_decode_kv4(q[last].contiguous(), pool, *meta, c.sm)])
    want = []
    for calls in sides:
        for call in calls:
            want.append([t.clone() for t in call()])
            torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(20):
        for s, calls in zip(streams, sides):
            with torch.cuda.stream(s):
                for call in calls:
                    call()
    torch.cuda.synchronize()
    for call, w in zip([c for calls in sides for c in calls], want):
        for a, b in zip(call.outputs, w):
            assert torch.equal(a, b)

"""Workspaces of prepared calls: one of its own where none is given, a shared one where the
caller says so."""
from __future__ import annotations

import ctypes

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
    monkeypatch.setattr(bd, "_stream", lambda: ctypes.c_void_p(None))


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


def test_own_workspaces_outlive_the_work_of_other_streams(on_cpu, monkeypatch):
    """The allocator is told once of each stream, besides the first, that uses one."""
    told, capturing = [], [False]
    monkeypatch.setattr(bd, "_used_here",
                        lambda t: not capturing[0] and (told.append(t) or True))
    own = lk.Call(_asks_for(512), (), None, "cpu")
    shared = lk.Call(_asks_for(512), (), lk.Workspace("cpu"), "cpu")
    for handle, n, capture in ((None, 0, False), (7, 0, True), (7, 1, False), (7, 1, False),
                               (9, 2, False), (None, 2, False)):
        monkeypatch.setattr(bd, "_stream", lambda h=handle: ctypes.c_void_p(h))
        capturing[0] = capture
        own()
        shared()
        assert len(told) == n and all(t is own.ws for t in told)


@pytest.mark.gpu
def test_calls_without_a_workspace_on_two_streams():
    """Prefill and decode calls of different requests, side by side on two streams: what each
    gives alone."""
    from tests.gpu_helpers import dev
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


@pytest.mark.gpu
def test_a_call_dropped_while_it_runs_on_another_stream():
    """Its workspace is not handed out again before its work has run."""
    from tests.test_gpu_kv4 import Case
    c = Case(93, [4000, 70], 16, 4, 64, stale=0.1)
    q, pool, meta, _ = c.gpu()
    want = [t.clone() for t in lk.local_paged_attn_decode_kv4(q, pool, *meta, c.sm)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        call = lk.prepare_paged_attn_decode_kv4(q, pool, *meta, c.sm)
        outputs, at, n = call.outputs, call.ws.data_ptr(), call.ws.numel()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            call()
        del call
        again = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        assert again.data_ptr() != at
        torch.cuda.synchronize()
        for a, b in zip(outputs, want):
            assert torch.equal(a, b)
        del again

"""Tensors that the binding makes for a call on a stream of its own belong to that stream: their
fills and memory are in its order, not in the current stream's (CPU: the library is a recorder)."""
import contextlib

import pytest
import torch

from paper_2405_19261_amd import spc


class Handle:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


CURRENT, SIDE = Handle(0x100), Handle(0x200)


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, as (name, stream, the streams that tensors of the call were made on,
    those that the tensors are kept for)."""
    now, made, kept, done = [CURRENT], [], [], []

    class Library:
        def __getattr__(self, name):
            def call(*a):
                done.append((name, a[-1], list(made), list(kept)))
                return 0
            return call

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(spc, "lib", lambda: Library())
    monkeypatch.setattr(spc, "_on_current_device", lambda t: None)
    monkeypatch.setattr(spc, "_raw_stream", lambda: now[-1].cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *a: {0x200: SIDE}[handle])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: kept.append(s))
    for name in ("zeros", "empty", "empty_like", "zeros_like", "empty_strided"):
        def make(*a, _make=getattr(torch, name), **kw):
            made.append(now[-1])
            return _make(*a, **kw)
        monkeypatch.setattr(torch, name, make)
    made.clear()
    yield done, made


def entries():
    B, H, heads, D, S, pages = 2, 2, 4, 64, 16, 8
    k = torch.zeros((pages, H, S, D), dtype=torch.bfloat16)
    cache = (k, torch.zeros((pages, H, D, S), dtype=torch.bfloat16),
             torch.zeros((B, 2), dtype=torch.int32), torch.zeros(B, dtype=torch.int32))
    q = torch.zeros((B, 3, heads, D), dtype=torch.bfloat16)
    rows, start = q.flatten(0, 1), torch.zeros(B + 1, dtype=torch.int32)
    z, u, w = torch.zeros((B, 5, 50)), torch.zeros((B, 5)), torch.zeros((B, H, 32))
    draft, one = torch.zeros((B, 4), dtype=torch.int32), torch.zeros(B)
    table = torch.zeros((B, 1), dtype=torch.int32)
    return dict(
        spc_verify=lambda **kw: spc.spc_verify(z, z, draft, u, 0, 0.5, 1.0, **kw),
        spc_greedy_verify=lambda **kw: spc.spc_greedy_verify(z, z, draft, 0, 0.5, **kw),
        spc_draft_sample=lambda **kw: spc.spc_draft_sample(z[:, 0].contiguous(), 1.0, one, **kw),
        spc_sample=lambda **kw: spc.spc_sample(z[:, 0], one, **kw),
        spc_truncate=lambda **kw: spc.spc_truncate(z, top_k=3, **kw),
        spc_kv_read=lambda **kw: spc.spc_kv_read(*cache, 9, **kw),
        spc_kv_attend=lambda **kw: spc.spc_kv_attend(q, *cache, **kw),
        spc_kv_attend_ragged=lambda **kw: spc.spc_kv_attend(rows, *cache, q_start=start, **kw),
        spc_kv_attend_shared=lambda **kw: spc.spc_kv_attend_shared(rows, *cache, 9, q_start=start, **kw),
        spc_cross_attend=lambda **kw: spc.spc_cross_attend(rows, *cache, q_start=start, **kw),
        spc_kv_weigh=lambda **kw: spc.spc_kv_weigh(q, *cache, w, **kw),
        spc_kv_evict=lambda **kw: spc.spc_kv_evict(*cache, w, 8, table, **kw))


@pytest.mark.parametrize("name", sorted(entries()))
def test_made_on_the_stream_of_the_call(name, calls):
    done, made = calls
    call = entries()[name]
    made.clear()
    call(stream=SIDE)
    _, stream, on, kept = done[-1]
    assert stream == SIDE.cuda_stream
    assert on and all(s is SIDE for s in on)
    # the caller, on the current stream, may drop them while kernels of that stream read them
    assert kept and all(s is CURRENT for s in kept)


@pytest.mark.parametrize("stream", [None, CURRENT])
@pytest.mark.parametrize("name", sorted(entries()))
def test_made_on_the_current_stream(name, stream, calls):
    done, made = calls
    call = entries()[name]
    made.clear()
    call(stream=stream)
    assert done[-1][1] == CURRENT.cuda_stream
    assert done[-1][2] and all(s is CURRENT for s in done[-1][2]) and done[-1][3] == []

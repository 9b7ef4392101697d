"""Calls on a stream of their own while the current stream is busy: what the binding makes for them is
not filled behind their kernels."""
import pytest
import torch

import ops_oracle
from cache_oracle import fill, i32, randn
from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def calls():
    lens, H, heads, D, S = [300, 77], 2, 4, 64, 16
    cache = ops_oracle.Cache(2, 19, H, D, S, True, DEV, spare=10)
    fill(cache, lens, 3)
    used = set(cache.table.flatten().tolist())
    other = i32([p for p in range(cache.pages) if p not in used][:10]).view(2, 5)
    args, kw = cache.args(i32(lens)), cache.scales()
    q = randn((2, 3, heads, D), 1).to(DEV)
    rows, start = q.flatten(0, 1), i32([1, 3, 5])  # the first and the last are no sequence's
    w = torch.rand((2, H, 304), device=DEV)
    z = randn((2, 5, 500), 2).to(DEV)
    return dict(
        read=lambda **s: spc.spc_kv_read(*args, 310, **kw, **s),
        attend=lambda **s: spc.spc_kv_attend(rows, *args, q_start=start, **kw, **s),
        shared=lambda **s: spc.spc_kv_attend_shared(rows, *args, 0, q_start=start, **kw, **s),
        cross=lambda **s: spc.spc_cross_attend(rows, *args, q_start=start, **kw, **s),
        weigh=lambda **s: spc.spc_kv_weigh(q, *args, w, **kw, **s),
        evict=lambda **s: spc.spc_kv_evict(*args, w, 80, other, recent=9, **kw, **s)[2],
        truncate=lambda **s: spc.spc_truncate(z, top_k=7, **s))


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", ["attend", "cross", "evict", "read", "shared", "truncate", "weigh"])
def test_on_another_stream(name, handle):
    call = calls()[name]
    want = [t.clone() for t in (lambda x: x if isinstance(x, tuple) else (x,))(call())]
    side = torch.cuda.Stream()
    a = torch.randn((4096, 4096), device=DEV)
    a @ a
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for _ in range(30):  # the current stream is busy for some milliseconds
        a = (a @ a) * 1e-2
    stream = side
    if handle:  # any object with a stream's handle
        stream = type("Stream", (), {"cuda_stream": side.cuda_stream})()
    got = call(stream=stream)
    side.synchronize()
    with torch.cuda.stream(side):
        first = [t.cpu() for t in (got if isinstance(got, tuple) else (got,))]
    torch.cuda.synchronize()  # (a fill on the current stream would be done now)
    for x, y, z in zip(want, first, got if isinstance(got, tuple) else (got,)):
        assert torch.equal(x.cpu().view(torch.uint8), y.view(torch.uint8))
        assert torch.equal(x.view(torch.uint8), z.view(torch.uint8))


@pytest.mark.parametrize("name", ["attend", "cross", "evict", "read", "shared", "truncate", "weigh"])
def test_on_a_captured_branch(name):
    """A call on a stream that a capture forks to and joins: what it makes is filled in the branch,
    every replay again."""
    def outputs(x):
        return x if isinstance(x, tuple) else (x,)

    call = calls()[name]
    want = [t.clone() for t in outputs(call())]
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        side.wait_stream(torch.cuda.current_stream())
        got = outputs(call(stream=side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        for t in got:
            t.fill_(3)
        call()  # (eager work between the replays)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))

"""Attention of a batch behind a shared prefix (spc_kv_attend_shared) against the 64-bit
definition (tolerances: ops_oracle.attend) and spc_kv_attend over tables that hold the prefix."""
import numpy as np
import pytest
import torch

import ops_oracle
from cache_oracle import BF16, check_rows, chunks, fill, i32, randn
from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


class Batch:
    """B sequences of which the first `shared` tokens lie in pages of sequence B (an extra one),
    and the others in their own; a sequence's own pages hold junk where the prefix would be."""

    def __init__(self, B, shared, own, H, D, S, f8, seed=0):
        lens = [shared + m for m in own]
        width = (max(lens + [shared]) + S - 1) // S
        self.all = ops_oracle.Cache(B + 1, width, H, D, S, f8, DEV, seed=seed)
        fill(self.all, lens + [shared], seed + 100)
        self.prefix = self.all.table[B, :(shared + S - 1) // S].contiguous()
        self.table = self.all.table[:B].contiguous()
        # entries of whole shared pages are not used: some are no page at all
        whole = shared // S
        self.table[:, :whole] = i32([-1, 7, self.all.pages])[torch.arange(whole) % 3]
        self.B, self.lens, self.shared, self.S = B, lens, shared, S

    def args(self, lens=None):
        return self.all.k, self.all.v, self.table, i32(self.lens if lens is None else lens)

    def lines(self, b):
        n = max(int(self.lens[b]), 0)
        k, v, there = self.all.dense(b, n)
        kp, vp, in_p = self.all.dense(self.B, n)
        pre = (np.arange(n) < self.shared)[:, None, None]
        return np.where(pre, kp, k), np.where(pre, vp, v), np.where(pre[:, 0, 0], in_p, there)


def sees(window):
    def f(b, at, n):
        t = np.arange(n)
        return (t <= at) & ((t > at - window) if window else True)
    return f


def check(x, q, starts=None, window=0, scale=None, **kw):
    D = q.shape[-1]
    out = spc.spc_kv_attend_shared(q, *x.args(), x.shared, shared_table=x.prefix, window=window,
                                   scale=scale, q_start=None if starts is None else i32(starts),
                                   **x.all.scales(), **kw)
    f = sees(window)
    worst = check_rows(out, q, x.lens, starts, x.lines, lambda b, at: f(b, at, x.lens[b]),
                       D ** -0.5 if scale is None else scale)
    return out, worst


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,shared,S", [(1, 1, 16), (1, 16, 16), (1, 300, 16), (3, 33, 48),
                                        (1, 64, 64), (5, 700, 32), (20, 130, 16)])
def test_lengths(n, shared, S, D, f8):
    B, H, heads = 3, 2, 4
    x = Batch(B, shared, [n, n + 40, n + 3], H, D, S, f8, seed=n + shared)
    check(x, randn((B, n, heads, D), 3).to(DEV))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("B,n,H,heads", [(1, 1, 1, 1), (40, 1, 2, 8), (17, 2, 1, 3), (9, 8, 1, 8),
                                         (2, 70, 2, 2), (5, 1, 3, 15)])
def test_rows_and_heads(B, n, H, heads, f8):
    """From one row to several tiles of 128 of all sequences together."""
    x = Batch(B, 530, [n + (7 * b) % 30 for b in range(B)], H, 64, 16, f8, seed=B)
    check(x, randn((B, n, heads, 64), 4).to(DEV))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 200, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("n", [1, 6, 50])
def test_windows(n, window, f8):
    """Windows that end in a sequence's own tokens, in the prefix, and before it."""
    x = Batch(3, 170, [n, n + 60, n + 2], 1, 128, 16, f8, seed=n)
    check(x, randn((3, n, 4, 128), 5).to(DEV), window=window)


@pytest.mark.parametrize("f8", [False, True])
def test_ragged_and_rows_inside_the_prefix(f8):
    """Chunks of 0 to many rows; rows at positions inside the prefix, before position 0; rows of
    no sequence; a chunk longer than max_q."""
    ns, own = [0, 1, 7, 40, 3, 60, 2], [5, 1, 7, 45, 0, -20, -49]
    x = Batch(len(ns), 50, own, 2, 128, 32, f8, seed=1)
    starts = (np.concatenate([[0], np.cumsum(ns)]) + 3).tolist()
    q = randn((starts[-1] + 2, 6, 128), 8).to(DEV)
    out = torch.full_like(q, 3.0)
    got, _ = check(x, q, starts, max_q=60, out=out)
    assert got is out
    assert bool((out[:3] == 3.0).all()) and bool((out[-2:] == 3.0).all())
    assert bool((out[starts[6]] == 0).all())  # before position 0
    check(x, q, starts)  # max_q: all rows
    part = torch.full_like(q, 5.0)
    spc.spc_kv_attend_shared(q, *x.args(), 50, shared_table=x.prefix, q_start=i32(starts), max_q=9,
                             out=part, **x.all.scales())
    for b, n in enumerate(ns):
        m = min(n, 9)
        assert torch.equal(part[starts[b]:starts[b] + m], out[starts[b]:starts[b] + m]) or m < n
        assert bool((part[starts[b] + m:starts[b + 1]] == 5.0).all())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [1, 9])
def test_tables_that_hold_the_prefix(n, f8):
    """shared_table None is the first sequence's row; the answer is spc_kv_attend's up to the order
    of its sums; shared = 0 is spc_kv_attend."""
    x = Batch(4, 96, [n + 11] * 4, 2, 64, 16, f8)
    x.table[:, :6] = x.prefix
    q = randn((4, n, 8, 64), 2).to(DEV)
    check(x, q)
    a = spc.spc_kv_attend_shared(q, *x.args(), 96, **x.all.scales())
    b = spc.spc_kv_attend_shared(q, *x.args(), 96, shared_table=x.prefix, **x.all.scales())
    assert torch.equal(a, b)
    a = spc.spc_kv_attend_shared(q, *x.args(), 0, **x.all.scales())
    b = spc.spc_kv_attend(q, *x.args(), **x.all.scales())
    assert torch.equal(a, b)


@pytest.mark.parametrize("f8", [False, True])
def test_pages_that_are_none_and_tables_of_the_prefix_alone(f8):
    x = Batch(3, 100, [5, 20, 1], 1, 64, 16, f8)
    x.prefix[2] = -1
    x.prefix[4] = x.all.pages
    x.all.table[3, :7] = x.prefix  # (what the definition reads)
    q = randn((3, 1, 2, 64), 2).to(DEV)
    check(x, q)
    # no table reaches past the prefix: nobody sees a token of its own
    x = Batch(3, 96, [0, 0, 0], 1, 64, 16, f8)
    assert x.table.shape[1] * 16 == 96
    check(x, q)
    # a prefix that no one reaches the end of
    x = Batch(2, 96, [-90, -96], 1, 64, 16, f8)
    out, _ = check(x, q[:2].contiguous())
    assert bool((out[1] == 0).all())


@pytest.mark.parametrize("f8", [False, True])
def test_what_lies_before_and_behind_may_be_anything(f8):
    """NaN behind the prefix's last token, and where a sequence's own page holds what the prefix has."""
    B, shared, S, H, D = 2, 21, 16, 1, 128
    x = Batch(B, shared, [9, 30], H, D, S, f8)
    byte = 0x7f if f8 else 0xff
    for pages, slots in ((x.prefix[1:2], range(5, 16)), (x.table[:, 1], range(0, 5))):
        for p in pages.tolist():
            for s in slots:
                x.all.k.view(torch.uint8)[p, :, s] = byte
                x.all.v.view(torch.uint8).view(x.all.pages, H, D, S, -1)[p, :, :, s] = byte
                if f8:
                    x.all.ks[p, :, s] = float("nan")
                    x.all.vs[p, :, s] = float("inf")
    check(x, randn((B, 3, 4, D), 2).to(DEV))


@pytest.mark.parametrize("f8", [False, True])
def test_strides_workspaces_and_streams(f8):
    B, n, H, heads, D = 3, 2, 2, 4, 64
    x = Batch(B, 300, [20, 9, 2], H, D, 16, f8)
    wide = randn((B, n, 3 * heads * D + 3), 2).to(DEV)
    q = wide[..., 5:5 + heads * D].unflatten(-1, (heads, D))
    full = torch.full((B, n, 2 * heads, D), 9.0, dtype=BF16, device=DEV)
    check(x, q, out=full[:, :, :heads])
    assert bool((full[:, :, heads:] == 9.0).all())
    need = spc.spc_kv_shared_workspace_bytes(*x.args(), 300, heads, B * n, **x.all.scales())
    assert need > 0
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = spc.spc_kv_attend_shared(q, *x.args(), 300, shared_table=x.prefix, workspace=ws[:need],
                                       **x.all.scales())
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, full[:, :, :heads])
    assert bool((ws[need:] == 255).all())
    with pytest.raises(spc.SpcError):
        spc.spc_kv_attend_shared(q, *x.args(), 300, shared_table=x.prefix, workspace=ws[:need - 256],
                                 **x.all.scales())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [3, 30])
@pytest.mark.parametrize("s,scale", [(12.0, None), (1.0, 0.0), (1.0, -0.3)])
def test_scales_and_peaked_scores(s, scale, n, f8):
    x = Batch(2, 500, [n, 77], 1, 128, 64, f8)
    fill(x.all, x.lens + [500], 9, s)
    check(x, randn((2, n, 4, 128), 1, BF16, s).to(DEV), scale=scale)


def test_captured_and_replayed():
    x = Batch(4, 400, [60, 60, 60, 60], 2, 128, 16, False)
    q = randn((4, 1, 8, 128), 2).to(DEV)
    lens = i32([409, 460, 430, 401])
    args = (x.all.k, x.all.v, x.table, lens)
    kw = dict(shared_table=x.prefix)
    out = torch.empty_like(q)
    spc.spc_kv_attend_shared(q, *args, 400, out=out, **kw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spc.spc_kv_attend_shared(q, *args, 400, out=out, **kw)
    for k in range(4):
        q.copy_(randn(q.shape, 20 + k))
        lens.copy_(i32([400 + (13 * k + 7 * b) % 60 + 1 for b in range(4)]))
        g.replay()
        torch.cuda.synchronize()
        want = spc.spc_kv_attend_shared(q, *args, 400, **kw)
        assert torch.equal(out, want)
        assert not bool(torch.isnan(out.float()).any())

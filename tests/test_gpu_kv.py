"""The paged cache (spc_kv_write, spc_kv_read) and the chunk attention over it
(spc_kv_attend) against the 64-bit definitions.  Writes and reads are exact
(one rounding that both sides make); the attention's tolerance is derived in
ops_oracle.attend."""
import numpy as np
import pytest
import torch

import ops_oracle
from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def randn(shape, seed, dtype=BF16, s=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * s).to(dtype)


def fill(cache, lens, seed, s=1.0):
    """Write every sequence's tokens 0 .. lens[b] - 1 (one ragged call); the dense values."""
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    N = int(start[-1])
    k, v = (randn((max(N, 1), cache.H, cache.D), seed + i, BF16, s) for i in range(2))
    if N:
        spc.spc_kv_write(k.to(DEV), v.to(DEV), *cache.args(i32(lens)), q_start=i32(start),
                         **cache.scales())
    return k, v, start


def check_attend(cache, q, lens, starts=None, scale=None, window=0, **kw):
    """q on the device: [B, n, heads, D], or [rows, heads, D] with starts."""
    B, H, D = cache.B, cache.H, cache.D
    out = spc.spc_kv_attend(q, *cache.args(i32(lens)), scale=scale, window=window,
                            q_start=None if starts is None else i32(starts), **cache.scales(), **kw)
    torch.cuda.synchronize()
    heads = q.shape[-2]
    host, got = q.cpu().double().numpy().reshape(-1, heads, D), out.cpu().double().numpy()
    got = got.reshape(-1, heads, D)
    if starts is None:
        n = q.shape[1]
        starts = [n * b for b in range(B + 1)]
    sc = D ** -0.5 if scale is None else scale
    worst = 0.0
    for b in range(B):
        k, v, there = cache.dense(b, max(int(lens[b]), 0))
        n = starts[b + 1] - starts[b]
        for i in range(n):
            at = int(lens[b]) - n + i
            for g in range(heads):
                h = g // (heads // H)
                o, tol = ops_oracle.attend(host[starts[b] + i, g], k[:, h], v[:, h], there,
                                           at - window + 1 if window else 0, at, sc)
                d = np.abs(got[starts[b] + i, g] - o)
                assert (d <= tol).all(), (b, i, g, float((d - tol).max()), at)
                worst = max(worst, float((d / np.maximum(tol, 1e-30)).max()))
    return out, worst


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("S,H,D", [(16, 1, 64), (48, 3, 128), (64, 2, 256), (1024, 1, 128)])
def test_write_and_read(S, H, D, dtype, f8):
    B, lens = 4, [1, 0, 2 * S - 3, S + 17]
    cache = ops_oracle.Cache(B, 3, H, D, S, f8, DEV, seed=S)
    before = cache.k.view(torch.uint8).clone(), cache.v.view(torch.uint8).clone()
    start = np.concatenate([[0], np.cumsum(lens)])
    N = int(start[-1])
    # rows inside a wider tensor, as a fused projection gives them
    wide = randn((N, 2 * H * D + 7), 3, dtype, 3.0)
    wide[0, 5] = 1e-30 if dtype == F32 else 0.0
    wide[N - 1] = 0.0
    dev = wide.to(DEV)
    k, v = (dev[:, i * H * D:(i + 1) * H * D].unflatten(1, (H, D)) for i in range(2))
    spc.spc_kv_write(k, v, *cache.args(i32(lens)), q_start=i32(start), **cache.scales())
    k_out, v_out = (torch.full((B, max(lens) + 2, H, D), 7.0, dtype=dtype, device=DEV)
                    for _ in range(2))
    spc.spc_kv_read(*cache.args(i32(lens)), out=(k_out, v_out), **cache.scales())
    for x, out in ((k, k_out), (v, v_out)):
        x, out = x.cpu().float().numpy(), out.cpu()
        for b in range(B):
            row = x[start[b]:start[b + 1]]
            if f8 and len(row):
                codes, scale = ops_oracle.quantised(row)
                want = torch.from_numpy(codes.astype(np.float32) * scale[..., None]).to(dtype)
            else:
                want = torch.from_numpy(row).to(BF16).to(dtype)
            assert torch.equal(out[b, :lens[b]], want)
            assert bool((out[b, lens[b]:] == 7.0).all())
    # nothing else of the cache changed
    touched = torch.zeros((cache.pages, S), dtype=torch.bool)
    for b in range(B):
        for t in range(lens[b]):
            touched[int(cache.table[b, t // S]), t % S] = True
    w = 1 if f8 else 2
    same_k = (cache.k.view(torch.uint8) == before[0]).cpu().view(cache.pages, H, S, D * w).all(-1).all(1)
    same_v = (cache.v.view(torch.uint8) == before[1]).cpu().view(cache.pages, H, D, S, w).all(-1).all(2).all(1)
    assert bool(same_k[~touched].all()) and bool(same_v[~touched].all())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("S,lens", [(16, [131, 300, 129]), (48, [400, 7, 257]), (128, [129, 128, 255])])
def test_long_chunks_written(S, lens, D, f8):
    """Chunks long enough to be written in tiles, from any slot, sequence after
    sequence inside a tile."""
    B, H = len(lens), 2
    cache = ops_oracle.Cache(B, (max(lens) + 5 + S - 1) // S, H, D, S, f8, DEV, seed=D)
    start = np.concatenate([[0], np.cumsum(lens)])
    k, v = randn((int(start[-1]), H, D), 1, F32), randn((int(start[-1]), H, D), 2, F32)
    at = np.array(lens) + [5, 0, 3]  # the chunks begin at slots 5, 0 and 3
    spc.spc_kv_write(k.to(DEV), v.to(DEV), *cache.args(i32(at)), q_start=i32(start), **cache.scales())
    for b in range(B):
        kd, vd, _ = cache.dense(b, int(at[b]))
        for got, x in ((kd, k), (vd, v)):
            x = x[start[b]:start[b + 1]]
            if f8:
                codes, scale = ops_oracle.quantised(x.numpy())
                want = codes * scale[..., None].astype(np.float64)
            else:
                want = x.to(BF16).double().numpy()
            np.testing.assert_array_equal(got[at[b] - lens[b]:], want)


@pytest.mark.parametrize("f8", [False, True])
def test_write_a_chunk_behind_what_is_there(f8):
    """Uniform chunks at any offset into a page leave the tokens before them alone."""
    B, S, H, D, n = 5, 16, 2, 64, 9
    cache = ops_oracle.Cache(B, 4, H, D, S, f8, DEV)
    lens = np.array([0, 3, 15, 16, 30])
    fill(cache, lens, 1)
    old = [cache.dense(b, int(lens[b])) for b in range(B)]
    k, v = randn((B, n, H, D), 5), randn((B, n, H, D), 6)
    spc.spc_kv_write(k.to(DEV), v.to(DEV), *cache.args(i32(lens + n)), **cache.scales())
    for b in range(B):
        kd, vd, _ = cache.dense(b, int(lens[b]) + n)
        np.testing.assert_array_equal(kd[:lens[b]], old[b][0])
        np.testing.assert_array_equal(vd[:lens[b]], old[b][1])
        for got, x in ((kd, k), (vd, v)):
            x = x[b].float().numpy()
            if f8:
                codes, scale = ops_oracle.quantised(x)
                x = codes * scale[..., None].astype(np.float64)
            np.testing.assert_array_equal(got[lens[b]:], x)


def test_tokens_outside_the_cache_are_skipped():
    """Page ids out of range, positions before 0 and past the table, rows of no
    sequence: no write, nothing read back, nothing attended to."""
    B, S, H, D, width = 4, 16, 1, 64, 3
    for f8 in (False, True):
        cache = ops_oracle.Cache(B, width, H, D, S, f8, DEV, seed=4)
        lens = [40, 40, 60, 5]
        fill(cache, [40, 40, 48, 5], 1)
        cache.table[0, 1] = -1
        cache.table[1, 0] = cache.pages
        cache.table[1, 2] = 2 ** 31 - 1
        snap = cache.k.view(torch.uint8).clone(), cache.v.view(torch.uint8).clone()
        # rows 0, 1 before every sequence and the last 3 behind
        starts = [2, 10, 18, 26, 34]
        k = randn((37, H, D), 8).to(DEV)
        # (8 rows a sequence: sequence 2 ends past the table, sequence 3 begins before 0)
        spc.spc_kv_write(k, k, *cache.args(i32(lens)), q_start=i32(starts), **cache.scales())
        kd, _, there = cache.dense(0, 40)
        assert list(there) == [True] * 16 + [False] * 16 + [True] * 8
        # sequence 3: rows 3 .. 7 of its 8 are positions 0 .. 4
        kd, _, _ = cache.dense(3, 5)
        x = k[29:34].cpu().float().numpy()
        want = x
        if f8:
            codes, scale = ops_oracle.quantised(x)
            want = codes * scale[..., None].astype(np.float64)
        np.testing.assert_array_equal(kd, want)
        # sequence 2: positions 52 .. 59 lie past its 48 slots; its pages are as they were
        for p in cache.table[2].tolist():
            assert torch.equal(cache.k.view(torch.uint8)[p], snap[0][p])
            assert torch.equal(cache.v.view(torch.uint8)[p], snap[1][p])
        q = randn((37, 2, D), 9).to(DEV)
        out = torch.full((37, 2, D), 3.0, dtype=BF16, device=DEV)
        check_attend(cache, q, lens, starts, out=out, max_q=8)
        assert bool((out[:2] == 3.0).all()) and bool((out[34:] == 3.0).all())
        assert bool((out[26:29] == 0.0).all())  # rows before position 0 see nothing
        ko = torch.full((B, 50, H, D), 7.0, dtype=F32, device=DEV)
        vo = ko.clone()
        spc.spc_kv_read(*cache.args(i32(lens)), out=(ko, vo), **cache.scales())
        assert bool((ko[0, 16:32] == 7.0).all()) and bool((ko[1, :16] == 7.0).all())
        assert bool((ko[1, 16:32] != 7.0).any()) and bool((ko[2, 48:] == 7.0).all())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,L", [(1, 1), (1, 2), (1, 33), (2, 2), (3, 16), (8, 100), (9, 31), (17, 17),
                                 (33, 70), (5, 513), (1, 1500), (70, 200)])
def test_attend_lengths(n, L, D, f8):
    B, H, heads, S = 2, 2, 8, 16
    cache = ops_oracle.Cache(B, (L + S - 1) // S, H, D, S, f8, DEV, seed=n)
    lens = [L, max(n, L - 5)]
    fill(cache, lens, L)
    check_attend(cache, randn((B, n, heads, D), 3).to(DEV), lens)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("H,heads", [(1, 1), (1, 3), (2, 2), (4, 4), (1, 16), (3, 15), (2, 64), (1, 71)])
@pytest.mark.parametrize("S,n", [(32, 1), (48, 4), (128, 3)])
def test_attend_heads_and_pages(S, n, H, heads, f8):
    B, D = 3, 64
    lens = [n, 3 * S // 2 + 1, 4 * S]
    cache = ops_oracle.Cache(B, 4, H, D, S, f8, DEV, seed=S + n)
    fill(cache, lens, heads)
    check_attend(cache, randn((B, n, heads, D), heads).to(DEV), lens)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 5000])
@pytest.mark.parametrize("n,L", [(1, 300), (8, 77), (40, 130)])
def test_attend_window(n, L, window, f8):
    B, H, heads, D, S = 2, 1, 2, 128, 16
    cache = ops_oracle.Cache(B, (L + S - 1) // S, H, D, S, f8, DEV, seed=window)
    fill(cache, [L, L - 1], 2)
    check_attend(cache, randn((B, n, heads, D), 4).to(DEV), [L, L - 1], window=window)


@pytest.mark.parametrize("f8", [False, True])
def test_attend_ragged_empty_and_short(f8):
    """Chunks of 0, 1 and many rows; empty caches; chunks longer than the cache."""
    H, heads, D, S = 2, 6, 128, 32
    ns = [0, 1, 7, 40, 3, 2]
    lens = [9, 130, 7, 64, 0, 1]
    starts = np.concatenate([[0], np.cumsum(ns)]).tolist()
    cache = ops_oracle.Cache(len(ns), 5, H, D, S, f8, DEV)
    fill(cache, lens, 7)
    q = randn((starts[-1], heads, D), 8).to(DEV)
    out, _ = check_attend(cache, q, lens, starts, max_q=40)
    assert bool((out[starts[4]:starts[5]] == 0).all()) and bool((out[starts[5]] == 0).all())
    check_attend(cache, q, lens, starts)  # max_q: all rows
    # a chunk longer than max_q: its rows past it are left as they are
    part = torch.full_like(q, 5.0)
    spc.spc_kv_attend(q, *cache.args(i32(lens)), q_start=i32(starts), max_q=8, out=part, **cache.scales())
    assert torch.equal(part[starts[3]:starts[3] + 8], out[starts[3]:starts[3] + 8])
    assert bool((part[starts[3] + 8:starts[4]] == 5.0).all())
    assert torch.equal(part[starts[2]:starts[3]], out[starts[2]:starts[3]])


@pytest.mark.parametrize("f8", [False, True])
def test_attend_strided_queries_and_outputs(f8):
    B, n, H, heads, D, S, L = 3, 4, 2, 4, 64, 16, 50
    cache = ops_oracle.Cache(B, 4, H, D, S, f8, DEV)
    lens = [50, 20, 4]
    fill(cache, lens, 1)
    wide = randn((B, n, 3 * heads * D + 3), 2).to(DEV)
    q = wide[..., 5:5 + heads * D].unflatten(-1, (heads, D))
    full = torch.full((B, n, 2 * heads, D), 9.0, dtype=BF16, device=DEV)
    check_attend(cache, q, lens, out=full[:, :, :heads])
    assert bool((full[:, :, heads:] == 9.0).all())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n,L", [(1, 40), (3, 700), (40, 300), (140, 300)])
def test_a_nan_that_a_row_sees_is_its_answer(n, L, f8):
    """A NaN among the keys or values a row sees is not lost: the row (the value's
    dimension of it) is NaN, wherever in a tile the key lies."""
    H, heads, D, S = 1, 4, 128, 16
    cache = ops_oracle.Cache(2, (L + S - 1) // S, H, D, S, f8, DEV)
    fill(cache, [L, L], 3)
    at = L - n  # the first row's own position: every row sees it
    page, slot = int(cache.table[0, at // S]), at % S
    nan = torch.tensor(0x7f, dtype=torch.uint8) if f8 else torch.tensor(float("nan"), dtype=BF16)
    cache.k[page, 0, slot, 5:6].view(torch.uint8 if f8 else BF16).fill_(nan.item())
    page, slot = int(cache.table[1, at // S]), at % S
    cache.v[page, 0, 7, slot:slot + 1].view(torch.uint8 if f8 else BF16).fill_(nan.item())
    q = randn((2, n, heads, D), 4).to(DEV)
    out = spc.spc_kv_attend(q, *cache.args(i32([L, L])), **cache.scales()).float()
    assert bool(out[0].isnan().all())
    assert bool(out[1, ..., 7].isnan().all())
    rest = torch.cat([out[1, ..., :7], out[1, ..., 8:]], -1)
    assert not bool(rest.isnan().any())


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("s,scale", [(12.0, None), (1.0, 0.0), (1.0, -0.3), (0.01, 1.0)])
def test_attend_scales_and_peaked_scores(s, scale, f8):
    """Scores of hundreds (a softmax of one key), equal scores, a negative scale."""
    B, H, heads, D, S, L = 2, 1, 4, 128, 64, 500
    cache = ops_oracle.Cache(B, 8, H, D, S, f8, DEV)
    fill(cache, [L, 77], 3, s)
    check_attend(cache, randn((B, 3, heads, D), 1, BF16, s).to(DEV), [L, 77], scale=scale)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("B,n,L,H,heads", [(1, 1, 20000, 1, 8), (2, 8, 9000, 2, 8), (1, 3, 5001, 1, 1),
                                           (40, 1, 700, 2, 4)])
def test_attend_long_caches(B, n, L, H, heads, f8):
    D, S = 64, 16
    cache = ops_oracle.Cache(B, (L + S - 1) // S, H, D, S, f8, DEV)
    lens = [max(n, L - 97 * b) if b % 3 else max(n, L // (b + 1)) for b in range(B)]
    fill(cache, lens, 3)
    q = randn((B, n, heads, D), 4).to(DEV)
    a, _ = check_attend(cache, q, lens)
    # split sums are joined in a fixed order
    assert torch.equal(a, spc.spc_kv_attend(q, *cache.args(i32(lens)), **cache.scales()))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("B,n,L,H,heads,D,window", [(1, 70, 6000, 1, 2, 64, 0), (2, 130, 3000, 1, 1, 128, 0),
                                                    (1, 33, 5000, 1, 4, 256, 0), (1, 65, 4000, 1, 2, 64, 2500)])
def test_many_rows_over_shares_of_the_keys(B, n, L, H, heads, D, window, f8):
    S = 32
    cache = ops_oracle.Cache(B, (L + S - 1) // S, H, D, S, f8, DEV)
    lens = [L - 401 * b for b in range(B)]
    fill(cache, lens, 3)
    check_attend(cache, randn((B, n, heads, D), 4).to(DEV), lens, window=window)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n,heads", [(3, 2), (20, 2), (90, 2), (1, 64)])
@pytest.mark.parametrize("S", [16, 48, 1024])
def test_attend_around_missing_pages(S, n, heads, f8):
    """Pages missing at the start, in the middle and at the end, for every kernel."""
    B, H, D, width = 3, 1, 64, 1 + 400 // S
    cache = ops_oracle.Cache(B, width + 1, H, D, S, f8, DEV, seed=S)
    lens = [min(400, S * width), n, min(371, S * width)]
    fill(cache, lens, 5)
    for b, at in ((0, 0), (0, width // 2), (2, width - 1)):
        cache.table[b, at] = -5 if at else cache.pages + 7
    check_attend(cache, randn((B, n, heads, D), 6).to(DEV), lens)


def test_a_capture_that_needs_a_larger_workspace_is_refused():
    """As for the verify calls: the call says so, and an eager call first mends it."""
    spc.spc_release()
    B, H, heads, D, S, L = 1, 1, 2, 64, 16, 4000
    cache = ops_oracle.Cache(B, L // S, H, D, S, False, DEV)
    fill(cache, [L], 1)
    q, lens = randn((B, 1, heads, D), 2).to(DEV), i32([L])
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(spc.SpcError) as e:
            spc.spc_kv_attend(q, *cache.args(lens), out=out)
        assert e.value.status == -6
        out.zero_()
    want = spc.spc_kv_attend(q, *cache.args(lens))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spc.spc_kv_attend(q, *cache.args(lens), out=out)
    for _ in range(2):
        out.fill_(1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_attend_offsets_past_32_bits():
    """Pages whose byte offsets pass 2^32: the last of 600 000 pages of 8 KiB."""
    S, H, D, pages = 16, 2, 128, 600_000
    k = torch.empty((pages, H, S, D), dtype=BF16, device=DEV)
    v = torch.empty((pages, H, D, S), dtype=BF16, device=DEV)
    cache = ops_oracle.Cache(1, 3, H, D, S, False, DEV)
    fill(cache, [45], 1)
    q = randn((1, 2, 4, D), 2).to(DEV)
    want = spc.spc_kv_attend(q, *cache.args(i32([45])))
    table = i32([[pages - 1, 5, pages - 300_000]])
    for i, p in enumerate(table[0].tolist()):
        k[p], v[p] = cache.k[int(cache.table[0, i])], cache.v[int(cache.table[0, i])]
    new_k, new_v = randn((1, 2, H, D), 5).to(DEV), randn((1, 2, H, D), 6).to(DEV)
    for kk, vv, tt in ((k, v, table), (cache.k, cache.v, cache.table)):
        spc.spc_kv_write(new_k, new_v, kk, vv, tt, i32([47]))
    assert torch.equal(spc.spc_kv_attend(q, k, v, table, i32([45])), want)
    assert torch.equal(spc.spc_kv_attend(q, k, v, table, i32([47])),
                       spc.spc_kv_attend(q, *cache.args(i32([47]))))
    for a, b in zip(spc.spc_kv_read(k, v, table, i32([47]), 47),
                    spc.spc_kv_read(*cache.args(i32([47])), 47)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("f8", [False, True])
def test_graph_replays_write_and_attend(f8):
    """A captured write and attention replay with new tokens and lengths (a
    rollback among them) as eager calls give them."""
    B, n, H, heads, D, S = 4, 5, 2, 8, 64, 16
    width = 130

    def steps(call, cache, q, k, kv_len):
        outs = []
        for r, lens in enumerate(([5, 5, 5, 5], [10, 7, 5, 9], [900, 8, 10, 14], [11, 12, 2000, 5])):
            q.copy_(randn((B, n, heads, D), r).to(DEV))
            k.copy_(randn((B, n, H, D), 10 + r).to(DEV))
            kv_len.copy_(i32(lens))
            call()
            torch.cuda.synchronize()
            outs.append(cache["out"].clone())
        return outs

    def setup():
        c = ops_oracle.Cache(B, width, H, D, S, f8, DEV, seed=2)
        fill(c, [2000] * B, 1)
        q = torch.empty((B, n, heads, D), dtype=BF16, device=DEV)
        k = torch.empty((B, n, H, D), dtype=BF16, device=DEV)
        kv_len = i32([5] * B)
        box = dict(out=torch.empty_like(q))

        def call():
            spc.spc_kv_write(k, k, *c.args(kv_len), **c.scales())
            spc.spc_kv_attend(q, *c.args(kv_len), out=box["out"], **c.scales())
        return call, box, q, k, kv_len

    call, box, q, k, kv_len = setup()
    want = steps(call, box, q, k, kv_len)
    call, box, q, k, kv_len = setup()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        k.copy_(randn((B, n, H, D), 10).to(DEV))
        q.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for a, b in zip(steps(g.replay, box, q, k, kv_len), want):
        assert torch.equal(a, b)


def test_caller_workspaces_on_two_streams():
    B, H, heads, D, S, L = 2, 1, 8, 128, 32, 6000
    runs = []
    for s in range(2):
        cache = ops_oracle.Cache(B, (L + S - 1) // S, H, D, S, s == 1, DEV, seed=s)
        fill(cache, [L, L // 2], s)
        q = randn((B, 2, heads, D), s).to(DEV)
        lens = i32([L, L // 2])
        n = spc.spc_kv_workspace_bytes(*cache.args(lens), heads, 2 * B, **cache.scales())
        ws = torch.full((max(n, 1),), 255, dtype=torch.uint8, device=DEV)
        runs.append((cache, q, lens, ws, spc.spc_kv_attend(q, *cache.args(lens), **cache.scales())))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        outs = []
        for (cache, q, lens, ws, _), st in zip(runs, streams):
            with torch.cuda.stream(st):
                outs.append(spc.spc_kv_attend(q, *cache.args(lens), workspace=ws, **cache.scales()))
        torch.cuda.synchronize()
        for o, r in zip(outs, runs):
            assert torch.equal(o, r[4])

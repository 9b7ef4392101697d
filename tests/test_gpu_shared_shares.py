"""Attention behind a shared prefix where a sequence's own tokens are cut into several shares, and where
more shares are joined than a wavefront has lanes; chunks longer than max_q, there and in the cross
attention.  Against the 64-bit definition (tolerances: ops_oracle.attend)."""
import numpy as np
import pytest
import torch

import ops_oracle
from cache_oracle import check_rows, fill, i32, randn
from paper_2405_19261_amd import spc
from test_gpu_shared_prefix import Batch, check, sees

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def shares(x, heads, n):
    """(bytes of the prefix's shares, own shares of a sequence) that the workspace is for: a table of
    the prefix alone has no own tokens, one of a page more has one share of them."""
    def need(width):
        table = torch.zeros((x.B, width), dtype=torch.int32, device=DEV)
        return spc.spc_kv_shared_workspace_bytes(x.all.k, x.all.v, table, i32(x.lens), x.shared, heads,
                                                 x.B * n, **x.all.scales())
    assert x.shared % x.S == 0
    whole = x.shared // x.S
    pre = need(whole)
    return pre, round((need(x.table.shape[1]) - pre) / (need(whole + 1) - pre))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 16, 70, 130])  # 2, 32, 140 and 260 rows a head: tiles of 16, 32 and 128
def test_own_tokens_in_several_shares(n, D, window, f8):
    x = Batch(3, 96, [2000, 611, n + 3], 1, D, 16, f8, seed=n)
    assert shares(x, 2, n)[1] > 3
    check(x, randn((3, n, 2, D), 3).to(DEV), window=window)


@pytest.mark.parametrize("f8,D,shared,own,n", [
    (False, 64, 10000, [5, 300], 1),         # 78 shares of the prefix, one of the others
    (False, 128, 10000, [2500, 1], 2),
    (False, 64, 17008, [9000, 8000], 1),     # 128 and 70
    (True, 64, 17008, [5000, 700], 1),       # 66 and 19
    (False, 256, 33008, [1300, 9], 70),      # tiles of 128 rows
])
@pytest.mark.parametrize("window", [0, 9700])
def test_many_shares(f8, D, shared, own, n, window):
    x = Batch(2, shared, own, 1, D, 16, f8, seed=1)
    pre, mine = shares(x, 1, n)
    tile = 16 if 2 * n <= 32 else 128
    rows = -(-2 * n // tile) * tile
    assert pre // (rows * (D + 2) * 4) > 64
    assert mine > max(own) // 300
    check(x, randn((2, n, 1, D), 3).to(DEV), window=window)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("max_q", [1, 9, 39])
def test_chunks_longer_than_max_q(max_q, f8):
    """Their first max_q rows are answered, at the positions that they have in the whole chunk."""
    ns, own = [0, 1, 7, 40, 3, 60], [5, 1, 7, 45, 0, 400]
    x = Batch(len(ns), 48, own, 2, 128, 16, f8, seed=1)
    starts = (np.concatenate([[0], np.cumsum(ns)]) + 3).tolist()
    q = randn((starts[-1] + 2, 6, 128), 8).to(DEV)
    enc_lens = [40, 130, 64, 300, 90, 0]
    enc = ops_oracle.Cache(len(ns), 20, 2, 128, 16, f8, DEV)
    fill(enc, enc_lens, 7)
    f = sees(0)
    for call, lens, lines, see in (
            (lambda **kw: spc.spc_kv_attend_shared(q, *x.args(), 48, shared_table=x.prefix,
                                                   q_start=i32(starts), **x.all.scales(), **kw),
             x.lens, x.lines, lambda b, at: f(b, at, x.lens[b])),
            (lambda **kw: spc.spc_cross_attend(q, *enc.args(i32(enc_lens)), q_start=i32(starts),
                                               **enc.scales(), **kw),
             enc_lens, lambda b: enc.dense(b, enc_lens[b]), lambda b, at: np.ones(enc_lens[b], bool))):
        whole, part = call(), call(max_q=max_q, out=torch.full_like(q, 5.0))
        for b, n in enumerate(ns):
            m = min(n, max_q)
            assert bool((part[starts[b] + m:starts[b + 1]] == 5.0).all())
            whole[starts[b]:starts[b] + m] = part[starts[b]:starts[b] + m]
        assert bool((part[:3] == 5.0).all()) and bool((part[-2:] == 5.0).all())
        check_rows(whole, q, lens, starts, lines, see, 128 ** -0.5)

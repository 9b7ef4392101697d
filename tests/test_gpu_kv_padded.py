"""Chunks with rows of no sequence before and behind them, as a captured call of a
fixed size has: what those rows hold does not matter, and nothing is written
for them."""
import numpy as np
import pytest
import torch

import ops_oracle
from paper_2405_19261_amd import spc
from test_gpu_kv import i32, randn

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lead,ns,tail", [(0, [3, 1], 900), (200, [0, 40, 2], 130), (67, [130, 61], 0),
                                          (64, [64], 64), (300, [0, 0], 300)])
def test_rows_of_no_sequence_are_not_looked_at(lead, ns, tail, D, dtype, f8):
    """Against the same chunks without the other rows, in calls that go row by row
    and in ones that go by tiles of 64 rows (of which some hold no row of a
    sequence, some one, and some rows past their sequence's table)."""
    B, H, S = len(ns), 2, 16
    N, rows = sum(ns), lead + sum(ns) + tail
    lens = [n + 7 for n in ns]
    lens[-1] = 6 * S + 5  # its last rows lie past the table
    ours, want = (ops_oracle.Cache(B, 6, H, D, S, f8, DEV, seed=9) for _ in range(2))
    k, v = (torch.full((rows, H, D), float("nan"), dtype=dtype) for _ in range(2))
    k[lead:lead + N], v[lead:lead + N] = randn((N, H, D), 1, dtype), randn((N, H, D), 2, dtype)
    at = np.concatenate([[0], np.cumsum(ns)])
    spc.spc_kv_write(k.to(DEV), v.to(DEV), *ours.args(i32(lens)), q_start=i32(at + lead), **ours.scales())
    for b in range(B):  # a row a call
        for i in range(ns[b]):
            r = lead + int(at[b]) + i
            start = i32([0] * (b + 1) + [1] * (B - b))
            upto = i32([lens[b] - ns[b] + i + 1] * B)
            spc.spc_kv_write(k[r:r + 1].to(DEV), v[r:r + 1].to(DEV), *want.args(upto), q_start=start,
                             **want.scales())
    for a, b in ((ours.k, want.k), (ours.v, want.v), (ours.ks, want.ks), (ours.vs, want.vs)):
        if a is not None:
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))

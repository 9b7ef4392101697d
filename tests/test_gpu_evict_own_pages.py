"""Eviction of sequences that keep their own pages: all of their tokens are in pages and fit the
budget, so that nothing moves, also where sequences share pages or their tables hold none behind
the last token."""
import numpy as np
import pytest
import torch

import ops_oracle
from cache_oracle import fill, i32
from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_own_pages_stay(D, f8):
    keep, S, lens = 200, 16, [200, 137, 1, 150, 400]
    cache = ops_oracle.Cache(5, 25, 2, D, S, f8, DEV, spare=15)
    fill(cache, lens, 3)
    cache.table[3, :6] = cache.table[1, :6]    # sequences that begin with the same pages
    cache.table[1, 9:] = -1                    # no page from the 144th token on
    cache.table[2, 1:] = cache.pages
    used = set(cache.table.flatten().tolist())
    out = cache.table[:, :13].clone()
    out[4] = i32([p for p in range(cache.pages) if p not in used][:13])
    w = torch.rand((5, 2, 400), generator=torch.Generator().manual_seed(1)).to(DEV)
    before = [cache.dense(b, n) for b, n in enumerate(lens)]
    raw = [x.view(torch.uint8).clone() for x in (cache.k, cache.v)]
    n, index, kept = spc.spc_kv_evict(*cache.args(i32(lens)), w, keep, out, first=3, recent=7,
                                      **cache.scales())
    assert n.tolist() == [200, 137, 1, 150, 200]
    for b in range(4):
        m = lens[b]
        want = torch.full((2, keep), -1, dtype=torch.int32)
        want[:, :m] = torch.arange(m, dtype=torch.int32)
        assert torch.equal(index[b].cpu(), want)
        assert torch.equal(kept[b, :, :m], w[b, :, :m])
    to = set(out[4].tolist())
    same = torch.tensor([p not in to for p in range(cache.pages)])
    for x, r in zip((cache.k, cache.v), raw):
        assert bool((x.view(torch.uint8) == r).flatten(1).all(1).cpu()[same].all())
    table, cache.table = cache.table, torch.cat([out, out[:, :12]], dim=1)
    k, v, there = cache.dense(4, keep)
    cache.table = table
    for h in range(2):
        at = index[4, h].cpu().numpy()
        assert there.all()
        np.testing.assert_array_equal(k[:, h], before[4][0][at, h])
        np.testing.assert_array_equal(v[:, h], before[4][1][at, h])

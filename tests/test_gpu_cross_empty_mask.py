"""Cross attention under masks of no tokens: every row that is some sequence's is zero."""
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


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [1, 20, 140])
def test_a_mask_of_no_tokens_masks_all(n, f8):
    lens = [300, 1500, 0]
    cache = ops_oracle.Cache(3, 100, 1, 128, 16, f8, DEV)
    fill(cache, lens, 4)
    q = randn((3, n, 4, 128), 2).to(DEV)
    for mask in (torch.ones((3, 0), dtype=torch.bool, device=DEV),
                 torch.ones((3, 9), dtype=torch.uint8, device=DEV)[:, 9:]):
        out = torch.full_like(q, 3.0)
        spc.spc_cross_attend(q, *cache.args(i32(lens)), key_mask=mask, out=out, **cache.scales())
        assert bool((out == 0).all())
    # ragged: rows of no sequence stay
    rows, start = q.flatten(0, 1), i32([1, n, n, 2 * n])
    out = torch.full_like(rows, 3.0)
    spc.spc_cross_attend(rows, *cache.args(i32(lens)), key_mask=mask, q_start=start, max_q=n, out=out,
                         **cache.scales())
    assert bool((out[1:2 * n] == 0).all()) and bool((out[:1] == 3).all()) and bool((out[2 * n:] == 3).all())


def test_captured_and_replayed():
    lens = i32([300, 200])
    cache = ops_oracle.Cache(2, 20, 1, 64, 16, False, DEV)
    fill(cache, [300, 200], 4)
    q = randn((2, 3, 4, 64), 2).to(DEV)
    mask = torch.ones((2, 0), dtype=torch.bool, device=DEV)
    out = torch.full_like(q, 3.0)
    spc.spc_cross_attend(q, *cache.args(lens), key_mask=mask, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spc.spc_cross_attend(q, *cache.args(lens), key_mask=mask, out=out)
    for _ in range(4):
        out.fill_(5.0)
        x = torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV)  # (eager work between)
        g.replay()
        torch.cuda.synchronize()
        assert bool((out == 0).all())
        del x

"""Weights read and written by one call, whose rows lie between each other in one buffer."""
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


def setup():
    lens = [130, 77, 0]
    cache = ops_oracle.Cache(3, 9, 2, 64, 16, False, DEV, spare=20)
    fill(cache, lens, 3)
    used = set(cache.table.flatten().tolist())
    other = i32([p for p in range(cache.pages) if p not in used][:9]).view(3, 3)
    w = torch.rand((3, 2, 130), generator=torch.Generator().manual_seed(2)).to(DEV)
    return cache, i32(lens), other, w


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("at,to", [(0, 130), (130, 270), (300, 10)])
def test_weigh(at, to, n):
    cache, lens, _, w = setup()
    q = randn((3, n, 4, 64), 1).to(DEV)
    want = spc.spc_kv_weigh(q, *cache.args(lens), w)
    wide = torch.full((3, 2, 430), 5.0, device=DEV)
    src, out = wide[..., at:at + 130], wide[..., to:to + 130]
    src.copy_(w)
    out.zero_()
    spc.spc_kv_weigh(q, *cache.args(lens), src, out=out)
    assert torch.equal(out, want) and torch.equal(src, w)


@pytest.mark.parametrize("at,to", [(0, 130), (0, 150), (48, 0), (60, 12)])
def test_evict(at, to):
    cache, lens, other, w = setup()
    n, index, kept = spc.spc_kv_evict(*cache.args(lens), w, 48, other, recent=5)
    wide = torch.full((3, 2, 200), 5.0, device=DEV)
    src, out = wide[..., at:at + 130], wide[..., to:to + 48]
    src.copy_(w)
    out.zero_()
    n2, index2, _ = spc.spc_kv_evict(*cache.args(lens), src, 48, other, recent=5, out_weights=out)
    assert torch.equal(n, n2) and torch.equal(index, index2) and torch.equal(out, kept)
    assert torch.equal(src, w)


@pytest.mark.parametrize("n", [1, 40])
def test_weigh_part_of_wider_rows(n):
    """Weights between others in wider rows, without an `out`."""
    cache, lens, _, w = setup()
    q = randn((3, n, 4, 64), 1).to(DEV)
    want = spc.spc_kv_weigh(q, *cache.args(lens), w)
    wide = torch.full((3, 2, 200), 5.0, device=DEV)
    wide[..., 31:161] = w
    got = spc.spc_kv_weigh(q, *cache.args(lens), wide[..., 31:161])
    assert torch.equal(got, want) and torch.equal(wide[..., 31:161], w)
    # and they can be the next call's
    again = spc.spc_kv_weigh(q, *cache.args(lens), got, out=got)
    assert again is got and torch.equal(got, spc.spc_kv_weigh(q, *cache.args(lens), want))

"""Weights where the workgroups of the second step, whose rows stay in LDS, go on to further keys
(33 to 128 rows a head over many keys), against the 64-bit definition.  The tolerance is that of
cache_oracle.weighed, for all rows of a head at once."""
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


def definition(q, cache, lens, old, window):
    """(weights, tolerance) [B][H][length] in float64."""
    B, n, heads, D = q.shape
    H, length, scale = cache.H, old.shape[2], D ** -0.5
    G = heads // H
    want, tol = torch.zeros((B, H, length), dtype=torch.double), torch.zeros((B, H, length), dtype=torch.double)
    host = q.cpu().double()
    for b in range(B):
        k, _, there = cache.dense(b, lens[b])
        t = torch.arange(lens[b])
        k, there = torch.from_numpy(k), torch.from_numpy(there)
        k = torch.where(there[:, None, None], k, 0.0)  # (what is in no page may be anything)
        at = torch.arange(lens[b] - n, lens[b]).repeat_interleave(G)
        see = there & (t <= at[:, None])
        if window:
            see &= t > at[:, None] - window
        for h in range(H):
            rows, keys = host[b, :, h * G:(h + 1) * G].reshape(n * G, D), k[:, h]
            s = (scale * (rows @ keys.T)).masked_fill(~see, -float("inf"))
            w = torch.softmax(s, dim=1)
            mag = (scale * (rows.abs() @ keys.abs().T)).masked_fill(~see, 0.0).amax(1, keepdim=True)
            delta = (D + 8) * 2.0 ** -24 * mag + 2.0 ** -21
            before = torch.where(t < lens[b] - n, old[b, h, :lens[b]].double(), 0.0)
            want[b, h, :lens[b]] = before + w.sum(0)
            tol[b, h, :lens[b]] = ((w * (2 * delta + (lens[b] + 64) * 2.0 ** -24)).sum(0)
                                   + want[b, h, :lens[b]].abs() * (n * G + 2) * 2.0 ** -24 + 1e-30)
    return want, tol * 1.01


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,window", [(17, 0), (64, 0), (40, 3001)])  # 34, 128 and 80 rows a head
def test_further_keys(n, window, D, f8):
    """Sixteen workgroups a head take the keys in turn, 4096 at a time: three turns and a part, two
    and a few keys of one wavefront, one whole, and less than one."""
    lens, H = [9001, 8192 + 70, 4096, 3333], 8
    cache = ops_oracle.Cache(4, 565, H, D, 16, f8, DEV, seed=n)
    fill(cache, lens, 3)
    cache.table[0, 300] = -1
    cache.table[1, 512] = cache.pages + 3
    q = randn((4, n, 2 * H, D), 5).to(DEV)
    old = torch.rand((4, H, 9040), generator=torch.Generator().manual_seed(6))
    got = spc.spc_kv_weigh(q, *cache.args(i32(lens)), old.to(DEV), window=window, **cache.scales()).cpu()
    want, tol = definition(q, cache, lens, old, window)
    d = (got.double() - want).abs()
    assert bool((d <= tol).all()), (float((d - tol).max()), float((d / (tol + 1e-40)).max()))
    for b in range(4):
        assert bool((got[b, :, lens[b]:] == 0).all())

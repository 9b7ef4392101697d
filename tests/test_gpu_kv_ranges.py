"""The attention (spc_kv_attend) at the ends of its arguments' ranges, against the
64-bit definition and against calls in the middle of them."""
import pytest
import torch

import ops_oracle
from paper_2405_19261_amd import spc
from test_gpu_kv import check_attend, fill, randn

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 30, 3])
@pytest.mark.parametrize("n,heads,D", [(16, 1, 64), (16, 2, 128), (150, 2, 128), (300, 1, 64)])
def test_windows_and_chunks_longer_than_the_cache(n, heads, D, window, f8):
    """Rows before position 0 see nothing and the others what they see without
    them, whatever the window: up to "no window" written as the largest one."""
    lens = [5, n - 1, 0, n + 40, 1]
    S = 16
    cache = ops_oracle.Cache(len(lens), (n + 40 + S - 1) // S, 1, D, S, f8, DEV)
    fill(cache, lens, 1)
    q = randn((len(lens), n, heads, D), 2).to(DEV)
    out, _ = check_attend(cache, q, lens, window=window)
    kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if window > n + 40:
        assert torch.equal(out, spc.spc_kv_attend(q, *cache.args(kv_len), **cache.scales()))
    assert bool((out[0, n - 5:] != 0).any(-1).all()) and bool((out[0, :n - 5] == 0).all())

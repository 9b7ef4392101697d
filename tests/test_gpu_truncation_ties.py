"""top-p over entries of one mass: "the fewest entries whose mass reaches top_p times
the mass of the first k" are then ceil(top_p * k) of them, however many."""
import numpy as np
import pytest
import torch

from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"
LEVELS = [0.0, 2.5, -3.7, 10.1, -20.3, 7.77, 30.0, -100.0]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def kept_of(z, T, k, p):
    kept = torch.empty(z.shape[0], dtype=torch.int32, device=DEV)
    u = torch.full((z.shape[0],), 0.4, device=DEV)
    spc.spc_sample(z.to(DEV), u, T, k, p, out_kept=kept)
    cut = spc.spc_truncate(z.to(DEV), T, k, p)
    assert torch.equal((cut > -float("inf")).sum(1).to(torch.int32), kept)
    return kept.cpu().numpy()


def count(p, n):
    """ceil(p n), exactly: p is a float32, n below 2^29."""
    return int(np.ceil(float(np.float32(p)) * n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [6, 1001, 32768, 32770, 131072, 256000, 262144])
def test_equal_logits(V, dtype):
    g = torch.Generator().manual_seed(V)
    z = torch.tensor(LEVELS).repeat(2)[:, None].expand(2 * len(LEVELS), V).clone()
    z[len(LEVELS):, torch.rand(V, generator=g) < 0.2] = float("-inf")
    z = z.to(dtype)
    live = (z > -float("inf")).sum(1).tolist()
    for T in (1.0, 0.7):
        for k in (0, V - 2, V // 8 * 4):
            for p in (0.5, 0.25, 0.9, 1 - 2.0 ** -24):
                want = [count(p, min(n, k) if k else n) for n in live]
                assert kept_of(z, T, k, p).tolist() == want, (T, k, p)


@pytest.mark.parametrize("V", [1001, 32767, 65535, 239517])
def test_temperatures_that_make_all_masses_equal(V):
    """Distinct logits whose masses differ by less than 2^-90."""
    g = torch.Generator().manual_seed(V)
    z = torch.stack([torch.randn(V, generator=g), torch.randn(V, generator=g) - 2000.0,
                     (torch.randn(V, generator=g) > 1).float() * 3 - 7])
    for T in (1e30, 3e38):
        for k in (0, V - 1, V - 2):
            for p in (0.5, 0.25, 0.999999):
                want = [count(p, k if k else V)] * 3
                assert kept_of(z, T, k, p).tolist() == want, (T, k, p)

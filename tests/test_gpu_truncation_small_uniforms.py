"""spc_sample at uniforms under the least share that the kernels' fixed-point
weights can hold (2^-50 of the largest, less in long rows): the token is still the
first kept one whose cumulative mass in 64 bits exceeds u times the total, so at
u = 0 the first kept one that has a mass."""
import numpy as np
import pytest
import torch

from test_gpu_truncation import check_sample

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


UNIFORMS = [0.0, 1e-45, 1e-30, 2.0 ** -60]
SETTINGS = [(1.0, 0, 1.0, 0.0), (0.05, 0, 1.0, 0.0), (0.5, 40, 1.0, 0.0), (1.0, 0, 1.0, 1e-30),
            (0.01, 0, 1.0, 0.0), (0.3, 3000, 1.0, 0.0)]


def rows(kind, V, dtype):
    """A few likely entries near the end; what comes before them by `kind`."""
    g = torch.Generator().manual_seed(V)
    z = {"noise": torch.randn(V, generator=g), "falling": -20.0 * torch.rand(V, generator=g) - 30.0,
         "rising": torch.linspace(-90.0, -5.0, V) + 0.01 * torch.randn(V, generator=g),
         "masked": torch.where(torch.rand(V, generator=g) < 0.9, float("-inf"),
                               -40.0 - torch.rand(V, generator=g))}[kind]
    z[V - 1 - V // 7] = 8.0
    z[V - 1] = 7.5
    return z.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("kind", ["noise", "falling", "rising", "masked"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 7, 1001, 8193, 32768, 32769, 150001])
def test_uniforms_below_a_unit(V, dtype, kind):
    z = rows(kind, V, dtype)
    for s in SETTINGS:
        n = len(UNIFORMS)
        check_sample(z.expand(n, V).contiguous(), np.array(UNIFORMS, np.float32), [s] * n)


@pytest.mark.parametrize("V", [3001, 70001])
def test_with_many_entries_in_question(V):
    """Rows that are read again and again (more entries of nearly one value than a
    list holds), and an unlikely entry before them all."""
    g = torch.Generator().manual_seed(1)
    z = 1e-3 * torch.randn(V, generator=g)
    z[0], z[1], z[2] = float("-inf"), -300.0, -60.0
    for s in ((1.0, V - 1, 1.0, 0.0), (1.0, V - 2, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1.0, V - 1, 1.0, 1e-28)):
        check_sample(z.expand(3, V).contiguous(), np.array([0.0, 1e-40, 1e-28], np.float32), [s] * 3)

"""Numbers as arguments of the truncation and cache calls (CPU: every call here
ends in the binding)."""
import numpy as np
import pytest
import torch

from paper_2405_19261_amd import spc

BIG = (1 << 31, (1 << 32) + 5, -(1 << 31) - 1)


def cache():
    k, v = torch.zeros((4, 2, 16, 64)), torch.zeros((4, 2, 64, 16))
    return (k.bfloat16(), v.bfloat16(), torch.zeros((3, 2), dtype=torch.int32),
            torch.zeros(3, dtype=torch.int32))


@pytest.mark.parametrize("x", BIG)
def test_integers_that_do_not_fit_are_refused(x):
    """They would reach the library modulo 2^32: top_k = 2^32 + 5 as 5."""
    z, u, q = torch.zeros(3, 50), torch.zeros(3), torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16)
    start = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: spc.spc_sample(z, u, top_k=x), lambda: spc.spc_truncate(z, top_k=x),
                 lambda: spc.spc_sample(z, u, top_k=x, temp_per_seq=u),
                 lambda: spc.spc_truncation_workspace_bytes(4, x, spc.SPC_BF16),
                 lambda: spc.spc_kv_attend(q, *cache(), window=x),
                 lambda: spc.spc_kv_attend(q.flatten(0, 1), *cache(), q_start=start, max_q=x),
                 lambda: spc.spc_kv_workspace_bytes(*cache(), x, 6),
                 lambda: spc.spc_kv_workspace_bytes(*cache(), 4, 6, x)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_lengths_that_do_not_fit_are_refused():
    with pytest.raises(ValueError, match="32 bits"):
        spc.spc_kv_read(*cache(), (1 << 32) + 5)
    out = torch.zeros(1, dtype=torch.bfloat16).expand(3, (1 << 32) + 5, 2, 64)
    with pytest.raises(ValueError, match="32 bits"):
        spc.spc_kv_read(*cache(), out=(out, out))


@pytest.mark.parametrize("shape", [(1, (1 << 32) + 1000), ((1 << 32) + 3, 1000)])
def test_rows_that_do_not_fit_are_refused(shape):
    """(Tensors on the meta device: sizes without memory.)"""
    z = torch.empty(shape, dtype=torch.bfloat16, device="meta")
    for call in (lambda: spc.spc_sample(z, temperature=0.0), lambda: spc.spc_truncate(z)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


@pytest.mark.parametrize("number", [np.float32, np.float64, torch.tensor, lambda x: np.array(x)])
def test_settings_of_any_number_type(number):
    """As the verify and drafter calls take theirs: these get as far as the tensors,
    which are the host's."""
    z, u, q = torch.zeros(3, 50), torch.zeros(3), torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16)
    kw = dict(temperature=number(0.5), top_p=number(0.75), min_p=number(0.25))
    for call in (lambda: spc.spc_sample(z, u, **kw), lambda: spc.spc_truncate(z, **kw),
                 lambda: spc.spc_sample(z, u, top_k_per_seq=torch.ones(3, dtype=torch.int32), **kw),
                 lambda: spc.spc_kv_attend(q, *cache(), scale=number(0.5))):
        with pytest.raises(ValueError, match="current HIP device"):
            call()
    cut = spc._truncation(kw["temperature"], np.int64(7), kw["top_p"], kw["min_p"], None, None, None,
                          None, z, 3)
    assert (cut.temperature, cut.top_k, cut.top_p, cut.min_p) == (0.5, 7, 0.75, 0.25)

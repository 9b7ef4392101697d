"""Outputs that would be written while the same call reads them as inputs are refused (CPU: every call
here fails its checks, so nothing is launched)."""
import pytest

from paper_2405_19261_amd import spc
from test_cache_refusals import evict, weigh
from test_ops_refusals import OK, cache

F = 4  # bytes of a float; the calls here: 3 sequences of 2 heads


@pytest.mark.parametrize("out,kw", [
    (1, {}), (63, {}), (64, {}), (383, {}), (-1, {}), (-191, {}), (-160, {}),
    # rows of 40, 64 apart: into the next row; and rows of 32 and 20, 64 and 100 apart
    (39, dict(length=40)), (33, dict(length=40)),
    (50, dict(length=32, keep=20, out_ld=100)), (-80, dict(length=32, keep=20, out_ld=100)),
])
def test_evicted_weights(out, kw):
    assert evict(cache(), out_w=OK + F * out, **kw) == -4
    assert "overlap" in spc.spc_last_error()


@pytest.mark.parametrize("n", [-2, -1, 0, 1, 2])
def test_evicted_lengths(n):
    assert evict(cache(), n=OK + F * n) == -4


@pytest.mark.parametrize("out,kw", [(1, {}), (63, {}), (-1, {}), (64, {}), (-128, {}), (383, {}),
                                    (30, dict(length=40)), (39, dict(length=40)), (25, dict(length=40))])
def test_weighed(out, kw):
    assert weigh(cache(), out=OK + F * out, **kw) == -4
    assert "overlap" in spc.spc_last_error()

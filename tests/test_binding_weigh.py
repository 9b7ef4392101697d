"""Calls of spc_kv_weigh that the binding answers or lays out itself (CPU: the library is a recorder)."""
import ctypes

import pytest
import torch

from paper_2405_19261_amd import spc


@pytest.fixture
def calls(monkeypatch):
    """spc_kv_weigh's (rows, first row of every sequence, most rows, weights, out, stride, length)."""
    seen = []

    class Library:
        def spc_kv_weigh(self, c, q, dtype, qs, heads, rows, start, most, scale, window, weights, out,
                         stride, length, ws, nbytes, stream):
            assert q
            start = start and [ctypes.c_int32.from_address(start + 4 * b).value for b in range(c.B + 1)]
            seen.append((rows, start, most, weights, out, stride, length))
            return 0

    monkeypatch.setattr(spc, "lib", lambda: Library())
    monkeypatch.setattr(spc, "_on_current_device", lambda t: None)
    monkeypatch.setattr(spc, "_stream", lambda s: 0)
    return seen


def cache(B=3, H=2, S=16, D=64, width=4, pages=12):
    k = torch.zeros((pages, H, S, D), dtype=torch.bfloat16)
    return (k, torch.zeros((pages, H, D, S), dtype=torch.bfloat16),
            torch.zeros((B, width), dtype=torch.int32), torch.full((B,), 40, dtype=torch.int32))


@pytest.mark.parametrize("ragged", [False, True])
def test_no_new_token(ragged, calls):
    """The weights as they were: a call whose only row is no sequence's."""
    q = torch.zeros((3, 0, 4, 64), dtype=torch.bfloat16)
    kw = dict(q_start=torch.zeros(4, dtype=torch.int32), max_q=5) if ragged else {}
    w = torch.rand((3, 2, 50))
    out = spc.spc_kv_weigh(q.flatten(0, 1) if ragged else q, *cache(), w, **kw)
    assert calls == [(1, [0, 0, 0, 0], 1, w.data_ptr(), out.data_ptr(), 50, 50)]


@pytest.mark.parametrize("B,H", [(3, 2), (3, 1), (1, 2), (1, 1)])
def test_weights_that_are_part_of_wider_rows(B, H, calls):
    """A new `out` has its rows at their stride."""
    q = torch.zeros((B, 1, 4, 64), dtype=torch.bfloat16)
    w = torch.rand((B, H, 70))[..., 3:53]
    out = spc.spc_kv_weigh(q, *cache(B, H), w)
    assert out.shape == w.shape and not bool(out.any())
    _, _, _, weights, to, stride, length = calls[0]
    assert (weights, to, length) == (w.data_ptr(), out.data_ptr(), 50)
    if B * H > 1:
        assert stride == 70 and (out.stride(1) if H > 1 else out.stride(0)) == 70
    # with weights of whole rows it is whole, as without any
    assert spc.spc_kv_weigh(q, *cache(B, H), w.contiguous()).is_contiguous()
    assert spc.spc_kv_weigh(q, *cache(B, H)).is_contiguous()

"""Masks of no tokens (CPU: the library is a recorder)."""
import ctypes

import pytest
import torch

from paper_2405_19261_amd import spc


def cache(B=3, H=2, S=16, D=64, width=4, pages=12):
    k = torch.zeros((pages, H, S, D), dtype=torch.bfloat16)
    return (k, torch.zeros((pages, H, D, S), dtype=torch.bfloat16),
            torch.zeros((B, width), dtype=torch.int32), torch.full((B,), 40, dtype=torch.int32))


@pytest.fixture
def masks(monkeypatch):
    """What spc_cross_attend is given: None, or the mask's rows as it reads them."""
    seen = []

    class Library:
        def spc_cross_attend(self, c, *a):
            mask, stride, width = a[8:11]
            seen.append(None if not mask else
                        [ctypes.string_at(mask + b * stride, width) for b in range(c.B)])
            return 0 if not mask or width >= 1 else -2

        def spc_last_error(self):
            return b"refused"

    monkeypatch.setattr(spc, "lib", lambda: Library())
    monkeypatch.setattr(spc, "_on_current_device", lambda t: None)
    monkeypatch.setattr(spc, "_stream", lambda s: 0)
    return seen


@pytest.mark.parametrize("dtype", [torch.bool, torch.uint8])
@pytest.mark.parametrize("make", [lambda t: torch.ones((3, 0), dtype=t),
                                  lambda t: torch.ones((3, 9), dtype=t)[:, :0],
                                  lambda t: torch.ones((3, 9), dtype=t)[:, 9:],
                                  lambda t: torch.ones((1, 0), dtype=t).expand(3, 0)])
def test_a_mask_of_no_tokens_masks_all(make, dtype, masks):
    """Tokens past a mask's width are masked: with a width of 0 all are."""
    q = torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16)
    spc.spc_cross_attend(q, *cache(), key_mask=make(dtype))
    assert masks[-1] is not None
    assert all(len(row) >= 1 and not any(row) for row in masks[-1])


def test_other_masks(masks):
    q = torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16)
    spc.spc_cross_attend(q, *cache())
    assert masks[-1] is None
    m = torch.tensor([[0, 1, 5], [1, 0, 0], [0, 0, 0]], dtype=torch.uint8)
    spc.spc_cross_attend(q, *cache(), key_mask=m)
    assert masks[-1] == [b"\0\1\5", b"\1\0\0", b"\0\0\0"]
    spc.spc_cross_attend(q, *cache(), key_mask=m[:1].expand(3, 3))
    assert masks[-1] == [b"\0\1\5"] * 3

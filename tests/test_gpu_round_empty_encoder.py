"""A decoding model whose encoder has no states for any sequence, or for some."""
import pytest
import torch

from paper_2405_19261_amd import decode


def model(lens, device, dtype=torch.bfloat16):
    base = decode.SyntheticLM(300, rows=32, seed=0, device=device)
    return decode.ContextLM(base, 3, 40, heads=8, kv_heads=2, head_dim=128, page_size=32, seed=6, mix=2.0,
                            cache_dtype=dtype, encoder_lens=lens)


def test_no_states_are_a_cache_of_some_page():
    """(CPU: the tensors that the calls will be given.)"""
    k, v, pages, lens = model([0, 0, 0], "cpu").encoder
    assert k.numel() and v.numel() and pages.shape == (3, 1) and lens.tolist() == [0, 0, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_no_states_add_nothing(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tokens = torch.tensor([[3, 5], [77, 1], [200, 9]], device="cuda")
    positions = torch.tensor([[0, 1]] * 3, device="cuda")
    got = [model(lens, "cuda", dtype)(tokens.view(-1), positions.view(-1)).view(3, 2, -1)
           for lens in ([0, 0, 0], None, [0, 40, 0])]
    assert torch.equal(got[0], got[1])
    assert torch.equal(got[2][[0, 2]], got[1][[0, 2]]) and not torch.equal(got[2][1], got[1][1])

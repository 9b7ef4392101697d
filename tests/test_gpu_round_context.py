"""Decoding rounds of models that begin with a prompt which all sequences share and that attend to an
encoder's states: one call's logits against float64 from the caches' own pages, rounds under
capture against eager ones, and rolling back."""
import numpy as np
import pytest
import torch

import ops_oracle
from paper_2405_19261_amd import decode, spc

pytestmark = pytest.mark.gpu
DEV = "cuda"
ENC = [40, 1, 133]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def models(V, max_len, dtype, prompt, mix=2.0):
    p = decode.SyntheticLM(V, rows=32, seed=0, device=DEV)
    q = p.derive(scale=0.8, sigma=1.0, seed=1)
    return (decode.ContextLM(q, 3, max_len, heads=2, kv_heads=1, seed=5, mix=mix, cache_dtype=dtype,
                             prompt=prompt),
            decode.ContextLM(p, 3, max_len, heads=8, kv_heads=2, head_dim=128, page_size=32, seed=6,
                             mix=mix, cache_dtype=dtype, prompt=prompt, encoder_lens=ENC))


def lines(k_pages, v_pages, scales, pages, n):
    """Keys and values [n, heads, dim] in float64 of the pages in a row."""
    t = torch.arange(n)
    S = k_pages.shape[2]
    page, slot = pages.cpu().long()[t // S], t % S
    k, v = (x.float().cpu().double() for x in (k_pages, v_pages))
    k, v = k[page, :, slot], v[page, :, :, slot]
    if scales:
        k = k * scales["k_scale"].cpu().double()[page, :, slot][..., None]
        v = v * scales["v_scale"].cpu().double()[page, :, slot][..., None]
    return k.numpy(), v.numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("prompt", [0, 32, 77, 500])
def test_logits(prompt, dtype):
    _, lm = models(500, 40, dtype, prompt)
    B, n, steps = 3, 5, 4
    for step in range(steps):  # chunks of 5 tokens, the last of them over the one before
        first = 5 * min(step, steps - 2)
        pos = (torch.arange(first, first + n, device=DEV)[None] + torch.tensor([[0], [2], [1]], device=DEV))
        tok = torch.randint(0, 500, (B, n), generator=torch.Generator().manual_seed(step)).to(DEV)
        z = lm(tok.view(-1), pos.view(-1)).double().cpu().numpy().reshape(B, n, -1)
    row = lm.base.row_of(tok.view(-1), pos.view(-1)).view(B, n).cpu()
    qs, cs = (t.cpu().double().numpy() for t in (lm.q_table, lm.cross_table))
    proj, cross = (t.cpu().double().numpy() for t in (lm.project, lm.cross_project))
    base = lm.base.logits_table.cpu().double().numpy()
    G, c = lm.heads // lm.kv_heads, lm.head_dim ** -0.5
    for b in range(B):
        total = prompt + int(pos[b, -1]) + 1
        k, v = lines(lm.k_pages, lm.v_pages, lm.scales, lm.page_table[b], total)
        if prompt:
            k[:prompt], v[:prompt] = lines(lm.k_pages, lm.v_pages, lm.scales, lm.shared_table, prompt)
        if dtype == torch.bfloat16:  # the chunk's own keys are where they belong
            np.testing.assert_array_equal(k[total - n:], lm.k_table.cpu().double().numpy()[row[b]])
        ek, ev = lines(*lm.encoder[:2], lm.encoder_scales, lm.encoder[2][b], ENC[b])
        for i in range(n):
            at, r = prompt + int(pos[b, i]), int(row[b, i])
            parts = []
            for q, K, V, last in ((qs, k, v, at), (cs, ek, ev, ENC[b])):
                o, tol = zip(*(ops_oracle.attend(q[r, g], K[:, g // G], V[:, g // G],
                                                 np.ones(len(K), bool), 0, last, c)
                               for g in range(lm.heads)))
                parts.append((np.concatenate(o), np.concatenate(tol)))
            (o, to), (x, tx) = parts
            z1, z2 = o @ proj, x @ cross
            # products in bfloat16 with sums in 32 bits, rounded; their sums, rounded
            e = to @ np.abs(proj) + tx @ np.abs(cross) + len(o) * 2.0 ** -23 * (
                np.abs(o) @ np.abs(proj) + np.abs(x) @ np.abs(cross)) + 2.0 ** -8 * (np.abs(z1) + np.abs(z2))
            want = base[r] + z1 + z2
            e += 2.0 ** -8 * (np.abs(z1 + z2) + np.abs(want) + 2 * e)
            assert (np.abs(z[b, i] - want) <= e * 1.01).all(), (b, i)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("prompt", [0, 100])
def test_rounds_captured_and_eager(prompt, dtype):
    first = torch.tensor([3, 77, 200], dtype=torch.int32)
    runs = []
    for graph in (False, True, True):
        q, p = models(300, 60, dtype, prompt)
        runs.append(decode.spec_decode(q, p, first, 8, 3, spc.SPC_RULE_DIFF, 0.05, 0.9, seed=4, graph=graph,
                                       top_k=40))
    for r in runs[1:]:
        assert r.tokens == runs[0].tokens
    # (what the models condition on matters)
    q, p = models(300, 60, dtype, prompt + 16)
    other = decode.spec_decode(q, p, first, 8, 3, spc.SPC_RULE_DIFF, 0.05, 0.9, seed=4, top_k=40)
    assert other.tokens != runs[0].tokens


def test_prompts_and_what_the_cache_holds():
    lm = models(300, 60, torch.bfloat16, 77)[1]
    assert lm.cache_tokens == 160 - 77  # pages of 32: 137 tokens take five
    with pytest.raises(RuntimeError, match="cache holds"):
        q, p = models(300, 20, torch.bfloat16, 77)
        decode.spec_decode(q, p, torch.zeros(3, dtype=torch.int32), 30, 4, spc.SPC_RULE_ALWAYS, 0.0, 1.0)

"""A decoding round's operators together, as decode.py runs them: models with a
paged KV cache (write, attend), truncated drafts (sample), truncated rows
(truncate), the verification, and rolling back.  Every recorded round is
checked against the 64-bit definitions on its own inputs."""
import numpy as np
import pytest
import torch

import ops_oracle
import oracle
from decode_oracle import _host
from paper_2405_19261_amd import decode
from paper_2405_19261_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def models(B, V, max_len, dtype, seed=0, mix=2.0):
    p = decode.SyntheticLM(V, rows=32, seed=seed, device=DEV)
    q = p.derive(scale=0.8, sigma=1.0, seed=seed + 1)
    return (decode.ContextLM(q, B, max_len, heads=2, kv_heads=1, seed=5, mix=mix, cache_dtype=dtype),
            decode.ContextLM(p, B, max_len, heads=8, kv_heads=2, head_dim=128, page_size=32, seed=6,
                             mix=mix, cache_dtype=dtype))


def expected_rows(lm, tokens, positions):
    """A ContextLM's logits after each of `tokens` (a whole prefix, positions
    0 ..), and a tolerance, in float64 from its tables alone."""
    row = lm.base.row_of(torch.tensor(tokens, device=DEV), torch.arange(len(tokens), device=DEV)).cpu()
    q, k, v = (t.cpu().double().numpy()[row] for t in (lm.q_table, lm.k_table, lm.v_table))
    if lm.scales:
        k, v = (c * s[..., None].astype(np.float64) for c, s in
                (ops_oracle.quantised(x.astype(np.float32)) for x in (k, v)))
    proj = lm.project.cpu().double().numpy()
    base = lm.base.logits_table.cpu().double().numpy()[row]
    out = []
    for t in positions:
        o, tol = zip(*(ops_oracle.attend(q[t, g], k[:, g // (lm.heads // lm.kv_heads)],
                                         v[:, g // (lm.heads // lm.kv_heads)], np.ones(len(k), bool),
                                         0, t, lm.head_dim ** -0.5) for g in range(lm.heads)))
        o, tol = np.concatenate(o), np.concatenate(tol)
        z, mag = o @ proj, np.abs(o) @ np.abs(proj)
        # the product in bfloat16 with sums in 32 bits, rounded; then the sum, rounded
        e = tol @ np.abs(proj) + len(o) * 2.0 ** -24 * mag + 2.0 ** -8 * np.abs(z)
        want = base[t] + z
        out.append((want, e + 2.0 ** -8 * (np.abs(want) + e)))
    return out


CUTS = [dict(top_k=40), dict(top_p=0.9), dict(top_k=60, top_p=0.95, min_p=0.01), {}]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("cut", CUTS)
def test_rounds_with_a_cache_and_truncation(cut, dtype):
    B, V, gamma, rounds = 4, 5003, 4, 5
    drafter, verifier = models(B, V, rounds * (gamma + 1) + gamma + 2, dtype)
    first = torch.tensor([3, 17, 99, 4000], device=DEV)
    T, rounds_in = 0.9, []
    res = decode.spec_decode(drafter, verifier, first, rounds, gamma, W.ALWAYS, 0.0, T, seed=3,
                             rounds_inputs=rounds_in, **cut)
    k, tp, mp = cut.get("top_k", 0), float(np.float32(cut.get("top_p", 1.0))), float(np.float32(cut.get("min_p", 0.0)))
    Tf = float(np.float32(T))
    done = [0] * B
    for r, x in enumerate(rounds_in):
        q, p, draft, u = (x[n].cpu() for n in ("q", "p", "draft", "uniforms"))
        for b in range(B):
            prefix = [int(first[b])] + res.tokens[b][:done[b]]
            block = prefix + draft[b].tolist()
            at = range(len(prefix) - 1, len(block))
            # the models saw exactly this prefix, whatever earlier rounds had drafted past it
            for lm, rows in ((drafter, q[b]), (verifier, p[b])):
                for j, (want, tol) in enumerate(expected_rows(lm, block, at)):
                    d = np.abs(rows[j].double().numpy() - want)
                    assert (d <= tol).all(), (r, b, j, float((d - tol).max()))
            for j in range(gamma):
                t, _, _ = ops_oracle.sample(q[b, j].float().numpy(), float(x["u_draft"][j, b]), Tf, k, tp, mp)
                if cut:
                    assert int(draft[b, j]) == t
            done[b] += int(res.accept_len[r][b]) + 1
        if cut:
            cutrow = lambda z: torch.from_numpy(  # noqa: E731
                np.stack([[ops_oracle.truncated(z[b, j].float().numpy(), Tf, k, tp, mp)
                           for j in range(gamma + 1)] for b in range(B)])).to(torch.bfloat16)
            q, p = cutrow(q), cutrow(p)
        o = oracle.verify(_host(q.contiguous()), _host(p.contiguous()), draft.numpy(), u.numpy(),
                          np.full(B, W.ALWAYS, np.int32), np.zeros(B, np.float32),
                          np.full(B, T, np.float32))
        np.testing.assert_array_equal(o["accept_len"], res.accept_len[r].numpy())
    for b in range(B):
        assert len(res.tokens[b]) == done[b]


def test_truncated_tokens_lie_in_the_verifiers_kept_sets():
    """With delta = 1 the emitted tokens follow the truncated verifier: each lies
    in its row's kept set; with identical models every draft is kept."""
    B, V, gamma = 3, 2000, 3
    p = decode.SyntheticLM(V, rows=16, seed=1, device=DEV)
    lms = [decode.ContextLM(p, B, 64, seed=2) for _ in range(2)]
    rounds_in = []
    res = decode.spec_decode(lms[0], lms[1], torch.arange(B, device=DEV), 4, gamma, W.ALWAYS, 0.0,
                             1.0, rounds_inputs=rounds_in, top_k=torch.tensor([5, 0, 20]),
                             top_p=torch.tensor([1.0, 0.7, 0.9]))
    for r, x in enumerate(rounds_in):
        for b, (k, tp) in enumerate(((5, 1.0), (0, 0.7), (20, 0.9))):
            n = int(res.accept_len[r][b])
            tok = res.tokens[b][sum(int(a[b]) + 1 for a in res.accept_len[:r]):][:n + 1]
            for j, t in enumerate(tok):
                kept, _ = ops_oracle.kept_set(ops_oracle.cleaned(x["p"][b, j].float().cpu().numpy()), 1.0,
                                              k, float(np.float32(tp)))
                assert t in kept


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_graph_rounds_equal_eager_rounds(dtype):
    B, V, gamma, rounds = 4, 40000, 3, 6
    first = torch.tensor([1, 2, 3, 4], device=DEV)
    T = torch.tensor([1.0, 0.0, 0.7, 1.0])
    kw = dict(top_k=torch.tensor([50, 0, 0, 10]), top_p=torch.tensor([1.0, 1.0, 0.9, 0.8]),
              min_p=torch.tensor([0.0, 0.0, 0.0, 0.02]))
    rule = torch.tensor([W.DIFF, W.OPT, W.TOKEN_V3, W.CHOW])
    alpha = torch.tensor([0.05, 0.1, 0.3, 0.4])
    runs = []
    for graph in (False, True):
        drafter, verifier = models(B, V, rounds * (gamma + 1) + gamma + 2, dtype)
        runs.append(decode.spec_decode(drafter, verifier, first, rounds, gamma, rule, alpha, T,
                                       seed=9, graph=graph, **kw))
    assert runs[0].tokens == runs[1].tokens
    assert [a.tolist() for a in runs[0].accept_len] == [a.tolist() for a in runs[1].accept_len]

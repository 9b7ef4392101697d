"""Truncated decoding rounds under every target of the verification: each round's
accept lengths and new tokens against the oracle on rows truncated by the 64-bit
definition (near-ties as in parity.py)."""
from collections import Counter

import numpy as np
import pytest
import torch

import oracle
import ops_oracle
import parity
from paper_2405_19261_amd import decode
from paper_2405_19261_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"

RULES = [(W.CHOW, 0.4), (W.DIFF, 0.05), (W.OPT, 0.1), (W.ALWAYS, 0.0), (W.NEVER, 0.0),
         (W.TOKEN_V1, 0.3), (W.TOKEN_V2, 0.3), (W.TOKEN_V3, 0.3), (W.LOSSY, 0.3), (W.BILD, 2.0),
         (W.CHOWLOG, 1.0), (W.DIFFLOG, 0.1), (W.OPTLOG, 0.1)]
CUTS = [dict(top_k=20), dict(top_p=0.8), dict(top_k=200, top_p=0.95, min_p=0.02)]
T = float(np.float32(0.9))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def cut_rows(z, cut):
    """Rows [B][rows][V] as the verification gets them."""
    s = (cut.get("top_k", 0), float(np.float32(cut.get("top_p", 1.0))),
         float(np.float32(cut.get("min_p", 0.0))))
    rows = z.reshape(-1, z.shape[-1])
    out = np.stack([ops_oracle.truncated(r.float().numpy(), T, *s) for r in rows])
    return torch.from_numpy(out).to(z.dtype).view(z.shape)


def check_rounds(rounds_in, res, cut, greedy=None):
    """Every recorded round against the oracle; greedy marks sequences at
    temperature 0, whose rows are not truncated."""
    B = len(res.tokens)
    done, rep = [0] * B, Counter()
    for r, x in enumerate(rounds_in):
        q, p = x["q"].cpu(), x["p"].cpu()
        h = dict(q=parity.host_logits(cut_rows(q, cut)), p=parity.host_logits(cut_rows(p, cut)),
                 draft=x["draft"].cpu().numpy(), uniforms=x["uniforms"].cpu().numpy(),
                 rule=x["rule"].cpu().numpy(), alpha=x["alpha"].cpu().numpy(),
                 temperature=np.full(B, T, np.float32))
        acc = res.accept_len[r].numpy()
        tok = np.array([res.tokens[b][done[b] + int(acc[b])] for b in range(B)], np.int32)
        kept = [res.tokens[b][done[b]:done[b] + int(acc[b])] for b in range(B)]
        for b in range(B):
            assert kept[b] == h["draft"][b, :int(acc[b])].tolist()
            done[b] += int(acc[b]) + 1
        sel = np.ones(B, bool) if greedy is None else ~greedy
        h = {k: v[sel] for k, v in h.items()}
        o = parity.run_oracle(h)
        # (the rounds report no defer decisions: the oracle's own stand in)
        parity.compare(dict(accept_len=acc[sel], next_token=tok[sel], defer=o["defer"]), o, h, "bf16",
                       rep=rep)
        if greedy is not None:
            g = {k: v[greedy] for k, v in dict(
                q=parity.host_logits(q), p=parity.host_logits(p), draft=x["draft"].cpu().numpy(),
                rule=x["rule"].cpu().numpy(), alpha=x["alpha"].cpu().numpy()).items()}
            o = oracle.greedy_verify(*(g[k] for k in ("q", "p", "draft", "rule", "alpha")))
            np.testing.assert_array_equal(acc[greedy], o["accept_len"])
            np.testing.assert_array_equal(tok[greedy], o["next_token"])
    assert [len(t) for t in res.tokens] == done
    return rep


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("rule,alpha", RULES)
def test_rounds_under_every_rule(rule, alpha, cut):
    B, V, gamma = 6, 3001, 4
    p = decode.SyntheticLM(V, rows=32, seed=rule, device=DEV)
    q = p.derive(scale=0.8, sigma=1.0, seed=rule + 1)
    rounds_in = []
    res = decode.spec_decode(q, p, torch.arange(B, device=DEV), 5, gamma, rule, alpha, T, seed=rule,
                             rounds_inputs=rounds_in, **cut)
    rep = check_rounds(rounds_in, res, cut)
    assert rep["exact"] >= 5 * B - 1


@pytest.mark.parametrize("V", [3001, 40000])
def test_rounds_of_mixed_rules_and_greedy_sequences(V):
    """A rule a sequence, every third sequence at temperature 0; rows that a
    workgroup holds and rows in slices."""
    B, gamma, cut = len(RULES), 3, CUTS[2]
    p = decode.SyntheticLM(V, rows=32, seed=21, device=DEV)
    q = p.derive(scale=0.8, sigma=1.0, seed=22)
    greedy = np.arange(B) % 3 == 0
    rounds_in = []
    res = decode.spec_decode(q, p, torch.arange(B, device=DEV), 3, gamma,
                             torch.tensor([r for r, _ in RULES]), torch.tensor([a for _, a in RULES]),
                             torch.tensor(np.where(greedy, 0.0, T)), seed=5, rounds_inputs=rounds_in,
                             **cut)
    check_rounds(rounds_in, res, cut, greedy)

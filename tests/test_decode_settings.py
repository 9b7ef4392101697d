"""What a run of the decoding loop makes of its settings: on the CPU with a
GpuBackend whose sampling and verification are replaced, so that nothing
reaches the library; on the GPU by the tokens."""
import pytest
import torch

from paper_2405_19261_amd import decode
from paper_2405_19261_amd import workloads as W

B, V = 3, 50


class Recorder(decode.GpuBackend):
    """Greedy drafts, none kept; the truncation that each call saw."""

    def __init__(self):
        super().__init__()
        self.cuts = []

    def draft_sample(self, logits, temperature, uniforms):
        self.cuts.append(self._cut)
        return logits.float().argmax(1).to(torch.int32)

    def verify(self, q, p, drafts, uniforms, rule, alpha, temperature):
        self.cuts.append(self._cut)
        n = q.shape[0]
        return torch.zeros(n, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)


def run(backend, n=B, **kw):
    lm = decode.SyntheticLM(V, rows=4, device="cpu")
    backend.cuts.clear()
    res = decode.spec_decode(lm, lm, torch.zeros(n, dtype=torch.long), rounds=2, gamma=2,
                             rule=W.ALWAYS, alpha=0.0, temperature=1.0, backend=backend, **kw)
    assert len(backend.cuts) == 2 * 3
    return res


@pytest.mark.parametrize("cut", [dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1),
                                 dict(top_k=torch.tensor([0, 3, 7]))])
def test_truncation_holds_for_one_run(cut):
    """A backend that ran truncated rounds runs whole distributions next, for
    another number of sequences too, and truncated ones again."""
    backend = Recorder()
    for _ in range(2):
        run(backend, **cut)
        assert all(c is not None for c in backend.cuts)
        top_k = torch.as_tensor(cut.get("top_k", 0), dtype=torch.int32).expand(B)
        assert all(torch.equal(c["top_k_per_seq"], top_k) for c in backend.cuts)
        run(backend)
        assert all(c is None for c in backend.cuts)
        run(backend, n=B + 2)
        assert all(c is None for c in backend.cuts)


@pytest.mark.gpu
def test_a_used_backend_decodes_as_a_new_one():
    p = decode.SyntheticLM(2000, rows=16, seed=1, device="cuda")
    q = p.derive(seed=2)
    first = torch.arange(4, device="cuda")

    def run_on(backend, **kw):
        return decode.spec_decode(q, p, first, 6, 3, W.ALWAYS, 0.0, 1.0, seed=7, backend=backend,
                                  **kw).tokens

    used = decode.GpuBackend()
    cut = run_on(used, top_k=3)
    whole = run_on(used)
    assert whole == run_on(decode.GpuBackend()) and whole != cut
    assert run_on(used, top_k=3) == cut

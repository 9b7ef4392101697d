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


NAN = float("nan")


@pytest.mark.parametrize("cut,b", [
    (dict(top_k=-1), 0), (dict(top_p=0.0), 0), (dict(top_p=1.5), 0), (dict(min_p=-0.1), 0),
    (dict(min_p=1.1), 0), (dict(top_p=NAN), 0), (dict(min_p=NAN), 0),
    (dict(top_k=torch.tensor([5, 0, -2])), 2), (dict(top_p=torch.tensor([1.0, 0.0, 0.5])), 1),
    (dict(top_k=4, min_p=torch.tensor([0.0, 1.0, 2.0])), 2)])
def test_settings_out_of_range_are_an_error(cut, b):
    """Not rounds of rows without an entry; and the backend goes on without them."""
    backend = Recorder()
    with pytest.raises(ValueError, match=f"sequence {b}:"):
        run(backend, **cut)
    assert backend.cuts == []
    run(backend)
    assert all(c is None for c in backend.cuts)


class Bounded:
    """A model with a cache of `capacity` tokens a sequence, noting how far it was called."""

    def __init__(self, capacity):
        self.lm, self.device = decode.SyntheticLM(V, rows=4, device="cpu"), torch.device("cpu")
        self.cache_tokens, self.reached = capacity, 0

    def __call__(self, last, positions):
        self.reached = max(self.reached, int(positions.max()) + 1)
        return self.lm(last, positions)


class Keeper(Recorder):
    """All drafts kept by sequence 0, none by the others."""

    def verify(self, q, p, drafts, *rest):
        acc = torch.zeros(len(q), dtype=torch.int32)
        acc[0] = drafts.shape[1]
        return acc, torch.zeros(len(q), dtype=torch.int32)


@pytest.mark.parametrize("backend,reached", [(Recorder, 3 + 5), (Keeper, 4 * 5)])
def test_rounds_past_a_cache_are_an_error(backend, reached):
    """4 rounds of gamma = 4: one token a round, or five.  A cache that just holds
    what the rounds reached is enough, whatever more they might have taken."""
    def decode_with(*capacities):
        lms = [Bounded(c) for c in capacities]
        decode.spec_decode(*lms, torch.zeros(B, dtype=torch.long), rounds=4, gamma=4, rule=W.ALWAYS,
                           alpha=0.0, temperature=1.0, backend=backend())
        assert all(lm.reached == reached for lm in lms)

    decode_with(reached, reached)
    for name, c in (("drafter", (reached - 1, reached)), ("verifier", (reached, reached - 1))):
        with pytest.raises(RuntimeError, match=f"{name}'s cache holds {reached - 1}"):
            decode_with(*c)


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


def test_a_context_model_holds_whole_pages():
    lm = decode.ContextLM(decode.SyntheticLM(V, rows=4, device="cpu"), B, 33, page_size=16)
    assert lm.cache_tokens == 48


@pytest.mark.gpu
def test_rounds_past_a_context_models_cache_are_an_error():
    p = decode.SyntheticLM(500, rows=16, seed=1, device="cuda")

    def run_in(tokens, rounds, graph):
        lms = [decode.ContextLM(p, 2, tokens, seed=3) for _ in range(2)]
        return decode.spec_decode(*lms, torch.arange(2, device="cuda"), rounds, 3, W.ALWAYS, 0.0, 1.0,
                                  graph=graph).tokens

    for graph in (False, True):  # (every draft of an identical model is kept: 4 tokens a round)
        assert run_in(16, 4, graph) == run_in(160, 4, graph)
        with pytest.raises(RuntimeError, match="cache holds 16"):
            run_in(16, 5, graph)

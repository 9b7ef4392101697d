"""Speculative-cascade decoding: GenSpecSample (Alg. 4) run round after round.

Each round, for every sequence b of the batch:

  1. drafts gamma tokens auto-regressively from the drafter,
     x_{t+j} ~ q(.|x_{<t+j}), j = 0..gamma-1 (``spc_draft_sample``), and takes
     the drafter's logits at the extra position t+gamma as well (the target
     at that position needs q_{t+gamma});
  2. scores the gamma+1 prefixes x_{<t}, ..., x_{<t+gamma} with the verifier
     in one batch;
  3. verifies the block (``spc_verify`` with the chosen target): the first
     rejection j*, and the token that replaces it (or the extra token when
     every draft is kept);
  4. emits x_t .. x_{t+j*-1} and the new token, and rolls back to t+j*+1:
     the drafts past j* are discarded, and the next round starts from the
     emitted token.

Models are callables ``logits_for(last_tokens, positions) -> [n, V]``: the
next-token logits given the last token and its position.  A real language
model conditions on the whole prefix through its KV cache; rolling back is
then truncating that cache to t + j* + 1.  ``SyntheticLM`` is such a callable
with seeded logits, standing in for the paper's drafter/verifier pairs,
whose weights are not used here.  ``ContextLM`` adds a paged KV cache to it:
its logits depend on every token before them through one attention layer
(``spc_kv_write``, ``spc_kv_attend``), one token at a time as a drafter and
gamma + 1 at a time as a verifier; behind a prompt that all sequences share
(``spc_kv_attend_shared``) and with an encoder's states (``spc_cross_attend``)
where it is given them.

With ``top_k``, ``top_p`` or ``min_p`` the drafts come from the drafter's
truncated distribution (``spc_sample``) and the verification sees both models'
rows truncated alike (``spc_truncate``), so that it still is exact.

The backend does the sampling and verification.  ``GpuBackend`` calls the C
library; a test may pass any object with the same two methods.
"""
from dataclasses import dataclass, field

import torch

from . import spc


class SyntheticLM:
    """Seeded next-token logits that depend on (last token, position):
    ``rows`` logit rows, each a Zipf(s) ranking over a per-row random
    permutation of the vocabulary plus N(0, noise^2), and the row for a
    context chosen by a hash of (token, position).  ``derive`` makes a model
    whose rows are ``scale`` times this model's rows plus fresh N(0, sigma^2)
    noise, i.e. a drafter that mostly agrees with its verifier."""

    def __init__(self, V, rows=64, s=1.2, noise=1.0, seed=0, dtype=torch.bfloat16,
                 device="cuda", table=None):
        self.V, self.rows, self.dtype, self.device = V, rows, dtype, torch.device(device)
        if table is None:
            g = torch.Generator(device="cpu").manual_seed(seed)
            rank = torch.argsort(torch.rand(rows, V, generator=g), dim=1).float() + 1.0
            table = -s * torch.log(rank) + noise * torch.randn(rows, V, generator=g)
        self.table = table.to(self.device, torch.float32)
        self.logits_table = self.table.to(dtype).contiguous()

    def derive(self, scale=0.8, sigma=1.0, seed=1):
        g = torch.Generator(device="cpu").manual_seed(seed)
        t = scale * self.table.cpu() + sigma * torch.randn(self.rows, self.V, generator=g)
        return SyntheticLM(self.V, self.rows, dtype=self.dtype, device=self.device, table=t)

    def row_of(self, last_tokens, positions):
        h = (last_tokens.long() * 1000003 + positions.long() * 7919) % self.rows
        return h.to(self.device)

    def __call__(self, last_tokens, positions):
        return self.logits_table.index_select(0, self.row_of(last_tokens, positions))


class ContextLM:
    """A SyntheticLM whose logits also depend on the tokens before the last
    one: ``base``'s row plus ``mix`` times a projection of one attention layer
    over a paged KV cache of its own.  A token's query, key and value are rows
    of seeded tables picked as its logit row is, by a hash of (token,
    position).  The cache holds up to ``max_len`` tokens of each of ``B``
    sequences in pages of ``page_size``, in bfloat16 or (``cache_dtype``
    torch.float8_e4m3fn) quantised as it is written.

    A call takes n tokens of every sequence, [B * n] (sequence by sequence,
    at consecutive positions), writes their keys and values and attends from
    all of them.  A position that comes again overwrites what it held, and a
    call reads no further than its last position: rolling back needs no more
    than going on from an earlier position.  A token at or past
    ``cache_tokens`` (``max_len`` in whole pages) is not kept: ``spec_decode``
    raises after rounds that came that far; one's own calls stay below.

    ``prompt`` tokens that all sequences begin with (seeded keys and values) stand
    in pages of their own, before position 0, and every call reads them once for
    the whole batch (``spc_kv_attend_shared``).  ``encoder_lens`` (B lengths) makes
    the model a decoder with an encoder's states of its own for each sequence, to
    which a second layer attends (``spc_cross_attend``)."""

    def __init__(self, base, B, max_len, heads=4, kv_heads=2, head_dim=64, page_size=16,
                 cache_dtype=torch.bfloat16, mix=1.0, seed=0, prompt=0, encoder_lens=None):
        self.base, self.B, self.V, self.device = base, B, base.V, base.device
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        g = torch.Generator(device="cpu").manual_seed(seed)

        def table(*shape, s=1.0):
            return (torch.randn(*shape, generator=g) * s).to(self.device, torch.bfloat16)

        self.q_table = table(base.rows, heads, head_dim)
        self.k_table = table(base.rows, kv_heads, head_dim)
        self.v_table = table(base.rows, kv_heads, head_dim)
        self.project = table(heads * head_dim, base.V, s=mix * (heads * head_dim) ** -0.5)
        # pages of a sequence of its own, from the one that the prompt ends in
        begin = prompt // page_size
        width = (prompt + max_len + page_size - 1) // page_size - begin
        self.prompt, self.cache_tokens = prompt, (begin + width) * page_size - prompt
        shared = (prompt + page_size - 1) // page_size
        # pages in a seeded order, as an allocator leaves them after a while
        order = torch.randperm(B * width + shared, generator=g).to(self.device, torch.int32)
        self.shared_table = order[B * width:].contiguous()
        self.page_table = torch.cat([self.shared_table[:begin].expand(B, begin),
                                     order[:B * width].view(B, width)], dim=1).contiguous()
        self.k_pages, self.v_pages, self.scales = self._pages(order.numel(), page_size, cache_dtype)
        if prompt:
            self._write(g, self.k_pages, self.v_pages, self.shared_table[None], [prompt], self.scales)
        self.encoder = None
        if encoder_lens is not None:
            lens = [int(x) for x in encoder_lens]
            w = (max(1, *lens) + page_size - 1) // page_size  # (of no states too, a page)
            pages = torch.randperm(B * w, generator=g).view(B, w).to(self.device, torch.int32)
            k, v, scales = self._pages(B * w, page_size, cache_dtype)
            self._write(g, k, v, pages, lens, scales)
            self.encoder = (k, v, pages, torch.tensor(lens, dtype=torch.int32, device=self.device))
            self.encoder_scales = scales
            self.cross_table = table(base.rows, heads, head_dim)
            self.cross_project = table(heads * head_dim, base.V, s=mix * (heads * head_dim) ** -0.5)

    def _pages(self, n, page_size, dtype):
        """Zeroed pages for keys and for values, and their scales (of 8 bits)."""
        shape = (n, self.kv_heads, page_size, self.head_dim)
        k = torch.zeros(shape, device=self.device, dtype=dtype)
        v = torch.zeros((n, self.kv_heads, self.head_dim, page_size), device=self.device, dtype=dtype)
        scales = {}
        if dtype == torch.float8_e4m3fn:
            scales = {name: torch.zeros(shape[:3], device=self.device)
                      for name in ("k_scale", "v_scale")}
        return k, v, scales

    def _write(self, g, k_pages, v_pages, table, lens, scales):
        """Seeded tokens 0 .. lens[b] - 1 of every sequence into their pages."""
        k, v = (torch.randn(sum(lens), self.kv_heads, self.head_dim, generator=g).to(
            self.device, torch.bfloat16) for _ in range(2))
        start = torch.tensor([sum(lens[:b]) for b in range(len(lens) + 1)], dtype=torch.int32)
        spc.spc_kv_write(k, v, k_pages, v_pages, table.contiguous(), start.diff().to(self.device),
                         q_start=start.to(self.device), **scales)

    def __call__(self, last_tokens, positions):
        B, n = self.B, last_tokens.numel() // self.B
        row = self.base.row_of(last_tokens, positions)

        def of(t):
            return t.index_select(0, row).view(B, n, t.shape[1], t.shape[2])

        kv_len = (positions.view(B, n)[:, -1] + (self.prompt + 1)).to(torch.int32)
        cache = (self.k_pages, self.v_pages, self.page_table, kv_len)
        spc.spc_kv_write(of(self.k_table), of(self.v_table), *cache, **self.scales)
        if self.prompt:
            o = spc.spc_kv_attend_shared(of(self.q_table), *cache, self.prompt,
                                         shared_table=self.shared_table, **self.scales)
        else:
            o = spc.spc_kv_attend(of(self.q_table), *cache, **self.scales)
        z = torch.matmul(o.view(B * n, -1), self.project)
        if self.encoder is not None:
            c = spc.spc_cross_attend(of(self.cross_table), *self.encoder, **self.encoder_scales)
            z = z + torch.matmul(c.view(B * n, -1), self.cross_project)
        return self.base.logits_table.index_select(0, row) + z.to(self.base.dtype)


class GpuBackend:
    """Sampling and verification through libspeccascade.

    ``prepare`` (called once by ``spec_decode`` before the rounds) reads the
    per-sequence parameters on the host.  When every sequence shares one
    rule, alpha and temperature the calls take the scalar forms, so the
    library launches only the kernels that rule needs (no argmax at T > 0);
    otherwise the per-sequence arrays go with the ``rules_present`` mask of
    the rules they hold.

    ``truncate`` (called before ``prepare`` where the rounds are truncated)
    takes top_k, top_p and min_p as [B] tensors and raises on values out of
    range, whose sequences the library would leave without a token.  They hold
    for one run: the next ``prepare`` without a ``truncate`` before it leaves
    distributions whole again."""

    def __init__(self):
        self._scalar = None
        self._rules_present = 0
        self._cut = self._next_cut = None

    def truncate(self, top_k, top_p, min_p):
        k, p, m = top_k.cpu(), top_p.cpu(), min_p.cpu()
        bad = (~((k >= 0) & (p > 0) & (p <= 1) & (m >= 0) & (m <= 1))).nonzero()
        if bad.numel():
            b = int(bad[0])
            raise ValueError(f"sequence {b}: top_k must be >= 0, top_p in (0, 1] and min_p in [0, 1] "
                             f"(got {int(k[b])}, {float(p[b]):g} and {float(m[b]):g})")
        self._cut = self._next_cut = dict(top_k_per_seq=top_k, top_p_per_seq=top_p,
                                          min_p_per_seq=min_p)

    def prepare(self, rule, alpha, temperature):
        self._cut, self._next_cut = self._next_cut, None
        r, a, t = rule.cpu(), alpha.cpu(), temperature.cpu()
        self._rules_present = sum(1 << int(x) for x in set(r.tolist()) if 0 <= x < 31)
        same = bool((r == r[0]).all() and (a == a[0]).all() and (t == t[0]).all())
        self._scalar = (int(r[0]), float(a[0]), float(t[0])) if same else None

    def draft_sample(self, logits, temperature, uniforms):
        if self._cut is not None:
            return spc.spc_sample(logits, uniforms, temp_per_seq=temperature, **self._cut)
        if self._scalar is not None:
            T = self._scalar[2]
            return spc.spc_draft_sample(logits, T, uniforms=uniforms if T > 0 else None)
        return spc.spc_draft_sample(logits, 0.0, uniforms=uniforms, temp_per_seq=temperature)

    def verify(self, q, p, drafts, uniforms, rule, alpha, temperature):
        if self._cut is not None:
            q = spc.spc_truncate(q, temp_per_seq=temperature, **self._cut)
            p = spc.spc_truncate(p, temp_per_seq=temperature, **self._cut)
        if self._scalar is not None:
            acc, tok, _ = spc.spc_verify_ex(q, p, drafts, uniforms, *self._scalar)
        else:
            acc, tok, _ = spc.spc_verify_ex(q, p, drafts, uniforms, 0, 0.0, 1.0,
                                            rule_per_seq=rule, alpha_per_seq=alpha,
                                            temp_per_seq=temperature,
                                            rules_present=self._rules_present)
        return acc, tok


@dataclass
class DecodeResult:
    tokens: list                      # per sequence: the emitted tokens, in order
    accept_len: list = field(default_factory=list)  # per round: [B] int tensor (j*)

    def tokens_per_round(self):
        """Mean emitted tokens per sequence and round (j* + 1)."""
        n = sum(int(a.sum()) + a.numel() for a in self.accept_len)
        return n / (len(self.accept_len) * self.accept_len[0].numel())


def spec_decode(drafter, verifier, first_tokens, rounds, gamma, rule, alpha, temperature,
                seed=0, backend=None, rounds_inputs=None, graph=False, top_k=0, top_p=1.0,
                min_p=0.0):
    """Run ``rounds`` rounds of GenSpecSample for B sequences whose last
    prefix token is ``first_tokens`` [B] (at position 0).  ``rule``,
    ``alpha`` and ``temperature`` are scalars or [B] tensors (temperature 0:
    greedy).  Uniforms come from a torch.Generator seeded with ``seed``;
    ``rounds_inputs`` (a list), when given, receives each round's inputs so a
    test can replay them through another backend.  ``top_k``, ``top_p`` and
    ``min_p`` (scalars or [B] tensors; 0, 1 and 0 leave a distribution whole)
    truncate both models' distributions; the backend then needs a ``truncate``
    method, which gets them as [B] tensors.

    The rounds run without waiting for the device: emitted tokens are
    scattered into a device buffer (a round writes its gamma+1 candidates at
    the sequence's length and advances the length by j* + 1, so the
    candidates past j* are overwritten by the next round), and the host reads
    the buffer and the accept lengths once, after the last round.  Rounds that
    went past a model's ``cache_tokens`` (an attribute it may have: the tokens
    of a sequence that its cache holds) are an error then.

    ``graph=True`` captures one round (the 2*gamma+1 model and sampling calls,
    the verification and the emission) into a HIP graph and replays it once
    per round, so a round costs one launch instead of dozens.  The round's
    uniforms are drawn up front in the eager order and copied into the
    graph's input buffers before each replay, so the tokens equal the eager
    loop's.  The models and the backend must be capturable (no host syncs,
    no allocation outside torch's allocator); one eager round, whose effects
    are undone, sizes the library's workspace before the capture."""
    backend = backend or GpuBackend()
    if graph and rounds_inputs is not None:
        raise ValueError("rounds_inputs needs the eager loop (graph=False)")
    dev = verifier.device
    B = first_tokens.numel()
    g1 = gamma + 1

    def per_seq(x, dtype):
        t = torch.as_tensor(x, dtype=dtype, device=dev)
        return t.expand(B).contiguous() if t.dim() == 0 else t.to(dev).contiguous()

    rule_t = per_seq(rule, torch.int32)
    alpha_t = per_seq(alpha, torch.float32)
    temp_t = per_seq(temperature, torch.float32)
    whole = (0, 1.0, 0.0)
    if any(torch.is_tensor(x) or x != w for x, w in zip((top_k, top_p, min_p), whole)):
        backend.truncate(per_seq(top_k, torch.int32), per_seq(top_p, torch.float32),
                         per_seq(min_p, torch.float32))
    if hasattr(backend, "prepare"):
        backend.prepare(rule_t, alpha_t, temp_t)
    gen = torch.Generator(device=dev).manual_seed(seed)
    # round state, updated in place by every round
    last = first_tokens.to(dev, torch.int32).clone()
    pos = torch.zeros(B, dtype=torch.int64, device=dev)
    buf = torch.zeros(B, rounds * g1 + g1, dtype=torch.int32, device=dev)
    length = torch.zeros(B, dtype=torch.int64, device=dev)
    acc_out = torch.zeros(B, dtype=torch.int64, device=dev)
    ar = torch.arange(g1, device=dev)

    def one_round(u_draft, u):
        # 1. draft gamma tokens from q, and q's logits at the extra position
        q_rows, drafts = [], []
        tok = last
        for j in range(g1):
            zq = drafter(tok, pos + j).contiguous()
            q_rows.append(zq)
            if j < gamma:
                tok = backend.draft_sample(zq, temp_t, u_draft[j].contiguous())
                drafts.append(tok)
        q = torch.stack(q_rows, dim=1).contiguous()            # [B, gamma+1, V]
        x = torch.stack(drafts, dim=1).to(torch.int32).contiguous()  # [B, gamma]
        # 2. score the gamma+1 prefixes with p in one batch
        ctx = torch.cat([last[:, None], x], dim=1)             # last tokens of x_{<t+j}
        p = verifier(ctx.reshape(-1), (pos[:, None] + ar).reshape(-1))
        p = p.reshape(B, g1, -1).contiguous()
        # 3. verify
        if rounds_inputs is not None:
            rounds_inputs.append(dict(q=q, p=p, draft=x, uniforms=u, u_draft=u_draft,
                                      rule=rule_t, alpha=alpha_t, temperature=temp_t))
        acc, nxt = backend.verify(q, p, x, u, rule_t, alpha_t, temp_t)
        # 4. emit x_t .. x_{t+j*-1} and the new token, roll back to t + j* + 1
        acc = acc.to(dev).long()
        nxt = nxt.to(dev, torch.int32)
        j = acc.clamp(min=0)
        cand = torch.cat([x, nxt[:, None]], dim=1)
        cand = torch.where(ar[None, :] == j[:, None], nxt[:, None], cand)
        buf.scatter_(1, length[:, None] + ar[None, :], cand)
        length.add_(j + 1)
        pos.add_(j + 1)
        last.copy_(nxt)
        acc_out.copy_(acc)

    def uniforms():
        return (torch.rand(gamma, B, generator=gen, device=dev),
                torch.rand(B, g1, generator=gen, device=dev))

    accs = torch.zeros(rounds, B, dtype=torch.int64, device=dev)
    if graph:
        drawn = [uniforms() for _ in range(rounds)]
        ud_in, u_in = torch.empty_like(drawn[0][0]), torch.empty_like(drawn[0][1])
        # warm-up on a side stream (the library sizes its workspace here);
        # the round state is restored afterwards
        state = [t.clone() for t in (last, pos, buf, length, acc_out)]
        side = torch.cuda.Stream(device=dev)
        side.wait_stream(torch.cuda.current_stream(dev))
        with torch.cuda.stream(side):
            ud_in.copy_(drawn[0][0])
            u_in.copy_(drawn[0][1])
            one_round(ud_in, u_in)
            for t, t0 in zip((last, pos, buf, length, acc_out), state):
                t.copy_(t0)
        torch.cuda.current_stream(dev).wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            one_round(ud_in, u_in)
        for r in range(rounds):
            ud_in.copy_(drawn[r][0])
            u_in.copy_(drawn[r][1])
            g.replay()
            accs[r].copy_(acc_out)
        torch.cuda.current_stream(dev).synchronize()
        del g
    else:
        for r in range(rounds):
            one_round(*uniforms())
            accs[r].copy_(acc_out)
    acc_h = accs.cpu()
    bad = (acc_h < 0).nonzero()
    if bad.numel():
        raise RuntimeError(f"sequence {int(bad[0, 1])}: invalid parameters (accept_len -1)")
    buf_h, len_h = buf.cpu(), length.cpu()
    if rounds:
        # the last round's models were called up to gamma past where it began
        reached = int((len_h - acc_h[-1]).max()) + gamma
        for name, lm in (("drafter", drafter), ("verifier", verifier)):
            if reached > getattr(lm, "cache_tokens", reached):
                raise RuntimeError(f"the rounds reached {reached} tokens of a sequence, the "
                                   f"{name}'s cache holds {lm.cache_tokens}")
    res = DecodeResult(tokens=[buf_h[b, :int(len_h[b])].tolist() for b in range(B)])
    res.accept_len = [a.to(torch.int32) for a in acc_h]
    return res


def synthetic_pair(V, seed=0, dtype=torch.bfloat16, device="cuda", rows=64):
    """A verifier SyntheticLM and a drafter derived from it as the Gemma-vocab
    workload's drafter (0.8 x verifier + N(0, 1))."""
    p = SyntheticLM(V, rows=rows, s=1.2, noise=1.0, seed=seed, dtype=dtype, device=device)
    return p.derive(scale=0.8, sigma=1.0, seed=seed + 1), p


__all__ = ["SyntheticLM", "ContextLM", "GpuBackend", "DecodeResult", "spec_decode", "synthetic_pair"]

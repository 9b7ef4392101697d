"""The operators of caches that batches share, that encoders fill and that are kept bounded,
over the ranges they run in.

A case is one call of one operator (``op``):

  shared  attention of new tokens over a paged cache whose first ``shared``
          positions are the same tokens for every sequence of the batch
  cross   attention of a decoder's tokens to an encoder's states, which a
          paged cache holds: every token sees all of them but masked ones
  weigh   the attention weight that every cached token gets from new tokens,
          summed over them and over the query heads of a group, on top of
          what it had
  evict   the tokens of the largest weights (of each sequence and key/value
          head), and the first and the last ones, into other pages

The plain forms below compute them with elementary torch operations; with
``own`` the library's calls run.  Keys are stored [page][head][slot][dim],
values [page][head][dim][slot], scales of 8-bit caches [page][head][slot].
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "f8": F8}


def _case(name, op, B, n, L, heads, kv_heads, D, page, cache, ragged=False, **more):
    """B sequences of up to L cached tokens, n new ones each (``ragged``: each its own numbers)."""
    c = dict(name=name, op=op, B=B, n=n, L=L, heads=heads, kv_heads=kv_heads, D=D, page=page,
             cache=cache, ragged=ragged, shared=0, window=0, masked=False, keep=0, first=0, recent=0)
    c.update(more)
    return c


def listed():
    return [
        # two sequences behind a short common instruction: latency
        _case("shared_small_bf16", "shared", 2, 1, 740, 4, 2, 64, 16, "bf16", shared=700),
        # a serving batch behind one long few-shot prompt, a token each
        _case("shared_token_bf16", "shared", 32, 1, 8704, 32, 8, 128, 16, "bf16", ragged=True,
              shared=8192),
        # the verifier scores gamma + 1 = 8 positions of each over an 8-bit cache
        _case("shared_block_f8", "shared", 32, 8, 8704, 32, 8, 128, 16, "f8", shared=8192),
        # one sequence, one token, a sentence to translate: latency
        _case("cross_one_bf16", "cross", 1, 1, 512, 8, 8, 64, 16, "bf16"),
        # an encoder-decoder verifier scores gamma + 1 = 6 positions, inputs of their own lengths
        _case("cross_block_bf16", "cross", 32, 6, 1024, 16, 16, 64, 32, "bf16", ragged=True),
        # long documents of which parts are masked, an 8-bit cache
        _case("cross_masked_f8", "cross", 16, 8, 4096, 32, 8, 128, 64, "f8", masked=True),
        # whole targets scored against their inputs
        _case("cross_chunk_bf16", "cross", 4, 1024, 4096, 32, 8, 128, 64, "bf16", ragged=True),
        # a serving batch's tokens weighed as it goes on
        _case("weigh_token_bf16", "weigh", 32, 1, 4096, 32, 8, 128, 16, "bf16"),
        # the last 32 tokens of long prompts, after which the cache is cut
        _case("weigh_window_f8", "weigh", 4, 32, 16384, 32, 8, 128, 16, "f8", ragged=True),
        # a prompt's chunk
        _case("weigh_chunk_bf16", "weigh", 2, 600, 2048, 16, 4, 128, 64, "bf16"),
        # one sequence that went a little past its budget: latency
        _case("evict_small_bf16", "evict", 1, 1, 1200, 2, 2, 64, 16, "bf16", keep=1024, first=4,
              recent=64),
        # long prompts cut to a budget
        _case("evict_half_bf16", "evict", 8, 1, 8192, 8, 8, 128, 16, "bf16", ragged=True, keep=4096,
              first=4, recent=256),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("shared", "cross", "weigh", "evict"))
    D = rng.choice((64, 128, 128, 256))
    H = rng.choice((1, 2, 4, 8))
    G = rng.choice((1, 2, 4, 8))
    page = rng.choice((16, 32, 64, 128))
    cache = rng.choice(("bf16", "f8"))
    kind = rng.choice(("one", "block", "chunk"))
    n = 1 if kind == "one" else rng.randint(2, 9) if kind == "block" else _log_int(rng, 17, 800)
    more = {}
    most = 3.2e7 if op == "evict" else 5.0e7  # values of K of the whole batch
    if op == "evict":
        n, G = 1, 1
        L = min(_log_int(rng, 100, 32768), int(most / (H * D)))
        more["keep"] = max(8, int(L * rng.choice((0.1, 0.5, 0.9)) * rng.uniform(0.8, 1.1)))
        more["first"] = rng.choice((0, 4))
        more["recent"] = rng.randint(0, more["keep"] // 2)
    else:
        L = max(n, min(_log_int(rng, 8, 32768), int(most / (H * D))))
        L = max(n, min(L, int(1.2e10 / (n * H * G * D))))
    if op == "shared":
        more["shared"] = max(1, int((L - min(n, L - 1)) * rng.uniform(0.5, 1.0)))
    if op in ("shared", "weigh"):
        more["window"] = rng.choice((0, 0, 0, max(1, L // 3)))
    if op == "cross":
        more["masked"] = rng.random() < 0.4
    B = min(64, int(most / (L * H * D)), int(1.2e10 / (L * n * H * G * D)))
    B = _log_int(rng, 1, max(1, B))
    c = _case("", op, B, n, L, H * G, H, D, page, cache, ragged=B > 1 and rng.random() < 0.5, **more)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _lengths(c):
    """(chunk lengths, cache lengths): all alike, or each sequence's own (the first the longest).
    Sequences that share a prefix differ in what comes behind it."""
    B, n, L, P = c["B"], c["n"], c["L"], c["shared"]
    if not c["ragged"]:
        return [n] * B, [L] * B
    ns = [max(1, int(n * (1.0 - 0.618 * b % 1.0))) for b in range(B)]
    return ns, [max(m, P + int((L - P) * (1.0 - 0.381 * b % 1.0))) for b, m in enumerate(ns)]


def _randn(shape, g, dtype):
    """N(0, 1) values in `dtype` (8 bits: 100 N(0, 1), within the type), made in pieces."""
    out = torch.empty(shape, device="cuda", dtype=dtype)
    flat, step = out.view(-1), 1 << 26
    for a in range(0, flat.numel(), step):
        m = min(step, flat.numel() - a)
        x = torch.randn(m, generator=g, device="cuda")
        if dtype == F8:
            x = x.mul_(100.0).clamp_(-448.0, 448.0)
            flat[a:a + m].view(torch.uint8).copy_(x.to(F8).view(torch.uint8))
        else:
            flat[a:a + m] = x.to(dtype)
    return out


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(int(seed) % (1 << 62))
    B, H, D, S, L = c["B"], c["kv_heads"], c["D"], c["page"], c["L"]
    ns, lens = _lengths(c)
    width, common = (L + S - 1) // S, c["shared"] // S  # pages of a sequence; whole ones of all
    out_width = (c["keep"] + S - 1) // S
    pages = B * (width - common + out_width) + (c["shared"] + S - 1) // S + 3
    dt = DT[c["cache"]]
    s = dict(case=c, k_pages=_randn((pages, H, S, D), g, dt), v_pages=_randn((pages, H, D, S), g, dt),
             k_scale=None, v_scale=None)
    if dt == F8:
        s["k_scale"] = torch.rand((pages, H, S), generator=g, device=dev).mul_(0.01).add_(0.005)
        s["v_scale"] = torch.rand((pages, H, S), generator=g, device=dev).mul_(0.01).add_(0.005)
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s["table"] = torch.empty((B, width), dtype=torch.int32, device=dev)
    s["table"][:, common:] = order[:B * (width - common)].view(B, width - common)
    order = order[B * (width - common):]
    if c["shared"]:
        s["shared_table"] = order[:(c["shared"] + S - 1) // S].contiguous()
        s["table"][:, :common] = s["shared_table"][:common]
        order = order[s["shared_table"].numel():]
    s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    starts = [0]
    for m in ns:
        starts.append(starts[-1] + m)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev) if c["ragged"] else None
    if c["op"] != "evict":
        lead = (starts[-1],) if c["ragged"] else (B, c["n"])
        s["q"] = _randn(lead + (c["heads"], D), g, torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
    if c["op"] == "cross":
        s["mask"] = None
        if c["masked"]:  # paragraphs of 100 tokens, a third of them left out
            left_out = torch.rand((B, (L + 99) // 100), generator=g, device=dev) < 0.33
            s["mask"] = ~left_out.repeat_interleave(100, 1)[:, :L].contiguous()
    if c["op"] in ("weigh", "evict"):
        # most of the weight on few tokens; what underflowed is zero
        w = torch.randn((B, H, L), generator=g, device=dev).mul_(3.0).exp_()
        s["weights"] = torch.where(w < 0.02, 0.0, w).contiguous()
    if c["op"] == "weigh":  # what a few calls like this one have left
        s["weights"].mul_(0.1 * c["n"] * (c["heads"] // H) / L)
        s["weighed"] = torch.zeros_like(s["weights"])
    if c["op"] == "evict":
        s["out_table"] = order[:B * out_width].view(B, out_width).contiguous()
        s["out_len"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["index"] = torch.zeros((B, H, c["keep"]), dtype=torch.int32, device=dev)
        s["out_weights"] = torch.zeros((B, H, c["keep"]), device=dev)
    return s


# ------------------------------------------------------------------ plain forms
def _dense(s):
    """Keys and values [B][H][L][D] in float32."""
    c = s["case"]
    B, H, D, S, L = c["B"], c["kv_heads"], c["D"], c["page"], c["L"]
    table = s["table"].long()
    f8 = c["cache"] == "f8"
    kp, vp = (x.view(torch.uint8) if f8 else x for x in (s["k_pages"], s["v_pages"]))

    def dense(pages):
        k, v = kp[pages], vp[pages]
        if f8:
            k, v = k.view(F8), v.view(F8)
        k, v = k.float(), v.float()
        if f8:
            k = k * s["k_scale"][pages][..., None]
            v = v * s["v_scale"][pages][..., None, :]
        n = pages.shape[-1] * S
        k = k.transpose(-4, -3).reshape(pages.shape[:-1] + (H, n, D))
        return k, v.permute(*range(v.dim() - 4), -3, -4, -1, -2).reshape(k.shape)

    k, v = dense(table)
    k, v = k[:, :, :L], v[:, :, :L]
    if c["shared"]:
        P = c["shared"]
        ks, vs = dense(s["shared_table"].long())
        k = torch.cat([ks[:, :P].expand(B, H, P, D), k[:, :, P:]], 2)
        v = torch.cat([vs[:, :P].expand(B, H, P, D), v[:, :, P:]], 2)
    return k, v


def _rows(s):
    """Queries [B][H][n G][D] in float32 (zeros where a sequence has fewer rows), the position
    [B][n] of each (-1: no row), and (sequence, place in it) of the packed rows."""
    c, lens = s["case"], s["kv_len"].long()
    B, n, H, D, G = c["B"], c["n"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    if s["q_start"] is None:
        ns = torch.full((B,), n, device="cuda", dtype=torch.long)
    else:
        ns = s["q_start"].long().diff()
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), ns, output_size=s["q"].numel() // (H * G * D))
    inside = torch.arange(seq.numel(), device="cuda") - (ns.cumsum(0) - ns)[seq]
    q = torch.zeros((B, n, H, G, D), device="cuda")
    at = torch.full((B, n), -1, device="cuda", dtype=torch.long)
    q[seq, inside] = s["q"].view(-1, H, G, D).float()
    at[seq, inside] = inside + (lens - ns)[seq]
    return q.permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D), at, seq, inside


def _probabilities(s, q, k, at):
    """[B][H][n][G][L], zero where a key is not seen."""
    c = s["case"]
    B, n, H, D, L = c["B"], c["n"], c["kv_heads"], c["D"], c["L"]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    score = score.view(B, H, n, -1, L)
    key = torch.arange(L, device="cuda")
    if c["op"] == "cross":
        seen = (key < s["kv_len"][:, None])[:, None].expand(B, n, L) & (at >= 0)[..., None]
        if s["mask"] is not None:
            seen = seen & s["mask"][:, None]
    else:
        seen = key <= at[..., None]
        if c["window"]:
            seen &= key > at[..., None] - c["window"]
    score = torch.where(seen[:, None, :, None], score, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    return p / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_attend(s):
    c = s["case"]
    B, n, H, D, G = c["B"], c["n"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    k, v = _dense(s)
    q, at, seq, inside = _rows(s)
    p = _probabilities(s, q, k, at).view(B, H, n * G, -1)
    o = torch.matmul(p, v.contiguous()).view(B, H, n, G, D).permute(0, 2, 1, 3, 4)
    s["out"].view(-1, H, G, D).copy_(o[seq, inside])
    return {"out": s["out"]}


def _plain_weigh(s):
    c = s["case"]
    k, _ = _dense(s)
    q, at, _, _ = _rows(s)
    new = _probabilities(s, q, k, at).sum((2, 3))
    key, lens = torch.arange(c["L"], device="cuda"), s["kv_len"]
    ns = c["n"] if s["q_start"] is None else s["q_start"].diff()
    old = torch.where((key < (lens - ns)[:, None])[:, None], s["weights"], 0.0)
    s["weighed"].copy_(torch.where((key < lens[:, None])[:, None], old + new, s["weighed"]))
    return {"weights": s["weighed"]}


def _cache(s):
    return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale") if s[k] is not None}


def _evicted(s):
    return dict(_cache(s), kv_len=s["out_len"], index=s["index"], weights=s["out_weights"])


def _plain_evict(s):
    c = s["case"]
    B, H, S, L, keep = c["B"], c["kv_heads"], c["page"], c["L"], c["keep"]
    key, lens = torch.arange(L, device="cuda"), s["kv_len"].long()[:, None]
    kept = torch.clamp(lens, max=keep)
    safe = (key < c["first"]) | (key >= lens - c["recent"])
    w = torch.where(safe[:, None], math.inf, s["weights"])
    w = torch.where((key < lens)[:, None], w, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices
    chosen = torch.where((key < kept)[:, None], order, L)  # (past the last one: L)
    index = torch.sort(chosen, dim=2).values
    if L < keep:
        index = torch.cat([index, index.new_full((B, H, keep - L), L)], 2)
    index = index[:, :, :keep]
    b, h, j = torch.nonzero(index < L, as_tuple=True)
    t = index[b, h, j]
    src, dst = s["table"][b, t // S].long(), s["out_table"][b, j // S].long()
    kp, vp = (x.view(torch.uint8) if c["cache"] == "f8" else x for x in (s["k_pages"], s["v_pages"]))
    kp[dst, h, j % S] = kp[src, h, t % S]
    vp[dst, h, :, j % S] = vp[src, h, :, t % S]
    if c["cache"] == "f8":
        for x in (s["k_scale"], s["v_scale"]):
            x[dst, h, j % S] = x[src, h, t % S]
    s["out_len"].copy_(kept[:, 0])
    s["index"].copy_(torch.where(index < L, index, -1))
    s["out_weights"][b, h, j] = s["weights"][b, h, t]
    return _evicted(s)


def _own(s):
    from paper_2405_19261_amd import spc
    c = s["case"]
    cache = (s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
    scales = dict(k_scale=s["k_scale"], v_scale=s["v_scale"])
    if c["op"] == "evict":
        spc.spc_kv_evict(*cache, s["weights"], c["keep"], s["out_table"], first=c["first"],
                         recent=c["recent"], out_len=s["out_len"], out_index=s["index"],
                         out_weights=s["out_weights"], **scales)
        return _evicted(s)
    rows = dict(q_start=s["q_start"], max_q=c["n"])
    if c["op"] == "shared":
        spc.spc_kv_attend_shared(s["q"], *cache, c["shared"], shared_table=s["shared_table"],
                                 window=c["window"], out=s["out"], **rows, **scales)
    elif c["op"] == "cross":
        spc.spc_cross_attend(s["q"], *cache, key_mask=s["mask"], out=s["out"], **rows, **scales)
    else:
        spc.spc_kv_weigh(s["q"], *cache, s["weights"], window=c["window"], out=s["weighed"], **rows,
                         **scales)
        return {"weights": s["weighed"]}
    return {"out": s["out"]}


def run(state):
    if own:
        return _own(state)
    return {"shared": _plain_attend, "cross": _plain_attend, "weigh": _plain_weigh,
            "evict": _plain_evict}[state["case"]["op"]](state)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    H, D = c["kv_heads"], c["D"]
    ns, lens = _lengths(c)
    f8 = c["cache"] == "f8"
    line = H * (D * (1 if f8 else 2) + (4 if f8 else 0))  # a token's keys
    if c["op"] == "evict":
        kept = sum(min(m, c["keep"]) for m in lens)
        return {"bytes": 4 * kept * line + 4 * H * sum(lens) + 8 * H * kept, "flops": H * sum(lens)}
    w = c["window"] or c["L"] + 1
    if c["op"] == "cross":
        keys, pairs = sum(lens), sum(n * m for n, m in zip(ns, lens))
    else:
        P = c["shared"]
        first = [max(0, m - n + 1 - w) for n, m in zip(ns, lens)]  # the first token seen
        keys = sum(m - max(P, f) for f, m in zip(first, lens)) + max(0, P - min(first))
        pairs = sum(sum(min(w, t + 1) for t in range(m - n, m)) for n, m in zip(ns, lens))
    rows = sum(ns) * c["heads"] * D
    if c["op"] == "weigh":
        return {"bytes": keys * line + 2 * rows + 8 * H * sum(lens), "flops": 2 * pairs * c["heads"] * D}
    masks = c["B"] * c["L"] if c["masked"] else 0
    return {"bytes": 2 * keys * line + 4 * rows + masks, "flops": 4 * pairs * c["heads"] * D}


# ------------------------------------------------------------------ in 64 bits
def _exact_lines(s, b, upto):
    """Keys and values [upto][H][D] of sequence b in float64, read line by line."""
    c = s["case"]
    t = torch.arange(upto, device="cuda")
    page, slot = s["table"][b].long()[t // c["page"]], t % c["page"]
    if c["shared"]:
        m = min(upto, c["shared"])
        page[:m] = s["shared_table"].long()[t[:m] // c["page"]]
    f8 = c["cache"] == "f8"
    kp, vp = (x.view(torch.uint8) if f8 else x for x in (s["k_pages"], s["v_pages"]))
    k, v = kp[page, :, slot], vp[page, :, :, slot]
    if f8:
        k, v = k.view(F8), v.view(F8)
    k, v = k.double(), v.double()
    if f8:
        k = k * s["k_scale"][page, :, slot].double()[..., None]
        v = v * s["v_scale"][page, :, slot].double()[..., None]
    return k, v


def _exact_attention(c, s):
    B, n, H, D, G = c["B"], c["n"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    lens = s["kv_len"].tolist()
    first = s["q_start"].tolist() if s["q_start"] is not None else [n * b for b in range(B + 1)]
    out = torch.zeros((first[-1], H, G, D), device="cuda", dtype=torch.float64)
    weights = s["weighed"].double() if c["op"] == "weigh" else None
    q = s["q"].view(-1, H, G, D).double()
    for b in range(B):
        k, v = _exact_lines(s, b, lens[b])
        m = first[b + 1] - first[b]
        at = torch.arange(lens[b] - m, lens[b], device="cuda")[:, None]
        key = torch.arange(lens[b], device="cuda")[None]
        if c["op"] == "cross":
            hidden = torch.zeros((m, lens[b]), dtype=torch.bool, device="cuda")
            if s["mask"] is not None:
                hidden |= ~s["mask"][b, :lens[b]]
        else:
            hidden = key > at
            if c["window"]:
                hidden |= key <= at - c["window"]
        if c["op"] == "weigh":
            weights[b, :, :lens[b] - m] = s["weights"][b, :, :lens[b] - m].double()
            weights[b, :, lens[b] - m:lens[b]] = 0.0
        for h in range(H):
            kh, vh = k[:, h].contiguous(), v[:, h].contiguous()
            for g in range(G):
                x = q[first[b]:first[b + 1], h, g].contiguous() @ kh.t().contiguous()
                p = torch.softmax((x / D ** 0.5).masked_fill(hidden, -math.inf), 1)
                p = p.masked_fill(hidden, 0.0)  # (a row that sees nothing)
                if c["op"] == "weigh":
                    weights[b, h, :lens[b]] += p.sum(0)
                else:
                    out[first[b]:first[b + 1], h, g] = p @ vh
    return {"weights": weights} if c["op"] == "weigh" else {"out": out.view(s["q"].shape)}


def _exact_evict(c, s):
    import numpy as np
    S, keep = c["page"], c["keep"]
    values = {k: x.double() for k, x in _cache(s).items()}
    w = s["weights"].double().cpu().numpy()
    index, out_w = s["index"].cpu().numpy(), s["out_weights"].double().cpu().numpy()
    lens, kept = s["kv_len"].tolist(), []
    for b, n in enumerate(lens):
        kept.append(min(n, keep))
        for h in range(c["kv_heads"]):
            t = np.arange(n)
            safe = (t < c["first"]) | (t >= n - c["recent"])
            some = np.sort(np.lexsort((t, -w[b, h, :n], ~safe))[:keep])
            index[b, h] = -1
            index[b, h, :len(some)] = some
            out_w[b, h, :len(some)] = w[b, h, some]
            src, j = torch.from_numpy(some).cuda(), torch.arange(len(some), device="cuda")
            p, q = s["table"][b].long()[src // S], s["out_table"][b].long()[j // S]
            for name, x in values.items():
                if name == "v_pages":
                    x[q, h, :, j % S] = x[p, h, :, src % S]
                else:
                    x[q, h, j % S] = x[p, h, src % S]
    return dict(values, kv_len=torch.tensor(kept, dtype=torch.int32), index=torch.from_numpy(index),
                weights=torch.from_numpy(out_w))


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_evict(case, s) if case["op"] == "evict" else _exact_attention(case, s)

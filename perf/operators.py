"""The operators around a decoding round's verification, over the ranges they run in.

A case is one call of one operator (``op``):

  sample    a token per row from softmax(z / T) cut by top-k, top-p and min-p,
            at a given uniform, with its log-probability and the number kept
  truncate  the same cut of the rows a verification reads, as logits that are
            -inf outside it
  write     new keys and values into a paged cache, in bfloat16 or quantised
            to 8 bits (e4m3) with a scale per token and head
  read      a paged cache back as dense keys and values
  attend    attention of a chunk of new tokens over the paged cache

The plain forms below compute them with elementary torch operations; with
``own`` the library's calls run.  Keys are stored [page][head][slot][dim],
values [page][head][dim][slot], scales [page][head][slot].
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": F8}

# how requests ask for their tokens: (T, top_k, top_p, min_p)
STYLES = {"k50": (1.0, 50, 1.0, 0.0), "p90": (1.0, 0, 0.9, 0.0), "p95t7": (0.7, 0, 0.95, 0.0),
          "k40p95": (0.8, 40, 0.95, 0.0), "min05": (1.0, 0, 1.0, 0.05), "k1000p99": (1.0, 1000, 0.99, 0.0),
          "all": (1.0, 0, 1.0, 0.0), "wide": (1.5, 0, 0.98, 0.001)}
MIX = ("k50", "p90", "p95t7", "k40p95", "min05", "wide")


def _rows(name, op, B, rows, V, dtype, style):
    return dict(name=name, op=op, B=B, rows=rows, V=V, dtype=dtype, style=style)


def _kv(name, op, B, n, L, heads, kv_heads, D, page, cache, src="bf16", ragged=False, window=0):
    return dict(name=name, op=op, B=B, n=n, L=L, heads=heads, kv_heads=kv_heads, D=D, page=page,
                cache=cache, src=src, ragged=ragged, window=window)


def listed():
    return [
        # the smallest draw: one sequence, a short vocabulary, nothing but latency
        _rows("sample_tiny_f32", "sample", 1, 1, 1000, "f32", "k40p95"),
        # a drafter's step at a T5-sized vocabulary
        _rows("sample_t5_f32", "sample", 8, 1, 32128, "f32", "p90"),
        # a serving batch at the Gemma vocabulary, every request with its own settings
        _rows("sample_gemma_mix_bf16", "sample", 32, 1, 256000, "bf16", "mix"),
        # a verification's rows at the T5-sized vocabulary
        _rows("truncate_t5_f32", "truncate", 8, 6, 32128, "f32", "k50"),
        # the benchmark step's verifier rows
        _rows("truncate_gemma_bf16", "truncate", 32, 8, 256000, "bf16", "p90"),
        # one drafted token a sequence into an 8-bit cache
        _kv("write_token_f8", "write", 32, 1, 1024, 8, 8, 128, 16, "f8"),
        # a prompt's chunk into a bfloat16 cache, sequences of their own lengths
        _kv("write_chunk_bf16", "write", 8, 1000, 2048, 8, 8, 128, 64, "bf16", "f32", ragged=True),
        # an 8-bit cache moved out whole
        _kv("read_f8", "read", 16, 1, 4096, 8, 8, 128, 16, "f8"),
        _kv("read_small_bf16", "read", 1, 1, 333, 4, 4, 64, 32, "bf16"),
        # one sequence, one token: latency
        _kv("attend_one_bf16", "attend", 1, 1, 1500, 32, 8, 128, 16, "bf16"),
        # the verifier scores gamma + 1 = 8 positions of a serving batch over an 8-bit cache
        _kv("attend_score_f8", "attend", 32, 8, 8192, 32, 8, 128, 16, "f8"),
        # a prompt's chunk behind what the cache holds
        _kv("attend_chunk_bf16", "attend", 4, 1024, 4096, 32, 8, 128, 64, "bf16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("sample", "sample", "truncate", "write", "read", "attend", "attend", "attend"))
    if op in ("sample", "truncate"):
        V = _log_int(rng, 1000, 256000)
        step = rng.choice((1, 8, 128))
        V = max(1000, V // step * step)
        rows = 1 if op == "sample" else rng.randint(2, 9)
        B = _log_int(rng, 1, max(1, min(256, int(3.0e7 / (V * rows)))))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        c = _rows("", op, B, rows, V, dtype, rng.choice(tuple(STYLES) + ("mix", "mix")))
    else:
        D = rng.choice((64, 128, 128, 256))
        kv_heads = rng.choice((1, 2, 4, 8))
        group = rng.choice((1, 2, 4, 8))
        cache = rng.choice(("bf16", "f8"))
        page = rng.choice((16, 32, 64, 128))
        kind = rng.choice(("one", "block", "block", "chunk"))
        n = 1 if kind == "one" else rng.randint(2, 9) if kind == "block" else _log_int(rng, 17, 800)
        most = 6.0e7 if op == "attend" else 2.0e7  # values of K of the whole batch
        L = max(n, _log_int(rng, 1, 32768))
        L = min(L, int(most / (kv_heads * D)))
        B = _log_int(rng, 1, max(1, min(64, int(most / (L * kv_heads * D)))))
        if op == "attend":  # no more operations than the largest listed case
            L = max(n, min(L, int(1.4e10 / (n * kv_heads * group * D))))
            B = max(1, min(B, int(1.4e10 / (L * n * kv_heads * group * D))))
        src = "bf16" if op == "attend" else rng.choice(("bf16", "f32"))
        window = rng.choice((0, 0, 0, max(1, L // 3))) if op == "attend" else 0
        c = _kv("", op, B, n, L, kv_heads * group, kv_heads, D, page, cache, src,
                ragged=B > 1 and rng.random() < 0.5, window=window)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _prepare_rows(c, seed):
    """Logits [B][rows][V]: a Zipf ranking with N(0, 1) noise, as a language model's; the
    settings of each sequence; the uniforms."""
    g, dev = _gen(seed), "cuda"
    B, n, V = c["B"], c["rows"], c["V"]
    R = B * n
    z = torch.empty((R, V), device=dev, dtype=DT[c["dtype"]])
    chunk = max(1, min(R, (1 << 27) // V))
    for r0 in range(0, R, chunk):
        m = min(R, r0 + chunk) - r0
        rank = torch.rand((m, V), generator=g, device=dev).mul_(V).floor_().add_(1.0)
        noise = torch.randn((m, V), generator=g, device=dev)
        z[r0:r0 + m] = rank.log_().mul_(-1.2).add_(noise).add_(12.0).to(z.dtype)
    styles = [MIX[b % len(MIX)] if c["style"] == "mix" else c["style"] for b in range(B)]
    s = dict(case=c, z=z.view(B, n, V), u=torch.rand(B, generator=g, device=dev))
    for k, name, dt in ((0, "T", torch.float32), (1, "top_k", torch.int32),
                        (2, "top_p", torch.float32), (3, "min_p", torch.float32)):
        s[name] = torch.tensor([STYLES[x][k] for x in styles], dtype=dt, device=dev)
    if c["op"] == "truncate":
        s["out"] = torch.empty_like(s["z"])
    else:
        s["token"] = torch.empty(B, dtype=torch.int32, device=dev)
        s["logprob"] = torch.empty(B, device=dev)
        s["kept"] = torch.empty(B, dtype=torch.int32, device=dev)
    return s


def _randn(shape, g, dtype):
    """N(0, 1) values in `dtype`, made in pieces."""
    out = torch.empty(shape, device="cuda", dtype=dtype)
    flat, step = out.view(-1), 1 << 26
    for a in range(0, flat.numel(), step):
        m = min(step, flat.numel() - a)
        x = torch.randn(m, generator=g, device="cuda")
        if dtype == F8:
            flat[a:a + m].view(torch.uint8).copy_(x.mul_(100.0).to(F8).view(torch.uint8))
        else:
            flat[a:a + m] = x.to(dtype)
    return out


def _lengths(c):
    """(chunk lengths, cache lengths): all alike, or each sequence's own (the first the longest)."""
    B, n, L = c["B"], c["n"], c["L"]
    if not c["ragged"]:
        return [n] * B, [L] * B
    ns = [max(1, int(n * (1.0 - 0.618 * b % 1.0))) for b in range(B)]
    return ns, [max(m, int(L * (1.0 - 0.381 * b % 1.0))) for b, m in enumerate(ns)]


def _prepare_kv(c, seed):
    g, dev = _gen(seed), "cuda"
    B, H, D, S = c["B"], c["kv_heads"], c["D"], c["page"]
    ns, lens = _lengths(c)
    width = (c["L"] + S - 1) // S
    pages = B * width + 3
    dt = DT[c["cache"]]
    s = dict(case=c, k_pages=_randn((pages, H, S, D), g, dt), v_pages=_randn((pages, H, D, S), g, dt))
    s["k_scale"] = s["v_scale"] = None
    if dt == F8:
        s["k_scale"] = torch.rand((pages, H, S), generator=g, device=dev).mul_(0.01).add_(0.005)
        s["v_scale"] = torch.rand((pages, H, S), generator=g, device=dev).mul_(0.01).add_(0.005)
    table = torch.randperm(pages, generator=g, device=dev)[:B * width]
    s["table"] = table.view(B, width).to(torch.int32)
    s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    starts = [0]
    for m in ns:
        starts.append(starts[-1] + m)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev) if c["ragged"] else None
    N = starts[-1]
    lead = (N,) if c["ragged"] else (B, c["n"])
    if c["op"] == "write":
        s["k"] = _randn(lead + (H, D), g, DT[c["src"]])
        s["v"] = _randn(lead + (H, D), g, DT[c["src"]])
    elif c["op"] == "read":
        s["k"] = torch.zeros((B, c["L"], H, D), device=dev, dtype=DT[c["src"]])
        s["v"] = torch.zeros_like(s["k"])
    else:
        s["q"] = _randn(lead + (c["heads"], D), g, torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
    return s


def prepare(case, seed):
    return _prepare_rows(case, seed) if case["op"] in ("sample", "truncate") else _prepare_kv(case, seed)


# ------------------------------------------------------------------ plain forms
def _plain_cut(z, T, top_k, top_p, min_p):
    """(kept, weights) of rows z [R][V] in float64; the settings are [R][1]."""
    V = z.shape[1]
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    c = torch.exp((zs - zs[:, :1]) / T).cumsum(1)
    place = torch.arange(V, device=z.device)
    n_k = torch.where(top_k > 0, top_k.clamp(max=V), V).long()
    whole = c.gather(1, n_k - 1)
    before = torch.cat([torch.zeros_like(c[:, :1]), c[:, :-1]], 1)
    keep = (place < n_k) & ((before < top_p * whole) | (top_p >= 1))
    keep &= (zs >= zs[:, :1] + T * torch.log(min_p)) & (zs > -math.inf)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    return kept, torch.exp((z - zs[:, :1]) / T)


def _plain_rows(s):
    c = s["case"]
    B, n, V = c["B"], c["rows"], c["V"]
    z = s["z"].view(B * n, V).double()
    of = [s[k].double().repeat_interleave(n)[:, None] for k in ("T", "top_k", "top_p", "min_p")]
    kept, w = _plain_cut(z, *of)
    if c["op"] == "truncate":
        s["out"].copy_(torch.where(kept, s["z"].view(B * n, V), -math.inf).view(B, n, V))
        return {"logits": s["out"]}
    w = torch.where(kept, w, 0.0)
    cum = w.cumsum(1)
    token = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1)
    s["token"].copy_(token)
    s["logprob"].copy_(torch.log(w.gather(1, token[:, None]) / cum[:, -1:])[:, 0])
    s["kept"].copy_(kept.sum(1))
    return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}


def _places(s):
    """(sequence, position) of every new token, in the order of the packed rows."""
    c, lens = s["case"], s["kv_len"].long()
    if s["q_start"] is None:
        ns = torch.full((c["B"],), c["n"], device="cuda", dtype=torch.long)
    else:
        ns = s["q_start"].long().diff()
    seq = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), ns)
    first = ns.cumsum(0) - ns
    return seq, torch.arange(seq.numel(), device="cuda") - first[seq] + (lens - ns)[seq]


def _quantise(x):
    x = x.float()
    scale = (x.abs().amax(-1, keepdim=True) / 448.0).clamp(min=2.0 ** -126)
    return (x / scale).clamp(-448.0, 448.0).to(F8), scale[..., 0]


def _plain_write(s):
    c = s["case"]
    H, D, S = c["kv_heads"], c["D"], c["page"]
    seq, pos = _places(s)
    page, slot = s["table"][seq, pos // S].long(), pos % S
    k, v = s["k"].view(-1, H, D), s["v"].view(-1, H, D)
    if c["cache"] == "f8":
        (k, ks), (v, vs) = _quantise(k), _quantise(v)
        s["k_scale"][page, :, slot] = ks
        s["v_scale"][page, :, slot] = vs
        s["k_pages"].view(torch.uint8)[page, :, slot] = k.view(torch.uint8)
        s["v_pages"].view(torch.uint8)[page, :, :, slot] = v.view(torch.uint8)
    else:
        s["k_pages"][page, :, slot] = k.to(torch.bfloat16)
        s["v_pages"][page, :, :, slot] = v.to(torch.bfloat16)
    return _cache(s)


def _cache(s):
    return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale") if s[k] is not None}


def _dense(s, width):
    """Keys and values [B][width * page][H][D] in float32."""
    c = s["case"]
    B, H, D, S = c["B"], c["kv_heads"], c["D"], c["page"]
    table = s["table"][:, :width].long()
    k, v = s["k_pages"].view(torch.uint8 if c["cache"] == "f8" else torch.bfloat16)[table], None
    v = s["v_pages"].view(k.dtype)[table]
    if c["cache"] == "f8":
        k, v = k.view(F8), v.view(F8)
    k, v = k.float(), v.float()
    if c["cache"] == "f8":
        k = k * s["k_scale"][table][..., None]
        v = v * s["v_scale"][table][:, :, :, None, :]
    k = k.permute(0, 1, 3, 2, 4).reshape(B, width * S, H, D)
    return k, v.permute(0, 1, 4, 2, 3).reshape(B, width * S, H, D)


def _plain_read(s):
    c = s["case"]
    k, v = _dense(s, s["table"].shape[1])
    there = (torch.arange(c["L"], device="cuda") < s["kv_len"][:, None])[..., None, None]
    s["k"].copy_(torch.where(there, k[:, :c["L"]].to(s["k"].dtype), s["k"]))
    s["v"].copy_(torch.where(there, v[:, :c["L"]].to(s["v"].dtype), s["v"]))
    return {"k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    B, n, H, D, G = c["B"], c["n"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    k, v = _dense(s, s["table"].shape[1])
    seq, pos = _places(s)
    row = torch.arange(seq.numel(), device="cuda")
    inside = row - torch.searchsorted(seq, seq)
    q = torch.zeros((B, n, H, G, D), device="cuda")
    at = torch.full((B, n), -1, device="cuda", dtype=torch.long)
    q[seq, inside] = s["q"].view(-1, H, G, D).float()
    at[seq, inside] = pos
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    score = score.view(B, H, n, G, -1)
    key = torch.arange(score.shape[-1], device="cuda")
    seen = key <= at[..., None]
    if c["window"]:
        seen &= key > at[..., None] - c["window"]
    seen = seen[:, None, :, None]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    p = (p / p.sum(-1, keepdim=True).clamp(min=1e-30)).view(B, H, n * G, -1)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()).view(B, H, n, G, D).permute(0, 2, 1, 3, 4)
    s["out"].view(-1, H, G, D).copy_(o[seq, inside])
    return {"out": s["out"]}


def _own(s):
    from paper_2405_19261_amd import spc
    c = s["case"]
    if c["op"] == "sample":
        spc.spc_sample(s["z"][:, 0], s["u"], temp_per_seq=s["T"], top_k_per_seq=s["top_k"],
                       top_p_per_seq=s["top_p"], min_p_per_seq=s["min_p"], out=s["token"],
                       out_logprob=s["logprob"], out_kept=s["kept"])
        return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}
    if c["op"] == "truncate":
        spc.spc_truncate(s["z"], temp_per_seq=s["T"], top_k_per_seq=s["top_k"],
                         top_p_per_seq=s["top_p"], min_p_per_seq=s["min_p"], out=s["out"])
        return {"logits": s["out"]}
    cache = (s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
    scales = dict(k_scale=s["k_scale"], v_scale=s["v_scale"])
    if c["op"] == "write":
        spc.spc_kv_write(s["k"], s["v"], *cache, q_start=s["q_start"], **scales)
        return _cache(s)
    if c["op"] == "read":
        spc.spc_kv_read(*cache, out=(s["k"], s["v"]), **scales)
        return {"k": s["k"], "v": s["v"]}
    spc.spc_kv_attend(s["q"], *cache, window=c["window"], q_start=s["q_start"],
                      max_q=c["n"], out=s["out"], **scales)
    return {"out": s["out"]}


def run(state):
    if own:
        return _own(state)
    return {"sample": _plain_rows, "truncate": _plain_rows, "write": _plain_write,
            "read": _plain_read, "attend": _plain_attend}[state["case"]["op"]](state)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    if c["op"] in ("sample", "truncate"):
        eb = 2 if c["dtype"] == "bf16" else 4
        n = c["B"] * c["rows"] * c["V"]
        return {"bytes": n * eb * (2 if c["op"] == "truncate" else 1) + 28 * c["B"],
                "flops": 6 * n}
    H, D = c["kv_heads"], c["D"]
    ns, lens = _lengths(c)
    line = H * (D * (1 if c["cache"] == "f8" else 2) + (4 if c["cache"] == "f8" else 0))
    dense = H * D * (2 if c["src"] == "bf16" else 4)
    if c["op"] == "write":
        return {"bytes": 2 * sum(ns) * (line + dense), "flops": 4 * sum(ns) * H * D}
    if c["op"] == "read":
        return {"bytes": 2 * sum(lens) * (line + dense), "flops": 2 * sum(lens) * H * D}
    w = c["window"] or c["L"] + 1
    keys = sum(min(m, n + w - 1) for n, m in zip(ns, lens))
    pairs = sum(sum(min(w, t + 1) for t in range(m - n, m)) for n, m in zip(ns, lens))
    return {"bytes": 2 * keys * line + 4 * sum(ns) * c["heads"] * D,
            "flops": 4 * pairs * c["heads"] * D}


# ------------------------------------------------------------------ in 64 bits
def _exact_row(z, T, k, p, m, u):
    """One row: (kept indices, in vocabulary order; token; logprob) by its definition."""
    import numpy as np
    V = z.shape[0]
    e = (z - z.max()) / T
    order = np.lexsort((np.arange(V), -z))
    mass = np.exp(e[order])
    n = min(k, V) if k > 0 else V
    if p < 1:
        run = np.add.accumulate(mass[:n].astype(np.longdouble))
        n = min(n, int(np.searchsorted(run, np.longdouble(p) * run[n - 1], side="left")) + 1)
    some = order[:n]
    some = some[np.isfinite(z[some])]
    if m > 0:
        some = some[z[some] >= z.max() + T * math.log(m)]
    some = np.sort(some)
    run = np.add.accumulate(np.exp(e[some]).astype(np.longdouble))
    j = int(np.searchsorted(run, np.longdouble(u) * run[-1], side="right"))
    return some, int(some[j]), float(e[some[j]] - np.log(run[-1]))


def _exact_rows(c, s):
    import numpy as np
    B, n, V = c["B"], c["rows"], c["V"]
    if B * n * V > 2.5e7:
        return None
    z = s["z"].double().cpu().numpy()
    T, k, p, m, u = (s[x].double().cpu().numpy() for x in ("T", "top_k", "top_p", "min_p", "u"))
    got = [[_exact_row(z[b, j], T[b], int(k[b]), p[b], m[b], u[b]) for j in range(n)]
           for b in range(B)]
    if c["op"] == "truncate":
        out = np.full(z.shape, -np.inf)
        for b in range(B):
            for j in range(n):
                out[b, j, got[b][j][0]] = z[b, j, got[b][j][0]]
        return {"logits": torch.from_numpy(out)}
    return {"token": torch.tensor([g[0][1] for g in got], dtype=torch.int32),
            "logprob": torch.tensor([g[0][2] for g in got], dtype=torch.float64),
            "kept": torch.tensor([len(g[0][0]) for g in got], dtype=torch.int32)}


def _exact_lines(s, b, upto):
    """Keys and values [upto][H][D] of sequence b in float64, read line by line."""
    c = s["case"]
    t = torch.arange(upto, device="cuda")
    page, slot = s["table"][b].long()[t // c["page"]], t % c["page"]
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


def _exact_kv(c, s):
    B, n, H, D = c["B"], c["n"], c["kv_heads"], c["D"]
    G = c["heads"] // H
    lens = s["kv_len"].tolist()
    first = s["q_start"].tolist() if s["q_start"] is not None else [n * b for b in range(B + 1)]
    if c["op"] == "write":
        f8 = c["cache"] == "f8"  # (what 8 bits hold of a value is a rounding's choice: no value)
        k_out, v_out = (s[x].double() for x in (("k_scale", "v_scale") if f8 else ("k_pages", "v_pages")))
        k, v = s["k"].view(-1, H, D).double(), s["v"].view(-1, H, D).double()
        for b in range(B):
            m = first[b + 1] - first[b]
            t = torch.arange(lens[b] - m, lens[b], device="cuda")
            page, slot = s["table"][b].long()[t // c["page"]], t % c["page"]
            kb, vb = k[first[b]:first[b + 1]], v[first[b]:first[b + 1]]
            if f8:
                k_out[page, :, slot] = kb.abs().max(-1).values / 448
                v_out[page, :, slot] = vb.abs().max(-1).values / 448
            else:
                k_out[page, :, slot] = kb
                v_out[page, :, :, slot] = vb
        if f8:
            return {"k_pages": None, "v_pages": None, "k_scale": k_out, "v_scale": v_out}
        return {"k_pages": k_out, "v_pages": v_out}
    if c["op"] == "read":
        k, v = s["k"].double(), s["v"].double()
        for b in range(B):
            k[b, :lens[b]], v[b, :lens[b]] = _exact_lines(s, b, lens[b])
        return {"k": k, "v": v}
    out = torch.zeros((first[-1], H, G, D), device="cuda", dtype=torch.float64)
    q = s["q"].view(-1, H, G, D).double()
    for b in range(B):
        k, v = _exact_lines(s, b, lens[b])
        m = first[b + 1] - first[b]
        at = torch.arange(lens[b] - m, lens[b], device="cuda")[:, None]
        key = torch.arange(lens[b], device="cuda")[None]
        hidden = key > at
        if c["window"]:
            hidden |= key <= at - c["window"]
        for h in range(H):
            kh, vh = k[:, h].contiguous(), v[:, h].contiguous()
            for g in range(G):
                x = q[first[b]:first[b + 1], h, g].contiguous() @ kh.t().contiguous()
                p = torch.softmax((x / D ** 0.5).masked_fill(hidden, -math.inf), 1)
                out[first[b]:first[b + 1], h, g] = p @ vh
    return {"out": out.view(s["q"].shape)}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rows(case, s) if case["op"] in ("sample", "truncate") else _exact_kv(case, s)

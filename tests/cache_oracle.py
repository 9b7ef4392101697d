"""Plain 64-bit implementations of the attentions whose rows share keys, of the
weights that tokens accumulate and of their eviction (numpy on the host), written
from their definitions for the tests."""
import numpy as np
import torch

import ops_oracle

BF16, F32 = torch.bfloat16, torch.float32


def i32(x, device="cuda"):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)


def randn(shape, seed, dtype=BF16, s=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * s).to(dtype)


def fill(cache, lens, seed, s=1.0):
    """Write every sequence's tokens 0 .. lens[b] - 1, one sequence after the other."""
    from paper_2405_19261_amd import spc
    for b, n in enumerate(lens):
        if n == 0:
            continue
        k, v = (randn((1, n, cache.H, cache.D), seed + 10 * b + i, BF16, s).cuda() for i in range(2))
        spc.spc_kv_write(k, v, cache.k, cache.v, cache.table[b:b + 1].contiguous(), i32([n]),
                         **cache.scales())


def chunks(q, lens, starts):
    """(sequence, row, position) of every new token of q: [B, n, heads, D], or packed."""
    if starts is None:
        B, n = q.shape[:2]
        starts = [n * b for b in range(B + 1)]
    return [(b, r, int(lens[b]) - (starts[b + 1] - starts[b]) + r - starts[b])
            for b in range(len(lens)) for r in range(starts[b], starts[b + 1])]


def check_rows(got, q, lens, starts, lines, sees, scale):
    """Rows of `got` against the definition: lines(b) gives (K, V, there), sees(b, position) the
    bool mask of the keys a row sees.  Returns the worst error over its tolerance."""
    heads, D = q.shape[-2:]
    host, got = (x.detach().cpu().double().numpy().reshape(-1, heads, D) for x in (q, got))
    worst, last = 0.0, None
    for b, r, at in chunks(q, lens, starts):
        if last != b:
            k, v, there = lines(b)
            last = b
        see = there & sees(b, at)
        for g in range(heads):
            h = g // (heads // k.shape[1])
            o, tol = ops_oracle.attend(host[r, g], k[:, h], v[:, h], see, 0, len(k), scale)
            d = np.abs(got[r, g] - o)
            assert (d <= tol).all(), (b, r, g, float((d - tol).max()), at)
            worst = max(worst, float((d / np.maximum(tol, 1e-30)).max()))
    return worst


def weighed(q, lens, starts, lines, window, scale, weights, length, most=None):
    """(weights, tolerance) [B][H][length] in float64; entries that no one writes are NaN.

    The tolerance follows the arithmetic the interface states: a score's error moves its
    exponent by delta (D products and three factors in 32 bits, and exp2's own 2^-21), so a weight
    by delta and the sum it is divided by by delta again; sums of the keys' weights and over rows
    add half a step 2^-24 a term."""
    heads, D = q.shape[-2:]
    host = q.detach().cpu().double().numpy().reshape(-1, heads, D)
    B, H = weights.shape[:2]
    G = heads // H
    out, tol = np.full((B, H, length), np.nan), np.zeros((B, H, length))
    rows = {b: [] for b in range(B)}
    for b, r, at in chunks(q, lens, starts):
        rows[b].append((r, at))
    for b in range(B):
        n = max(int(lens[b]), 0)
        k, _, there = lines(b)
        m = min(n, length, len(there))
        new = n - len(rows[b])
        t = np.arange(m)
        out[b, :, :m] = np.where(t < new, weights[b, :, :m], 0.0)
        total = len(rows[b]) * G
        for r, at in rows[b][:most]:
            key = np.arange(len(k))
            see = there & (key <= at)
            if window:
                see &= key > at - window
            if not see.any():
                continue
            for g in range(heads):
                h = g // G
                s = np.where(see, scale * (np.where(see[:, None], k[:, h], 0.0) @ host[r, g]), -np.inf)
                w = np.exp(s - s.max())
                w /= w.sum()
                mag = abs(scale) * (np.abs(np.where(see[:, None], k[:, h], 0.0)) @ np.abs(host[r, g]))
                delta = (D + 8) * 2.0 ** -24 * mag.max() + 2.0 ** -21
                out[b, h, :m] += w[:m]
                tol[b, h, :m] += w[:m] * (2 * delta + (len(k) + 64) * 2.0 ** -24)
        tol[b, :, :m] += np.abs(out[b, :, :m]) * (total + 2) * 2.0 ** -24 + 1e-30
        # what lies past the sequence stays
    return out, tol * 1.01


def evicted(weights, n, there, keep, first, recent):
    """Positions kept of n tokens, of which `there` are in the cache."""
    t = np.arange(n)
    w = np.zeros(n)
    w[:min(n, len(weights))] = weights[:n]
    w = np.where(np.isnan(w), -np.inf, w)
    nan = np.zeros(n, bool)
    nan[:min(n, len(weights))] = np.isnan(weights[:n])
    safe = (t < first) | (t >= n - recent)
    order = np.lexsort((t, nan & ~safe, np.where(safe, 0.0, -w), ~safe))
    order = order[there[order]]
    return np.sort(order[:keep])

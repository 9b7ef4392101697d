"""Plain 64-bit implementations of the truncated distributions, the paged
cache and the chunk attention (numpy on the host), written from their
definitions for the tests."""
import math

import numpy as np
import torch


def cleaned(z):
    """A row as the order sees it: NaN as -inf, +inf as the largest finite float32."""
    z = np.array(z, dtype=np.float64)
    z[np.isnan(z)] = -np.inf
    return np.minimum(z, float(np.finfo(np.float32).max))


def kept_set(z, T, top_k=0, top_p=1.0, min_p=0.0):
    """Indices kept (vocabulary order) and the masses of all entries relative
    to the largest, of a cleaned row; T > 0, settings valid."""
    V = z.shape[0]
    zmax = z.max()
    if zmax == -np.inf:
        return np.zeros(0, np.int64), np.zeros(V)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        w = np.exp((z - zmax) / np.float64(T))
    order = np.lexsort((np.arange(V), -z))
    n = min(top_k, V) if top_k > 0 else V
    if top_p < 1.0:
        run = np.cumsum(w[order[:n]].astype(np.longdouble))
        n = min(n, int(np.searchsorted(run, np.longdouble(top_p) * run[-1], side="left")) + 1)
    some = order[:n]
    if min_p > 0.0:
        some = some[z[some] >= zmax + np.float64(T) * math.log(min_p)]
    return np.sort(some[z[some] > -np.inf]), w


def sample(z, u, T, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, kept) of one row."""
    z = cleaned(z)
    if not (z > -np.inf).any():
        return -1, -math.inf, 0
    if T == 0:
        return int(np.argmax(z)), 0.0, 1
    some, w = kept_set(z, T, top_k, top_p, min_p)
    run = np.cumsum(w[some].astype(np.longdouble))
    j = min(int(np.searchsorted(run, np.longdouble(u) * run[-1], side="right")), len(some) - 1)
    return int(some[j]), float((z[some[j]] - z.max()) / T - np.log(run[-1])), len(some)


def truncated(z, T, top_k=0, top_p=1.0, min_p=0.0):
    """A row's entries, -inf outside the kept set (unchanged at T = 0)."""
    if T == 0:
        return np.array(z, dtype=np.float64)
    some, _ = kept_set(cleaned(z), T, top_k, top_p, min_p)
    out = np.full(len(z), -np.inf)
    out[some] = np.asarray(z, dtype=np.float64)[some]
    return out


# ------------------------------------------------------------------ the cache
class Cache:
    """A paged cache's tensors, on `device`, filled with junk (NaN among it)."""

    def __init__(self, B, width, H, D, S, f8, device, seed=0, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.pages = B * width + spare
        dt = torch.float8_e4m3fn if f8 else torch.bfloat16
        junk = torch.randint(0, 256, (2, self.pages, H, S, D * (1 if f8 else 2)), generator=g,
                             dtype=torch.uint8)
        self.k = junk[0].contiguous().view(dt).to(device)
        self.v = junk[1].contiguous().view(dt).reshape(self.pages, H, D, S).contiguous().to(device)
        nan = torch.full((self.pages, H, S), float("nan"), device=device)
        self.ks, self.vs = (nan, nan.clone()) if f8 else (None, None)
        self.table = torch.randperm(self.pages, generator=g)[:B * width].view(B, width).to(
            device, torch.int32)
        self.B, self.width, self.H, self.D, self.S, self.f8 = B, width, H, D, S, f8

    def args(self, kv_len):
        return (self.k, self.v, self.table, kv_len)

    def scales(self):
        return dict(k_scale=self.ks, v_scale=self.vs)

    def dense(self, b, n):
        """(K, V) [n, H, D] in float64 and which of the positions are in the cache."""
        t = np.arange(n)
        page = np.full(n, -1, np.int64)
        inside = t // self.S < self.width
        table = self.table.cpu().numpy()
        page[inside] = table[b, t[inside] // self.S]
        there = (page >= 0) & (page < self.pages)
        page = np.where(there, page, 0)
        k = self.k.cpu().float().double().numpy()[page, :, t % self.S]
        v = self.v.cpu().float().double().numpy()[page, :, :, t % self.S]
        if self.f8:
            k = k * self.ks.cpu().double().numpy()[page, :, t % self.S][..., None]
            v = v * self.vs.cpu().double().numpy()[page, :, t % self.S][..., None]
        return k, v, there


def quantised(x):
    """(codes' values, scale) of rows of float32 values along the last axis."""
    scale = np.maximum(np.abs(x).max(-1, keepdims=True) / np.float32(448), np.float32(2.0 ** -126))
    y = torch.from_numpy(np.clip(x / scale, -448, 448).astype(np.float32))
    return y.to(torch.float8_e4m3fn).float().double().numpy(), scale[..., 0]


def attend(q, k, v, there, first, last, scale):
    """One row's (output, tolerance) over keys first .. last that are there:
    q [D], k and v [n, D] of the row's head, all float64.

    The tolerance follows the arithmetic the interface states: scores in 32
    bits (D products and three factors, each off by half a step 2^-24, so the
    exponent by delta), probabilities rounded to bfloat16 (2^-8), sums of n
    terms in 32 bits, and the output rounded to bfloat16 (2^-8)."""
    t = np.arange(len(k))
    see = there & (t >= max(first, 0)) & (t <= last)
    if not see.any():
        return np.zeros_like(q), np.zeros_like(q)
    k, v = k[see], v[see]
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    w /= w.sum()
    delta = (len(q) + 8) * 2.0 ** -24 * (abs(scale) * (np.abs(k) @ np.abs(q))).max() + 2.0 ** -21
    o, mass = w @ v, w @ np.abs(v)
    # twice delta: on a weight and on their sum
    rel = 2.0 ** -8 + 2 * delta + (len(k) + 64) * 2.0 ** -23
    return o, rel * mass * 1.01 + 2.0 ** -8 * np.abs(o) + 1e-30

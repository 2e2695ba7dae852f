"""The 4-bit cache and the eviction in plain numpy, 64 bits where numbers are computed: what the kernels are compared with."""
import numpy as np


def bf16(a):
    """fp32 values rounded to bf16, nearest even."""
    u = np.asarray(a, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def quantise(x):
    """Codes [..., D] uint8 and pairs [..., 2] fp32 (step, low) of rows [..., D], in the 32-bit steps that define them."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        low, step = bf16(lo), bf16((hi - lo) / np.float32(15))
        code = np.where(step > 0, np.clip(np.rint((x - low) / step), 0, 15), 0)
        bad = ~(np.isfinite(x).all(-1, keepdims=True) & np.isfinite(hi - lo) & np.isfinite(low))
    code = np.where(bad, 0, code).astype(np.uint8)
    return code, np.concatenate([np.where(bad, np.nan, step), np.where(bad, np.nan, low)], -1).astype(np.float32)


def pack(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def values(code, pair):
    """What rows stand for, exactly."""
    pair = pair.astype(np.float64)
    return pair[..., 1:] + pair[..., :1] * code


class Paged:
    """Sequences' positions in a paged cache (page 0: one run of `cap` positions each)."""

    def __init__(self, rng, B, positions, page):
        self.B, self.page = B, page
        self.cap = -(-positions // page) if page else positions
        self.positions = self.cap * (page or 1)
        self.pages = B * self.cap + 3 if page else 0
        self.table = rng.permutation(self.pages)[:B * self.cap].reshape(B, self.cap).astype(np.int32) if page else None
        self.shape = (self.pages, page) if page else (B, positions)

    def at(self, b, pos):
        pos = np.asarray(pos)
        return (self.table[b][pos // self.page], pos % self.page) if self.page else (np.full_like(pos, b), pos)


def weights(x):
    """Softmax over the last axis in place of scores; a row of -inf gives zeros."""
    top = x.max(-1, keepdims=True)
    with np.errstate(invalid="ignore"):
        e = np.where(x == -np.inf, 0.0, np.exp(x - np.where(np.isfinite(top), top, 0.0)))
    s = e.sum(-1, keepdims=True)
    return e / np.where(s == 0, 1.0, s)


def attend(q, k, v, spread, L, mask, scale):
    """q [T, G, D]; k, v, spread [L + N, D] of one kv-head; mask [T, N]. The outputs, and how far rounding each weight to
    bf16 can move them per unit of relative error: sum_p w_p spread_p."""
    x = np.einsum("tgd,pd->tgp", q, k) * scale
    seen = np.concatenate([np.ones((q.shape[0], L), bool), mask], 1)
    x = np.where(seen[:, None], x, -np.inf)
    w = weights(x)
    vis = np.where(seen[:, None] & (w > 0), 1.0, 0.0)
    clean = np.isfinite(v).all(1)
    o = np.einsum("tgp,pd->tgd", w[..., clean], v[clean])
    o[(vis[..., ~clean] > 0).any(-1)] = np.nan
    return o, np.einsum("tgp,pd->tgd", w[..., clean], spread[clean])


def mass_of(q, k, seen_to, scale):
    """Summed weights [P] of rows q [n, G, D], row i seeing the positions below seen_to[i]."""
    x = np.einsum("tgd,pd->tgp", q, k) * scale
    x = np.where((np.arange(k.shape[0])[None] < np.asarray(seen_to)[:, None])[:, None], x, -np.inf)
    return weights(x).sum((0, 1))


def keep(mass, n, budget, recent):
    """Kept positions, ascending, of a sequence of n positions with weights mass[:n]."""
    if n <= budget:
        return np.arange(n)
    m = np.where(np.isnan(mass[:n - recent]), -np.inf, mass[:n - recent])
    nan = np.isnan(mass[:n - recent])
    order = np.lexsort((np.arange(n - recent), nan, -m))  # weight descending, NaN behind -inf, lower position first
    return np.sort(np.concatenate([order[:budget - recent], np.arange(n - recent, n)])).astype(np.int64)

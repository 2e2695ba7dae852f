"""Appending rows, chunk attention and windowed tree attention in plain numpy, 64 bits: what the kernels are compared with."""
import numpy as np


def normalised(x, weight, eps):
    return x if weight is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)


def rotated(x, pos, inv_freq, interleaved, magnitude):
    """x [rows, heads, D]; pos [rows]. The first 2 len(inv_freq) dims turn."""
    r = 2 * len(inv_freq)
    if r == 0:
        return x
    lo = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
    hi = lo + (1 if interleaved else r // 2)
    z = (x[..., lo] + 1j * x[..., hi]) * (magnitude * np.exp(1j * (np.asarray(pos, np.float64)[:, None] * inv_freq)))[:, None]
    y = x.copy()
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def sight(L, stands, window, sinks, tree=None):
    """Whether rows see positions [T, L + T]: `stands` [T] is the position of a row; `tree` [T, T] its mask, or causal."""
    pos = np.concatenate([np.arange(L), stands])
    seen = pos[None] <= stands[:, None]
    if tree is not None:
        seen[:, L:] = tree
    if window:
        seen &= (stands[:, None] - pos[None] < window) | (pos[None] < sinks)
    return seen


def attend(q, k, v, seen, scale):
    """q [T, G, D]; k, v [P, D] of one kv-head; seen [T, P]. The outputs, sum_p w_p |v_p|, and the largest sum_d |q_d k_d| that a row sees."""
    hidden_k = np.where(seen.any(0)[:, None], k, 0.0)
    x = np.einsum("tgd,pd->tgp", q, hidden_k) * scale
    with np.errstate(invalid="ignore"):
        size = np.where(seen[:, None], np.einsum("tgd,pd->tgp", np.abs(q), np.abs(hidden_k)) * abs(scale), 0.0).max(-1, initial=0.0)
        x = np.where(seen[:, None], x, -np.inf)
        top = x.max(-1, keepdims=True, initial=-np.inf)
        e = np.where(seen[:, None], np.exp(x - np.where(top == -np.inf, 0.0, top)), 0.0)
    s = e.sum(-1, keepdims=True)
    w = e / np.where(s == 0, 1.0, s)
    clean = np.isfinite(v).all(1)
    o = np.einsum("tgp,pd->tgd", w[..., clean], v[clean])
    spread = np.einsum("tgp,pd->tgd", w, np.abs(np.where(np.isfinite(v), v, 0.0)))
    for p in np.flatnonzero(~clean):  # one by one: 0 times infinity is no term of the sum where the row does not see it
        hit = seen[:, p]
        with np.errstate(invalid="ignore"):
            o[hit] += w[hit][..., p:p + 1] * v[p]
    return o, spread, size

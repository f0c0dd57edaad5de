"""Float64 definitions of the serving operators (prompt attention, paged cache), one
row, slot and head at a time, and the error bounds the GPU tests hold them to.

Bounds: a dot product of d float32 terms is off by at most (d + 2) 2^-24 of the sum
of its terms' magnitudes (dx, in natural-log units); a probability then is off by
2 dx relative (itself and its normaliser), the float32 exponential, sum and division
by less than 2^-19 together.  A rounding to bf16 is off by 2^-8 relative."""
import math

import numpy as np

U24, U_BF16 = 2.0 ** -24, 2.0 ** -8
EXP = 2.0 ** -19


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(dtype):
    """Half a step of a torch type, relative."""
    import torch
    return torch.finfo(dtype).eps / 2


def attend(q, k, v, seen):
    """One query row over keys [n][d]: out, lse, weights, bound of a logit's error."""
    d = q.shape[-1]
    out, w = np.zeros(d), np.zeros(len(k))
    if not seen.any():
        return out, -math.inf, w, 0.0
    ks = k[seen]
    x = ks @ q / math.sqrt(d)
    dx = (d + 2) * U24 * float(np.max(np.abs(ks) @ np.abs(q))) / math.sqrt(d)
    top = x.max()
    e = np.exp(x - top)
    w[seen] = e / e.sum()
    return w[seen] @ v[seen], top + math.log(e.sum()), w, dx


def visible(n, keys, position, window, sinks):
    """Which of `keys` slots a row at `position` of a sequence of n keys sees."""
    t = np.arange(keys)
    seen = (t < n) & (t <= position)
    if window:
        seen &= (t > position - window) | (t < sinks)
    return seen


def rows_of(table, n_slots, page, n_pages):
    """(page, row) of every slot of a sequence; page -1 where the entry is not a page."""
    s = np.arange(n_slots)
    p = table[s // page]
    return np.where((p >= 0) & (p < n_pages), p, -1), s % page


def evict(acc, pos, has_page, n, budget, window, sinks, seen):
    """One head's eviction: the slot that each slot below the budget gets its content
    from (-1 behind n) and the new length."""
    if n <= budget:
        return np.array([s if s < n else -1 for s in range(budget)]), n
    def rank(s):
        if not has_page[s]:
            return (3, 0.0, s)
        if pos[s] < sinks or (window > 0 and pos[s] >= seen - window):
            return (0, 0.0, s)
        return (2, 0.0, s) if math.isnan(acc[s]) else (1, -float(acc[s]), s)
    kept = set(sorted(range(n), key=rank)[:budget])
    late = sorted(s for s in kept if s >= budget)
    holes = [s for s in range(budget) if s not in kept]
    source = list(range(budget))
    for d, s in zip(holes, late):
        source[d] = s
    return np.array(source), budget


def rotated(x, weight, eps, position, inv_freq):
    """One head's row, normed and rotated; and the bound of its float32 error."""
    x = x.copy()
    off = np.zeros_like(x)
    if weight is not None:
        x = x / math.sqrt(float(np.mean(x * x)) + eps) * weight
        off += np.abs(x) * (len(x) / 2 + 8) * U24  # sum of squares (halved by the root), root, two products
    if inv_freq is not None:
        h = len(inv_freq)
        a = float(position) * inv_freq
        lo, hi = x[:h].copy(), x[h:2 * h].copy()
        size = np.abs(lo) + np.abs(hi)
        x[:h] = lo * np.cos(a) - hi * np.sin(a)
        x[h:2 * h] = hi * np.cos(a) + lo * np.sin(a)
        o = off[:h] + off[h:2 * h]
        # the angle in half turns is rounded to float32 (pi 2^-25), sine and cosine to 4 steps
        off[:h] = off[h:2 * h] = o + size * (2 ** -23 + 8 * U24)
    return x, off

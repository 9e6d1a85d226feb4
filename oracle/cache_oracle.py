"""Plain fp64 oracle of packed prompts with grouped heads and of the 8-bit cache (numpy, one head at a time).

Nothing here is shared with the library or with the plain forms it is timed against.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64


# ------------------------------------------------------------------------------------------------ packed prompts
def packed_attend(q, k, v, lens):
    """q [total, H, D], k and v [total, G, D]: (out [total, H, D], lse [H, total], spread [total, H, D], reach [H, total]).
    spread is sum_j p_j |v_j| and reach max_j sum_d |q_d k_jd| / sqrt(D), which bounds on rounding errors are made of."""
    total, heads, dim = q.shape
    group = heads // k.shape[1]
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.zeros((heads, total)), np.zeros((heads, total))
    lo = 0
    for n in lens:
        for h in range(heads):
            x = q[lo:lo + n, h] @ k[lo:lo + n, h // group].T / math.sqrt(dim)
            seen = np.tril(np.ones((n, n), bool))
            x = np.where(seen, x, -np.inf)
            if n:
                top = x.max(1, keepdims=True)
                e = np.exp(x - top)
                s = e.sum(1, keepdims=True)
                out[lo:lo + n, h] = e / s @ v[lo:lo + n, h // group]
                spread[lo:lo + n, h] = e / s @ np.abs(v[lo:lo + n, h // group])
                lse[h, lo:lo + n] = (np.log(s) + top)[:, 0]
                reach[h, lo:lo + n] = (np.abs(q[lo:lo + n, h]) @ np.abs(k[lo:lo + n, h // group]).T * seen).max(1) / math.sqrt(dim)
        lo += n
    return out, lse, spread, reach


def packed_weights(q, k, lse, lens, window=0):
    """One [G, n] array per sequence: what each token has received from the last `window` queries (0: all)."""
    heads, dim = q.shape[1:]
    group, got, lo = heads // k.shape[1], [], 0
    for n in lens:
        w = np.zeros((k.shape[1], n))
        begin = max(0, n - window) if window else 0
        for h in range(heads):
            x = q[lo + begin:lo + n, h] @ k[lo:lo + n, h // group].T / math.sqrt(dim)
            p = np.exp(x - lse[h, lo + begin:lo + n, None])
            w[h // group] += (p * (np.arange(n)[None] <= np.arange(begin, n)[:, None])).sum(0)
        got.append(w)
        lo += n
    return got


# -------------------------------------------------------------------------------------------------- the cache
def block_scale(rows):
    """The smallest 2^e, -60 <= e <= 60, with max|rows| <= 127 * 2^e."""
    top = float(np.abs(rows).max()) if rows.size else 0.0
    e = -60
    while e < 60 and top > 127.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def codes(rows, scale):
    return np.clip(np.rint(rows / scale), -127, 127)


class Head:
    """The rows of one (sequence, head): values, position and weight of each, and the scale of each block of 64."""

    def __init__(self, dim):
        self.k, self.v = np.zeros((0, dim)), np.zeros((0, dim))
        self.ks, self.vs = [], []
        self.ids, self.weights = [], []

    def __len__(self):
        return len(self.ids)

    def store(self, k, v, pos=None):
        start = len(self)
        pos = start if pos is None else pos
        for name, new in (("k", k), ("v", v)):
            rows, scales = np.concatenate([getattr(self, name), new]), getattr(self, name + "s")
            for r in range(start // BLOCK * BLOCK, len(rows), BLOCK):
                fresh = max(r, start)
                need = block_scale(rows[fresh:r + BLOCK])
                if r < start:
                    scales[r // BLOCK] = max(scales[r // BLOCK], need)
                else:
                    scales.append(need)
                s = scales[r // BLOCK]
                rows[r:r + BLOCK] = codes(rows[r:r + BLOCK], s) * s
            setattr(self, name, rows)
        self.ids += list(range(pos, pos + len(k)))
        self.weights += [0.0] * len(k)

    def attend(self, q):
        """q [group, D]: (out, probabilities [group, rows], spread, reach)."""
        if not len(self):
            return np.zeros(q.shape), np.zeros((len(q), 0)), np.zeros(q.shape), 0.0
        x = q @ self.k.T / math.sqrt(q.shape[1])
        e = np.exp(x - x.max(1, keepdims=True))
        p = e / e.sum(1, keepdims=True)
        return p @ self.v, p, p @ np.abs(self.v), (np.abs(q) @ np.abs(self.k).T).max() / math.sqrt(q.shape[1])

    def evict(self, keep, recent, seen):
        n = len(self)
        if n <= keep:
            return
        fresh = [i >= seen - recent for i in self.ids]
        weight = [-math.inf if math.isnan(w) else w for w in self.weights]
        order = sorted(range(n), key=lambda r: (not fresh[r], 0.0 if fresh[r] else -weight[r], self.ids[r]))
        stay = set(order[:keep])
        movers = iter(sorted(r for r in stay if r >= keep))
        src = [r if r in stay else next(movers) for r in range(keep)]
        for name in "kv":
            rows, scales = getattr(self, name)[src], getattr(self, name + "s")[:-(-keep // BLOCK)]
            for b in range(len(scales)):
                at = slice(b * BLOCK, (b + 1) * BLOCK)
                if any(s != r for r, s in list(enumerate(src))[at]):
                    scales[b] = block_scale(rows[at])
                    rows[at] = codes(rows[at], scales[b]) * scales[b]
            setattr(self, name, rows)
            setattr(self, name + "s", scales)
        self.ids = [self.ids[r] for r in src]
        self.weights = [self.weights[r] for r in src]

"""Plain 64-bit statements of the 8-bit key/value cache's operators and of the rotary positions, for the tests.

A cache is held here as what it stands for: values [layers, rows, kv heads, slots, size] (float64) and the exponents [layers, rows, kv heads, blocks] of the
powers of two that its blocks share."""
import math

import numpy as np

BLOCK = 32
LEAST = -110


def round_e4m3(x):
    """Nearest e4m3 number, ties to even (|x| <= 448; what is not finite becomes NaN)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    _, e = np.frexp(a)                                     # a = m 2^e, m in [1/2, 1)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(np.isfinite(x), np.rint(x / step) * step, np.nan)


def exponent(top):
    """Smallest E >= LEAST with top <= 448 * 2^E."""
    e = LEAST
    while top > math.ldexp(448.0, e):
        e += 1
    return e


class Cache:
    def __init__(self, layers, rows, kv_heads, capacity, size):
        blocks = -(-capacity // BLOCK)
        self.capacity = capacity
        self.k, self.v = (np.zeros((layers, rows, kv_heads, blocks * BLOCK, size)) for _ in range(2))
        self.ke, self.ve = (np.full((layers, rows, kv_heads, blocks), LEAST) for _ in range(2))

    def append(self, layer, r, start, k, v):
        """k, v [tokens, kv heads, size] of one layer and row into slots start .. (what does not fit is dropped)."""
        n = max(0, min(k.shape[0], self.capacity - start))
        for x, held, ex in ((k, self.k, self.ke), (v, self.v, self.ve)):
            for h in range(x.shape[1]):
                for b in range(start // BLOCK, (start + n - 1) // BLOCK + 1 if n else 0):
                    lo, hi = max(start, b * BLOCK), min(start + n, (b + 1) * BLOCK)
                    new = np.asarray(x[lo - start:hi - start, h], dtype=np.float64)
                    fin = np.abs(new[np.isfinite(new)])
                    e = exponent(fin.max() if fin.size else 0.0)
                    if lo > b * BLOCK:
                        e = max(e, ex[layer, r, h, b])
                        old = held[layer, r, h, b * BLOCK:lo]
                        held[layer, r, h, b * BLOCK:lo] = round_e4m3(old / 2.0 ** e) * 2.0 ** e
                    held[layer, r, h, lo:hi] = round_e4m3(new / 2.0 ** e) * 2.0 ** e
                    ex[layer, r, h, b] = e

    def evict(self, layer, r, length, keep, recent, mass, pos):
        """mass, pos [kv heads, slots] of one layer and row.  Returns (mass, pos) afterwards, zeros behind the new length."""
        left = min(length, keep)
        mass_out, pos_out = np.zeros_like(mass), np.zeros_like(pos)
        for h in range(mass.shape[0]):
            origin = list(range(left))
            if length > keep:
                newest = int(pos[h, :length].max())

                def rank(i):
                    if pos[h, i] > newest - recent:
                        return (2, 0.0)
                    return (1, 0.0) if np.isnan(mass[h, i]) else (0, float(mass[h, i]))

                order = sorted(range(length), key=lambda i: (rank(i)[0], rank(i)[1], -i), reverse=True)
                kept = set(order[:keep])
                sources = [i for i in range(keep, length) if i in kept]
                origin = [i if i in kept else sources.pop(0) for i in range(keep)]
                for held, ex in ((self.k, self.ke), (self.v, self.ve)):
                    was, was_e = held[layer, r, h].copy(), ex[layer, r, h].copy()
                    for b in range(keep // BLOCK):
                        from_ = origin[b * BLOCK:(b + 1) * BLOCK]
                        if from_ == list(range(b * BLOCK, (b + 1) * BLOCK)):
                            continue
                        e = max(was_e[i // BLOCK] for i in from_)
                        held[layer, r, h, b * BLOCK:(b + 1) * BLOCK] = round_e4m3(was[from_] / 2.0 ** e) * 2.0 ** e
                        ex[layer, r, h, b] = e
            mass_out[h, :left], pos_out[h, :left] = mass[h, origin], pos[h, origin]
        return mass_out, pos_out

    def attend(self, layer, r, length, q, k, v, see, scale, counted):
        """q [tokens, heads, size]; k, v [tokens, kv heads, size] or None; see [tokens, tokens].  Returns out, lse, weights of the cached slots and of the block
        tokens [kv heads, ...], and bounds on |scores| and |values| for the tolerances."""
        T, H, D = q.shape
        kv_heads = self.k.shape[2]
        G = H // kv_heads
        n_block = 0 if k is None else T
        out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
        mass, block = np.zeros((kv_heads, length)), np.zeros((kv_heads, n_block))
        top_s = top_v = 0.0
        for h in range(kv_heads):
            keys, vals = self.k[layer, r, h, :length], self.v[layer, r, h, :length]
            if k is not None:
                keys, vals = np.concatenate([keys, k[:, h]]), np.concatenate([vals, v[:, h]])
            vis = np.ones((T, length + n_block), dtype=bool)
            if n_block:
                vis[:, length:] = see
            for g in range(G):
                ask = q[:, h * G + g]
                for t in range(T):
                    m = vis[t]
                    if not m.any():
                        continue
                    s = keys[m] @ ask[t] * scale
                    size = np.abs(keys[m]) @ np.abs(ask[t]) * scale
                    top_s = max(top_s, size[np.isfinite(size)].max(initial=0.0))
                    top_v = max(top_v, np.abs(vals[m][np.isfinite(vals[m])]).max(initial=0.0))
                    top = s.max()
                    e = np.exp(s - top)
                    lse[t, h * G + g] = top + np.log(e.sum())
                    p = e / e.sum()
                    out[t, h * G + g] = p @ vals[m]
                    if t < counted:
                        w = np.zeros(length + n_block)
                        w[m] = p
                        mass[h] += w[:length]
                        block[h] += w[length:]
        return out, lse, mass, block, top_s, top_v


def ancestors(parent, n):
    """[n, n]: token i sees j (parent None: all up to itself)."""
    if parent is None:
        return np.tril(np.ones((n, n), dtype=bool))
    see = np.eye(n, dtype=bool)
    for j in range(1, n):
        see[j] |= see[parent[j - 1]]
    return see


def rope(x, pos, pairs, base, shared, halves, inverse=False):
    """x [tokens, heads, size] (float64), pos [tokens, axes]."""
    size, total = x.shape[-1], sum(pairs)
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    rate = [base ** (-2.0 * j / size) for j in range(total)] if shared else [base ** (-i / n) for n in pairs for i in range(n)]
    y = np.array(x, dtype=np.float64)
    for j in range(total):
        a, b = (j, j + total) if halves else (2 * j, 2 * j + 1)
        angle = pos[:, axis[j]].astype(np.float64) * rate[j] * (-1 if inverse else 1)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, a] * s + x[:, :, b] * c
    return y

"""Rotary positions, the 16-bit key/value cache, attention over it and drafts verified by sampling, in 64 bits on the CPU, written from their definition: rows one after the other, plain loops and numpy."""
import math

import numpy as np


def turned(x, positions, freq, part, interleaved, amplitude=1.0):
    """x [rows, heads, head_dim], each pair turned by position * frequency radians."""
    y = np.array(x, dtype=np.float64)
    for r, pos in enumerate(positions):
        for i, f in enumerate(freq):
            c, s = amplitude * math.cos(float(pos) * f), amplitude * math.sin(float(pos) * f)
            m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + part // 2)
            a, b = np.array(y[r, :, m]), np.array(y[r, :, n])
            y[r, :, m], y[r, :, n] = a * c - b * s, a * s + b * c
    return y


class Pool:
    """pages [page][head][2][tokens * hd] (64-bit numbers) as the library lays them out."""

    def __init__(self, pages, hd, page_tokens):
        self.pages, self.hd, self.pt = np.array(pages, dtype=np.float64), hd, page_tokens
        e = np.arange(hd)
        self.at = (np.stack([(e // 8) * 128 + t * 8 + e % 8 for t in range(16)]),
                   np.stack([(e // 32) * 512 + (t // 4) * 128 + (e % 16) * 8 + (e // 16 % 2) * 4 + t % 4 for t in range(16)]))

    def place(self, table, pos):
        """(page, block in it, token in the block) of a position; None where there is none."""
        if pos < 0 or pos // self.pt >= len(table) or not 0 <= table[pos // self.pt] < self.pages.shape[0]:
            return None
        return int(table[pos // self.pt]), pos % self.pt // 16, pos % 16

    def token(self, table, pos, which):
        """[heads, hd], or None"""
        p = self.place(table, pos)
        return None if p is None else self.pages[p[0], :, which][:, self.at[which][p[2]] + p[1] * 16 * self.hd]

    def write(self, table, pos, which, x):
        p = self.place(table, pos)
        if p is not None:
            self.pages[p[0], :, which, self.at[which][p[2]] + p[1] * 16 * self.hd] = np.asarray(x).T

    def append(self, start, prefix, tables, k, v):
        for s in range(len(prefix)):
            for i, row in enumerate(range(start[s], start[s + 1])):
                self.write(tables[s], prefix[s] + i, 0, k[row])
                self.write(tables[s], prefix[s] + i, 1, v[row])

    def keep(self, start, prefix, tables, path, accepted):
        for s in range(len(prefix)):
            for d in range(min(accepted[s] + 1, start[s + 1] - start[s])):
                l = path[start[s] + d]
                if d < l < start[s + 1] - start[s]:
                    for which in (0, 1):
                        x = self.token(tables[s], prefix[s] + l, which)
                        if x is not None:
                            self.write(tables[s], prefix[s] + d, which, x)

    def attention(self, start, prefix, tables, q, scale, masks=None):
        """(out, lse, sum of weight * |value|), [rows, heads, hd] and [rows, heads]; masks: a Python integer a row."""
        rows, heads, hd = q.shape
        out, lse, size = np.zeros((rows, heads, hd)), np.full((rows, heads), -np.inf), np.zeros((rows, heads, hd))
        for s in range(len(prefix)):
            n = start[s + 1] - start[s]
            there = [(t, self.token(tables[s], t, 0), self.token(tables[s], t, 1)) for t in range(prefix[s] + n)]
            there = [x for x in there if x[1] is not None]
            if not there:
                continue
            pos, K, V = np.array([x[0] for x in there]), np.stack([x[1] for x in there]), np.stack([x[2] for x in there])
            group = heads // K.shape[1]
            for i in range(n):
                row = start[s] + i
                if masks is None:
                    see = pos <= prefix[s] + i
                else:
                    see = np.array([p < prefix[s] or bool(masks[row] >> int(p - prefix[s]) & 1) for p in pos])
                if not see.any():
                    continue
                for h in range(heads):
                    x = scale * (K[see, h // group] @ q[row, h])
                    top = x.max()
                    w = np.exp(x - top)
                    lse[row, h] = top + math.log(w.sum())
                    out[row, h] = (w @ V[see, h // group]) / w.sum()
                    size[row, h] = (w @ np.abs(V[see, h // group])) / w.sum()
        return out, lse, size


def probabilities(x, t):
    """Of a row of logits at a temperature; None where it has none."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    top = x.max()
    if not np.isfinite(top):
        return None
    if not t > 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0
        return p
    e = np.exp((x - top) / t) if math.isfinite(t) else (x > -np.inf).astype(np.float64)
    return e / e.sum()


def drawn(w, u):
    """The lowest id at which the sum passes u times the whole; -1: nothing there."""
    total = np.cumsum(w)
    if not total[-1] > 0:
        return -1
    passed = np.nonzero(total > u * total[-1])[0]
    return int(passed[0]) if len(passed) else int(np.nonzero(w > 0)[0][-1])


def verify(start, logits, tokens, u, temperature, draft_probs=None, parent=None):
    """(accepted, next, path, probs)"""
    n, rows, vocab = len(start) - 1, logits.shape[0], logits.shape[1]
    accepted, following, path, probs = np.zeros(n, int), np.full(n, -1), np.full(rows, -1), np.zeros(rows)
    for s in range(n):
        r0, m = start[s], min(start[s + 1], rows) - start[s]
        if m <= 0:
            continue
        ps = [probabilities(logits[r0 + i], temperature[s]) for i in range(m)]
        up = [-1] + ([int(parent[r0 + i]) for i in range(1, m)] if parent is not None else list(range(m - 1)))
        probs[r0] = 1.0
        for i in range(1, m):
            t = tokens[r0 + i]
            if 0 <= up[i] < i and ps[up[i]] is not None and 0 <= t < vocab:
                probs[r0 + i] = ps[up[i]][t]
        node, depth, left = 0, 0, ps[0]
        path[r0] = 0
        for i in range(1, m):
            if up[i] != node or (parent is None and i != node + 1):
                continue
            t = int(tokens[r0 + i])
            good = left is not None and 0 <= t < vocab
            if draft_probs is not None:
                q = draft_probs[r0 + i].astype(np.float64)
                ok = good and u[r0 + i][0] * q[t] < left[t]
            else:
                ok = good and u[r0 + i][0] * left.sum() < left[t]
            if ok:
                node, depth, left = i, depth + 1, ps[i]
                path[r0 + depth] = i
            elif left is not None:
                if draft_probs is not None:
                    rest = np.maximum(left - np.where(np.isnan(q), np.inf, q), 0)
                    left = rest if rest.sum() > 0 else left
                    break
                left = left.copy()
                if good:
                    left[t] = 0.0
        accepted[s] = depth
        if left is not None:
            following[s] = drawn(left, u[r0 + node][1])
    return accepted, following, path, probs

"""The 8-bit key/value cache and the attention over it in 64 bits on the CPU, written from their definition: tokens one after the other, plain loops and numpy."""
import math

import numpy as np


def e4m3_values():
    """What the 256 codes stand for."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        v[c] = math.nan if (c & 127) == 127 else s * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return v


VALUES = e4m3_values()
_POS = VALUES[:127]                                        # ascending: code c has value _POS[c]


def encode(x):
    """Codes of 64-bit numbers of at most 448 in magnitude: the nearest value, the even code of two as near; not finite: 0x7F in magnitude."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    c = np.where(np.isfinite(x), c, 127)
    return (c | np.where(np.signbit(x) & ~np.isnan(x), 128, 0)).astype(np.uint8)


def need_byte(amax):
    """The byte of the smallest power of two, from 2^-100 on, that leaves no code above 448."""
    b = 27
    while amax > 448 * 2.0 ** (b - 127):
        b += 1
    return b


def scale_byte(b):
    return min(max(int(b), 1), 253)


class Pool:
    """codes [page][head][2][tokens * hd], scales [page][head][tokens / 16][2] as the library lays them out."""

    def __init__(self, codes, scales, hd, page_tokens):
        self.codes, self.scales, self.hd, self.pt = codes.copy(), scales.copy(), hd, page_tokens
        e = np.arange(hd)
        self.k_at = np.stack([(e // 16) * 256 + t * 16 + e % 16 for t in range(16)])
        self.v_at = np.stack([(e // 64) * 1024 + (t // 4) * 256 + (e % 16) * 16 + (e // 16 % 4) * 4 + t % 4 for t in range(16)])

    def place(self, table, pos):
        """(page, block in it, token in the block) of a position; None where there is none."""
        if pos < 0 or pos // self.pt >= len(table) or not 0 <= table[pos // self.pt] < self.codes.shape[0]:
            return None
        return int(table[pos // self.pt]), pos % self.pt // 16, pos % 16

    def token_codes(self, page, head, which, sub, t):
        at = (self.k_at, self.v_at)[which][t] + sub * 16 * self.hd
        return self.codes[page, head, which], at

    def append(self, row_start, prefix, tables, k, v):
        n_rows = k.shape[0]
        for s, table in enumerate(tables):
            r0, r1 = int(row_start[s]), min(int(row_start[s + 1]), n_rows)
            if r0 < 0 or r1 < r0 or prefix[s] < 0:
                continue
            i = r0
            while i < r1:
                pos = int(prefix[s]) + i - r0
                off, n = pos % 16, min(16 - pos % 16, r1 - i)
                at = self.place(table, pos)
                if at is not None:
                    page, sub, _ = at
                    for head in range(k.shape[1]):
                        for which, x in enumerate((k, v)):
                            x = x[i:i + n, head].astype(np.float64)
                            fin = np.abs(x[np.isfinite(x)])
                            old = scale_byte(self.scales[page, head, sub, which]) if off else 0
                            b = max(old, need_byte(fin.max() if fin.size else 0.0))
                            for t in range(off if b != old else 0):
                                arr, ix = self.token_codes(page, head, which, sub, t)
                                arr[ix] = encode(VALUES[arr[ix]] * 2.0 ** (old - b))
                            for t in range(n):
                                arr, ix = self.token_codes(page, head, which, sub, off + t)
                                arr[ix] = encode(x[t] * 2.0 ** (127 - b))
                            if b != old:
                                self.scales[page, head, sub, which] = b
                i += n

    def tokens(self, table, first, n):
        """(k, v) [n][heads][hd] and which of them exist."""
        heads = self.codes.shape[1]
        out, there = np.zeros((2, n, heads, self.hd)), np.zeros(n, dtype=bool)
        for i in range(n):
            at = self.place(table, first + i)
            if at is None:
                continue
            there[i] = True
            page, sub, t = at
            for head in range(heads):
                for which in (0, 1):
                    arr, ix = self.token_codes(page, head, which, sub, t)
                    out[which, i, head] = VALUES[arr[ix]] * 2.0 ** (scale_byte(self.scales[page, head, sub, which]) - 127)
        return out[0], out[1], there


def attention(pool, row_start, prefix, tables, q, scale, masks=None):
    """(out, lse, sum of weight * |value|, which rows belong to a sequence)."""
    n, heads, hd = q.shape
    out, lse, mag, mine = np.full(q.shape, np.nan), np.full((n, heads), np.nan), np.zeros(q.shape), np.zeros(n, dtype=bool)
    for s, table in enumerate(tables):
        r0, r1 = int(row_start[s]), min(int(row_start[s + 1]), n)
        if r0 < 0 or r1 <= r0 or prefix[s] < 0:
            continue
        total = min(int(prefix[s]) + r1 - r0, len(table) * pool.pt)
        k, v, there = pool.tokens(table, 0, total)
        group = heads // k.shape[1]
        p = np.arange(total)
        mine[r0:r1] = True
        for row in range(r0, r1):
            if masks is None:
                see = p <= prefix[s] + row - r0
            else:
                slot = p - int(prefix[s])
                see = (slot < 0) | ((slot < 64) & (((int(masks[row]) >> np.clip(slot, 0, 63).astype(object)) & 1).astype(bool) if total else True))
            see = see & there
            for h in range(heads):
                kk, vv = k[see, h // group], v[see, h // group]
                if not len(kk):
                    out[row, h], lse[row, h] = 0.0, -np.inf
                    continue
                sc = kk @ q[row, h].astype(np.float64) * scale
                m = np.max(sc)
                w = np.exp(sc - m)
                lse[row, h] = m + np.log(w.sum())
                w = w / w.sum()
                out[row, h], mag[row, h] = w @ vv, w @ np.abs(vv)
    return out, lse, mag, mine

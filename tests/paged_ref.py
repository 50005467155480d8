"""Reference of the paged KV cache and its attention, from the definitions: pages moved one by one in
Python, attention in 64 bits with numpy, no code of the package."""
import math

import numpy as np

PAGES, TABLE, CONTROL, CAPACITY = 32, 64, 4, 2


class Cache:
    """pages [N][L][2][heads][P][hd] (any numpy type), table [n][W], refs [N]; `err` collects bits."""

    def __init__(self, n_layers, heads, hd, n_pages, page, n, width, dtype=np.float32):
        self.P, self.W, self.n = page, width, n
        self.pages = np.zeros((n_pages, n_layers, 2, heads, page, hd), dtype)
        self.table = [[-1] * width for _ in range(n)]
        self.refs = [0] * n_pages
        self.err = 0

    def _bad(self, p, m, M):
        if m < 0 or m > M:
            return CONTROL
        return CAPACITY if p < 0 or p + m > self.W * self.P else 0

    def fork(self, parent=None, length=None):
        old = [list(line) for line in self.table]
        for b in range(self.n):
            p = parent[b] if parent is not None else b
            m = length[b] if length is not None else self.W * self.P
            if not -1 <= p < self.n or m < 0:
                self.err |= CONTROL
                continue
            self.table[b] = [old[p][i] if p >= 0 and i * self.P < m else -1 for i in range(self.W)]
        self._count()

    def _count(self):
        self.refs = [0] * len(self.refs)
        for line in self.table:
            for e in line:
                if e >= 0:
                    self.refs[e] += 1

    def reserve(self, pos, rows, M=None):
        M = self.W * self.P if M is None else M
        table, refs = [list(line) for line in self.table], list(self.refs)
        free = [e for e, r in enumerate(refs) if r == 0]
        copies, at = [], 0
        for b in range(self.n):
            bad = self._bad(pos[b], rows[b], M)
            if bad:
                self.err |= bad
                continue
            if rows[b] == 0:
                continue
            for i in range(pos[b] // self.P, (pos[b] + rows[b] - 1) // self.P + 1):
                e = table[b][i]
                if e >= 0 and refs[e] == 1:
                    continue
                if at == len(free):
                    self.err |= PAGES
                    return
                new, at = free[at], at + 1
                table[b][i] = new
                refs[new] = 1
                if e >= 0:
                    refs[e] -= 1
                    if pos[b] > i * self.P:
                        copies.append((new, e, pos[b] - i * self.P))
        self.table, self.refs = table, refs
        for new, e, kept in copies:
            self.pages[new, ..., :kept, :] = self.pages[e, ..., :kept, :]

    def compact(self):
        used = [e for e, r in enumerate(self.refs) if r]
        low = len(used)
        holes = [e for e in range(low) if not self.refs[e]]
        to = dict(zip([e for e in used if e >= low], holes))
        for a, z in to.items():
            self.pages[z] = self.pages[a]
        self.table = [[to.get(e, e) for e in line] for line in self.table]
        self._count()
        return low

    def append(self, layer, k, v, pos, rows):
        """k, v [n][M][heads][hd]"""
        for b in range(self.n):
            bad = self._bad(pos[b], rows[b], k.shape[1])
            if bad:
                self.err |= bad
                continue
            for m in range(rows[b]):
                p = pos[b] + m
                e = self.table[b][p // self.P]
                if e < 0 or self.refs[e] > 1:
                    self.err |= TABLE
                    continue
                self.pages[e, layer, 0, :, p % self.P] = k[b, m]
                self.pages[e, layer, 1, :, p % self.P] = v[b, m]

    def rows(self, layer, side, b, lo, hi):
        """Positions lo .. hi - 1 of sequence b as [heads][hi - lo][hd], 64 bits."""
        j = np.arange(lo, hi)
        at = np.asarray(self.table[b])[j // self.P]
        return self.pages[at, layer, side, :, j % self.P].astype(np.float64).transpose(1, 0, 2)


def attention(cache, layer, q, pos, rows, first, window, bits):
    """(out, bound) [n][M][heads][hd] in 64 bits of q (any type); nan where a row is not computed.
    bits: of an operand of the products (24, or 8 for a probability that is rounded to bf16).

    The bound of a row counts: the scores' sums of hd products in fp32 in blocks of 16 (each of hd / 16 + 1
    additions, and as many again for single additions in them, off by 2^-23 of the sum of magnitudes),
    their scaling and exponential (2^-22 each way of a score's magnitude in powers of two, plus
    2^-22); a probability rounded to `bits` bits (2^-bits); sums of n terms in fp32, each
    warp's in steps and the parts after one another (2^-24 times a generous 64 + n / 64); the result's
    own rounding is the caller's."""
    n, M, H, hd = q.shape
    kvh = cache.pages.shape[3]
    out = np.full((n, M, H, hd), np.nan)
    bound = np.full((n, M, H, hd), np.nan)
    for b in range(n):
        lo0 = max(first[b], 0)
        hi = pos[b] + rows[b]
        if rows[b] <= 0:
            continue
        lo = lo0 if window == 0 else max(lo0, pos[b] - window + 1)
        kk, vv = (cache.rows(layer, s, b, min(lo, hi), hi) for s in (0, 1))
        j = np.arange(min(lo, hi), hi)
        for m in range(rows[b]):
            p = pos[b] + m
            see = (j <= p) & (j >= lo0)
            if window:
                see &= j > p - window
            if not see.any():
                out[b, m], bound[b, m] = 0.0, 0.0
                continue
            x = q[b, m].astype(np.float64).reshape(kvh, H // kvh, hd)
            with np.errstate(all="ignore"):
                s = np.einsum("ghd,gjd->ghj", x, kk[:, see]) / math.sqrt(hd)
                mag = np.einsum("ghd,gjd->ghj", abs(x), abs(kk[:, see])) / math.sqrt(hd)
                e = np.exp(s - s.max(-1, keepdims=True))
                w = e / e.sum(-1, keepdims=True)
                o = np.einsum("ghj,gjd->ghd", w, vv[:, see])
                off = (2 * (hd / 16 + 1) * 2.0 ** -23 * mag + 2.0 ** -22 * abs(s) + 2.0 ** -22)
                off = off.max(-1, keepdims=True)
                rel = 2 * off + 2.0 ** -bits + (64 + see.sum() / 64) * 2.0 ** -24
                bd = rel * np.einsum("ghj,gjd->ghd", w, abs(vv[:, see]))
            out[b, m], bound[b, m] = o.reshape(H, hd), bd.reshape(H, hd)
    return out, bound

"""The 8-bit transformer operators in plain numpy, sums in 64 bits: the oracle of
their tests.  Codes and scales are formed in fp32, as their definition is."""
import numpy as np

F = np.float32
C127 = F(1.0) / F(127.0)
FLOOR = F(2.0) ** F(-100)


def scale_of(x):
    """Scale of a block of values (any shape)."""
    x = np.asarray(x, np.float32)
    if not np.isfinite(x).all():
        return F(np.nan)
    a = np.abs(x).max() if x.size else F(0)
    return max(F(a * C127), FLOOR)


def codes_of(x, s):
    if not np.isfinite(s):
        return np.zeros(np.shape(x), np.int8)
    return np.clip(np.rint(np.asarray(x, np.float32) * (F(1.0) / s)), -127, 127).astype(np.int8)


def quantize_rows(x):
    s = np.array([scale_of(r) for r in x], np.float32)
    return np.stack([codes_of(r, t) for r, t in zip(x, s)]) if len(x) else np.zeros(x.shape, np.int8), s


def linear(q, s, w, ws, bias=None):
    """In fp64, where the integer sums (below 2^53) are exact."""
    t = q.astype(np.float64) @ w.astype(np.float64).T
    y = t * s.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :]
    return y if bias is None else y + bias.astype(np.float64)


class Cache:
    """k, v int8 [pages, heads, page, dim] (both token by token here), scales [pages, heads]."""

    def __init__(self, pages, heads, page, dim):
        self.k = np.zeros((pages, heads, page, dim), np.int8)
        self.v = np.zeros((pages, heads, page, dim), np.int8)
        self.ks = np.ones((pages, heads), np.float32)
        self.vs = np.ones((pages, heads), np.float32)
        self.page = page

    def append(self, table, lens, starts, k, v):
        """The new rows of every request, block by block."""
        P = self.page
        for r, ln in enumerate(lens):
            n = starts[r + 1] - starts[r]
            for j0 in range(max(0, ln - n), ln):
                if j0 != max(0, ln - n) and j0 % P:
                    continue  # inside a block already taken
                j1 = min(ln, (j0 // P + 1) * P)
                pid, kept = table[r][j0 // P], j0 % P
                if not 0 <= pid < len(self.k):
                    continue
                rows = slice(starts[r] + j0 - (ln - n), starts[r] + j1 - (ln - n))
                for codes, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
                    for h in range(codes.shape[1]):
                        new = np.asarray(x[rows, h], np.float32)
                        s = scale_of(new)
                        if kept:
                            had = scales[pid, h]
                            if np.isnan(had) or np.isnan(s):
                                s = F(np.nan)
                            elif s > had:
                                old = codes[pid, h, :kept]
                                codes[pid, h, :kept] = np.rint(old.astype(np.float32) * (had / s)).astype(np.int8)
                            else:
                                s = had
                        scales[pid, h] = s
                        codes[pid, h, kept:kept + j1 - j0] = codes_of(new, s)

    def values(self, table, r, ln, h, which):
        """fp64 [ln, dim] of one request and head, and which tokens exist."""
        codes, scales = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        P = self.page
        out, there = np.zeros((ln, codes.shape[3])), np.zeros(ln, bool)
        for j in range(ln):
            pid = table[r][j // P]
            if 0 <= pid < len(codes):
                out[j] = codes[pid, h, j % P].astype(np.float64) * np.float64(scales[pid, h])
                there[j] = True
        return out, there

    def read(self, table, lens, starts):
        """fp32 k, v [rows, heads, dim] of the last tokens of every request."""
        heads, dim = self.k.shape[1], self.k.shape[3]
        out = [np.zeros((starts[-1], heads, dim), np.float32) for _ in range(2)]
        for o, which in zip(out, "kv"):
            for r, ln in enumerate(lens):
                n = starts[r + 1] - starts[r]
                for h in range(heads):
                    x, _ = self.values(table, r, ln, h, which)
                    m = min(n, ln)
                    if m:
                        o[starts[r + 1] - m:starts[r + 1], h] = x[ln - m:].astype(np.float32)
        return out

    def attend(self, table, lens, starts, q, scale, causal=True, window=0):
        """fp64 outputs and, for the error bound, sum p |v|, the largest |q| |k| sum, and the seen tokens of each row."""
        tokens, hq, dim = q.shape
        heads = self.k.shape[1]
        group = hq // heads
        out, mass = np.zeros((tokens, hq, dim)), np.zeros((tokens, hq, dim))
        reach, seen = np.zeros((tokens, hq)), np.zeros((tokens, hq))
        for r, ln in enumerate(lens):
            n = starts[r + 1] - starts[r]
            j = np.arange(ln)
            for h in range(heads):
                k, there = self.values(table, r, ln, h, "k")
                v, _ = self.values(table, r, ln, h, "v")
                for t in range(n):
                    sees = there.copy()
                    if causal:
                        pos = ln - n + t
                        sees &= j <= pos
                        if window:
                            sees &= j > pos - window
                    if not sees.any():
                        continue
                    for g in range(group):
                        x = q[starts[r] + t, h * group + g].astype(np.float64)
                        s = (k[sees] @ x) * scale
                        with np.errstate(invalid="ignore"):
                            p = np.exp(s - s.max())
                        p /= p.sum()
                        at = starts[r] + t, h * group + g
                        out[at], mass[at] = p @ v[sees], p @ np.abs(v[sees])
                        reach[at] = (np.abs(k[sees]) @ np.abs(x)).max() * abs(scale)
                        seen[at] = sees.sum()
        return out, mass, reach, seen

"""What stands around the cache in a generation step, in plain numpy with 64 bits and
more: the oracle of the tests of head norms with rotation, trees of drafted tokens,
attention with sinks and over trees, and log probabilities."""
import numpy as np


def new_tokens(starts, r):
    return starts[r + 1] - starts[r]


def sees_new(mask, row, b):
    """Bit b of a row of masks (uint64 [tokens, words])."""
    return b < 64 * mask.shape[1] and bool(int(mask[row, b // 64]) >> (b % 64) & 1)


def positions(lens, starts, mask=None):
    """Position of every row, row starts[r] first."""
    out = []
    for r, ln in enumerate(lens):
        n = new_tokens(starts, r)
        for t in range(n):
            if mask is None:
                out.append(ln - n + t)
            else:
                out.append(ln - n + sum(sees_new(mask, starts[r] + t, b) for b in range(n) if b != t))
    return np.array(out, np.int64)


def norm_rotate(x, pos, freq=(), interleaved=False, weight=None, eps=None):
    """longdouble result of x [tokens, heads, dim], and of each element the magnitudes that it comes from."""
    y = x.astype(np.longdouble)
    with np.errstate(all="ignore"):
        if eps is not None:
            y = y / np.sqrt((y * y).mean(-1, keepdims=True) + np.longdouble(np.float32(eps)))
            if weight is not None:
                y = y * weight.astype(np.longdouble)
        n = len(freq)
        out, size = y.copy(), np.abs(y)
        if n:
            a, b = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
            t = pos.astype(np.longdouble)[:, None] * np.asarray(freq, np.longdouble)
            c, s = np.cos(t)[:, None], np.sin(t)[:, None]
            ya, yb = y[..., a], y[..., b]
            out[..., a], out[..., b] = ya * c - yb * s, yb * c + ya * s
            size[..., a] = size[..., b] = np.abs(ya) + np.abs(yb)
    return out, size


def log_probs(x, scale, ids, top):
    """fp64 log probabilities of ids [rows, given], entropy, top ids and their log probabilities; and what their error
    bounds are made of: ln S and sums p t, p t^2 of t = (largest - x) scale."""
    rows, vocab = x.shape
    x = x.astype(np.float64)
    out, ent = np.full(ids.shape, np.nan), np.full(rows, np.nan)
    top_ids, top_out = np.full((rows, top), -1, np.int64), np.full((rows, top), np.nan)
    size = np.zeros((rows, 3))
    for r in range(rows):
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            continue
        most = x[r].max()
        order = np.argsort(-x[r], kind="stable")[:top]
        if most == -np.inf:
            l, ent[r] = np.full(vocab, -np.inf), 0.0
        else:
            with np.errstate(over="ignore"):
                t = (most - x[r]) * np.float64(np.float32(scale))
                w = np.exp(-t)
            s = w.sum()
            l = -t - np.log(s)
            live = w > 0
            p, t = w[live] / s, t[live]
            size[r] = np.log(s), (p * t).sum(), (p * t * t).sum()
            ent[r] = np.log(s) + size[r, 1]
        top_ids[r], top_out[r] = order, l[order]
        for g, i in enumerate(ids[r]):
            if 0 <= i < vocab:
                out[r, g] = l[i]
    return out, ent, top_ids, top_out, size


def attend(cache, table, lens, starts, q, scale, window=0, sinks=0, mask=None, limit=None):
    """As oracle.serve.Cache.attend: fp64 outputs, sum p |v|, the largest |q| |k| sum, the seen tokens of each row.  limit: the
    tokens that a request holds at most; later ones are left out, and positions stay."""
    tokens, hq, dim = q.shape
    heads = cache.k.shape[1]
    group = hq // heads
    out, mass = np.zeros((tokens, hq, dim)), np.zeros((tokens, hq, dim))
    reach, seen = np.zeros((tokens, hq)), np.zeros((tokens, hq))
    pos = positions(lens, starts, mask)
    for r, ln in enumerate(lens):
        n = new_tokens(starts, r)
        old = ln - n
        ln = ln if limit is None else min(ln, limit)
        j = np.arange(ln)
        for h in range(heads):
            k, there = cache.values(table, r, ln, h, "k")
            v, _ = cache.values(table, r, ln, h, "v")
            for t in range(n):
                row = starts[r] + t
                sees = there & (j <= pos[row - starts[0]])
                if window:
                    sees &= (j > pos[row - starts[0]] - window) | (j < sinks)
                if mask is not None:
                    for i in range(max(old, 0), ln):
                        sees[i] = there[i] and sees_new(mask, row, i - old)
                if not sees.any():
                    continue
                for g in range(group):
                    x = q[row, h * group + g].astype(np.float64)
                    s = (k[sees] @ x) * scale
                    with np.errstate(invalid="ignore"):
                        p = np.exp(s - s.max())
                    p /= p.sum()
                    at = row, h * group + g
                    out[at], mass[at] = p @ v[sees], p @ np.abs(v[sees])
                    reach[at] = (np.abs(k[sees]) @ np.abs(x)).max() * abs(scale)
                    seen[at] = sees.sum()
    return out, mass, reach, seen

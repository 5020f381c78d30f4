"""GPU checks of attention with sinks and over trees and of head norms with rotation where a batch's arrays go past its
bounds: starts before the first row, past the last one or backwards, lengths past the table, below 0 or near 2^31.  Results lie inside
larger tensors, whose other elements stay, as do rows of no request; the rows that are left are the oracle's."""
import numpy as np
import pytest

from tests.test_gpu_serve import EPS, TINY, Pair, dev, host, paged, say
from tests.test_gpu_step import check_rotated, freqs, masks_dev

pytestmark = pytest.mark.gpu
TOKENS, PAGE, WIDTH = 40, 16, 4
LIMIT = PAGE * WIDTH

WILD = [
    ([50, 60], [-5, 20, 50], 1 << 20),
    ([50, 60], [-5, 20, 50], 10),              # rows 0 to 4 of the first request, as its first five are outside
    ([70, 1 << 30], [3, 15, 40], 1 << 20),
    ([66, 64, 0], [-20, 9, 30, 38], 1 << 20),
    ([9, 9], [-5, 100, 7], 1 << 20),
    ([1 << 30, -4], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], 1 << 20),
    ([2 ** 31 - 1, 2 ** 31 - 1], [0, 20, 40], 1 << 20),
    ([3, 2 ** 31 - 1], [-2 ** 31, 0, 60], 1 << 20),
    ([-9, 5], [0, 30, 40], 1 << 20),
    ([64, 64], [30, 10, 25], 1 << 20),
]


def rows_of(lens, starts, max_new, masks=None):
    """For every row of a request: request, index among its new tokens, tokens before the first new one, position."""
    out = {}
    for r, ln in enumerate(lens):
        s0, s1 = starts[r], starts[r + 1]
        for row in range(max(s0, 0), min(s1, TOKENS, s0 + max_new)):
            old, new = ln - (s1 - s0), row - s0
            bits = set() if masks is None else {b for b in range(min(s1 - s0, 64 * masks.shape[1])) if int(masks[row, b // 64]) >> b % 64 & 1}
            out[row] = r, bits, old, old + (new if masks is None else len(bits - {new}))
    return out


def inside(shape, dtype):
    """A tensor of 7s, and a part of it with margins on every side."""
    import torch
    big = torch.full((shape[0] + 64, shape[1] + 2, shape[2]), 7.0, dtype=dtype, device="cuda")
    return big, big[32:-32, 1:-1]


@pytest.mark.parametrize("words", [0, 2])
@pytest.mark.parametrize("window,sinks", [(0, 0), (7, 3), (20, 50), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("lens,starts,max_new", WILD)
def test_attention(palq, lens, starts, max_new, window, sinks, words):
    import torch
    from paper_2208_01944_amd import palq as P
    say("wild attention", lens, starts, max_new, window, sinks, words)
    g = np.random.default_rng(len(lens) + words)
    dim, group = 64, 2
    table, pages = paged(g, [LIMIT] * len(lens), PAGE)
    pair = Pair(P, pages, 1, PAGE, dim)
    pair.fill(g, table, None)
    masks = g.integers(0, 1 << 63, (TOKENS, words), dtype=np.uint64) if words else None
    q = dev(g.standard_normal((TOKENS, group, dim)), "bf16")
    big, out = inside(q.shape, q.dtype)
    b = P.Batch(dev(table), dev(np.int32(lens)), dev(np.int32(starts)), max_new, 2 ** 31 - 1)
    palq.attention(pair.gpu, q, out, b, 0.125, window=window, sinks=sinks, tree=masks_dev(masks) if words else None)
    palq.sync()
    got, x = host(out), host(q).astype(np.float64)
    live = rows_of(lens, starts, max_new, masks)
    assert (got[[r for r in range(TOKENS) if r not in live]] == 7).all()
    out.fill_(7.0)
    assert (big == 7.0).all()
    for row, (r, bits, old, pos) in live.items():
        ln = max(0, min(lens[r], LIMIT))
        k, v = (pair.ref.values(table, r, ln, 0, w)[0] for w in "kv")
        j = np.arange(ln)
        sees = j <= pos
        if window:
            sees &= (j > pos - window) | (j < sinks)
        if words:
            sees[j >= old] = [t - old in bits for t in j[j >= old]]
        for h in range(group):
            if not sees.any():
                assert (got[row, h] == 0).all(), row
                continue
            # as tests/test_gpu_serve.py's check_attend: scores, weights in fp16, and the result's rounding
            s = k[sees] @ x[row, h] * 0.125
            p = np.exp(s - s.max())
            p /= p.sum()
            want, mass = p @ v[sees], p @ np.abs(v[sees])
            es = (dim + 8) * 2.0 ** -24 * (np.abs(k[sees]) @ np.abs(x[row, h])).max() * 0.125 + 2.0 ** -15
            tol = mass * (2.0 ** -11 + 2 * es) + sees.sum() * 2.0 ** -25 * 127 * float(pair.ref.vs.max())
            tol += EPS["bf16"] * (np.abs(want) + tol) + TINY["bf16"]
            assert (np.abs(got[row, h] - want) <= tol).all(), (row, h)


@pytest.mark.parametrize("words", [0, 2])
@pytest.mark.parametrize("lens,starts,max_new", [w for w in WILD if min(w[0]) >= 0])
def test_norm_rotate(palq, lens, starts, max_new, words):
    from paper_2208_01944_amd import palq as P
    say("wild rotation", lens, starts, max_new, words)
    g = np.random.default_rng(len(lens) + words)
    masks = g.integers(0, 1 << 63, (TOKENS, words), dtype=np.uint64) if words else None
    q, k = dev(g.standard_normal((TOKENS, 5, 64)), "f16"), dev(g.standard_normal((TOKENS, 3, 64)), "f16")
    (qb, qo), (kb, ko) = inside(q.shape, q.dtype), inside(k.shape, k.dtype)
    f = freqs(32)
    b = P.Batch(dev(np.full((len(lens), 1), -1, np.int32)), dev(np.int32(lens)), dev(np.int32(starts)), max_new, 2 ** 31 - 1)
    palq.norm_rotate(b, q, qo, k, ko, eps=1e-6, rotation=P.Rotation(palq, f), tree=masks_dev(masks) if words else None)
    palq.sync()
    live = rows_of(lens, starts, max_new, masks)
    at, pos = list(live), np.array([p for _, _, _, p in live.values()], np.int64)
    for x, big, out in ((q, qb, qo), (k, kb, ko)):
        got = host(out)
        assert (got[[r for r in range(TOKENS) if r not in live]] == 7).all()
        check_rotated(got[at], host(x)[at], pos, "f16", freq=f, eps=1e-6)
        out.fill_(7.0)
        assert (big == 7.0).all()

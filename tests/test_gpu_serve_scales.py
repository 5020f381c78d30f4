"""Attention over blocks whose value scales lie far apart, against the numpy oracle,
channel by channel: a block of a large scale must not cost the channels in which it
holds zeros any of the other blocks' bits."""
import numpy as np
import pytest

from tests.test_gpu_serve import EPS, TINY, Pair, cumsum, dev, host, paged, say

pytestmark = pytest.mark.gpu


def check_channels(pair, got, table, lens, starts, q, scale, dtype, causal=True, window=0):
    """Bound for each output channel d: as in check_attend, but the weights' absolute rounding (half a subnormal fp16 step,
    2^-25, of a weight of which the largest is 1 / 2 or more of L) counts with each token's own |v_jd|: blocks below 2^-20 of
    the largest scale of their 64 tokens, or 2^-72 of all, are rounded as blocks of that scale are."""
    ref, mass, reach, _ = pair.ref.attend(table, lens, starts, q, scale, causal, window)
    tokens, hq, dim = q.shape
    heads, page = pair.ref.k.shape[1], pair.ref.page
    group, sub = hq // heads, np.zeros_like(ref)
    for r, ln in enumerate(lens):
        n, j = starts[r + 1] - starts[r], np.arange(ln)
        pid = np.array([table[r][i // page] for i in j], int)
        for h in range(heads):
            v, there = pair.ref.values(table, r, ln, h, "v")
            vs = np.where(there, pair.ref.vs[np.where(there, pid, 0), h].astype(np.float64), 0.0)
            vs = np.where(np.isfinite(vs), vs, 0.0)
            most = np.array([vs[i // 64 * 64:i // 64 * 64 + 64].max() for i in j])
            with np.errstate(divide="ignore", invalid="ignore"):
                up = np.maximum(1.0, np.maximum(2.0 ** -20 * most, 2.0 ** -72 * vs.max(initial=0.0)) / vs)
                w = np.where(vs > 0, np.abs(v).T * up, 0.0).T if ln else v
            for t in range(n):
                pos = ln - n + t
                sees = (j <= pos if causal else j >= 0) & (j > pos - window if causal and window else j >= 0)
                sub[starts[r] + t, h * group:(h + 1) * group] = 2.0 ** -24 * w[sees].sum(0)
    es = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -15
    tol = mass * (2.0 ** -11 + 2 * es)[..., None] + sub
    tol = tol + EPS[dtype] * (np.abs(ref) + tol) + TINY[dtype]
    if dtype == "f16":  # past its range: inf
        over = np.abs(ref) >= 65520
        assert (got[over] == np.copysign(np.inf, ref[over])).all()
        got, ref = np.where(over, 0, got), np.where(over, 0, ref)
    err = np.abs(got - ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaN in the wrong places"
    bad = err > tol
    assert not bad.any(), f"{bad.sum()} of {err.size} off, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.3g} of the bound"


# few rows of 16 and 32 a workgroup, with splits, and the 128-row kernel (more than 768 blocks of 32 rows)
SHAPES = {"rows16": (2, 2, [200, 131], [1, 5], None), "rows32": (1, 4, [300, 90], [40, 7], None),
          "splits": (1, 2, [2100], [1], 5000), "tiles": (16, 2, [128, 150, 131, 260, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], None)}


def case(P, shape, page, dim, seed):
    heads, group, lens, new, max_len = SHAPES[shape]
    g = np.random.default_rng(seed)
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, heads, page, dim)
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], heads * group, dim)), "bf16")
    return g, pair, table, lens, starts, q, pair.batch(table, lens, starts, max_len=max_len)


def attend(palq, pair, table, lens, starts, q, b, scale=0.125, **kw):
    import torch
    out = torch.full_like(q, 3.0)
    palq.attention(pair.gpu, q, out, b, scale, **kw)
    palq.sync()
    check_channels(pair, host(out), table, lens, starts, host(q), scale, "bf16", **kw)
    return host(out)


@pytest.mark.parametrize("power", [10, 16, 20, 24, 40, 70])
@pytest.mark.parametrize("shape,page,dim", [("rows16", 16, 64), ("rows16", 64, 128), ("rows32", 32, 96), ("rows32", 64, 128),
                                            ("rows16", 128, 256), ("splits", 64, 64), ("splits", 16, 128), ("tiles", 16, 64),
                                            ("tiles", 64, 128), ("tiles", 128, 96)])
def test_attention_one_large_element(palq, shape, page, dim, power):
    """One value of 2^power among ordinary ones, in every head of every request: its block's other codes are 0, and the other
    channels come from the other blocks alone."""
    from paper_2208_01944_amd import palq as P
    say("one large element", shape, page, dim, power)
    g, pair, table, lens, starts, q, b = case(P, shape, page, dim, power)
    heads, whole = pair.ref.k.shape[1], cumsum(lens)
    k, v = (g.standard_normal((whole[-1], heads, dim)).astype(np.float32) for _ in range(2))
    for r, ln in enumerate(lens):
        for h in range(heads):
            v[whole[r] + (ln // 3 + h * 7) % ln, h, (5 + h) % dim] = 2.0 ** power
    pair.ref.append(table, lens, whole, k, v)
    palq.cache_append(pair.gpu, dev(k), dev(v), pair.batch(table, lens, whole))
    palq.sync()
    for kw in (dict(), dict(window=60)):
        attend(palq, pair, table, lens, starts, q, b, **kw)


@pytest.mark.parametrize("shape,page,dim", [("rows16", 16, 64), ("rows32", 64, 128), ("splits", 32, 128), ("tiles", 16, 64), ("tiles", 64, 128)])
def test_attention_zero_value_scales(palq, shape, page, dim):
    """Value scales of 0, which other quantisers give a block of zeros, whatever its codes: its tokens count in the softmax
    with the value 0.  Blocks of zeros as this library appends them (scale 2^-100) lie among them.  Then nothing but zeros."""
    from paper_2208_01944_amd import palq as P
    say("zero scales", shape, page, dim)
    g, pair, table, lens, starts, q, b = case(P, shape, page, dim, 2)
    pair.fill(g, table, lens)
    r = pair.ref
    kind = g.integers(0, 4, r.vs.shape)
    r.vs[kind == 0] = 0
    r.vs[kind == 1] = 2.0 ** -100
    r.v[kind == 1] = 0
    pair.upload()
    for kw in (dict(), dict(window=60), dict(causal=False)):
        attend(palq, pair, table, lens, starts, q, b, **kw)
    r.vs[:] = 0
    pair.upload()
    assert not attend(palq, pair, table, lens, starts, q, b).any()


@pytest.mark.parametrize("shape,page,dim,spread", [("rows16", 64, 64, 30), ("rows16", 16, 128, 9), ("rows32", 64, 128, 30), ("rows32", 32, 64, 9),
                                                   ("splits", 128, 128, 30), ("splits", 16, 64, 9), ("tiles", 64, 128, 30),
                                                   ("tiles", 128, 64, 30), ("tiles", 16, 128, 9)])
def test_attention_scales_of_any_size(palq, shape, page, dim, spread):
    """Value scales of 2^-spread to 2^spread at random, their codes dense or in a few channels; a NaN among them."""
    from paper_2208_01944_amd import palq as P
    say("any scales", shape, page, dim, spread)
    g, pair, table, lens, starts, q, b = case(P, shape, page, dim, 3)
    pair.fill(g, table, lens)
    r = pair.ref
    r.vs[:] = np.exp2(g.uniform(-spread, spread, r.vs.shape))
    few = g.random(r.vs.shape) < 0.5
    r.v[few] *= (g.random((few.sum(), 1, dim)) < 0.1).astype(np.int8)
    pair.upload()
    for kw in (dict(), dict(window=70), dict(causal=False)):
        attend(palq, pair, table, lens, starts, q, b, **kw)
    r.vs[table[0][lens[0] // page // 2], 0] = np.nan
    pair.upload()
    with np.errstate(invalid="ignore"):
        out = attend(palq, pair, table, lens, starts, q, b)
    assert np.isnan(out).any()


@pytest.mark.parametrize("power", [10, 20, 26])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape,page,dim", [("rows16", 16, 64), ("rows32", 64, 96), ("splits", 32, 128), ("rows16", 64, 256), ("tiles", 16, 64)])
def test_attention_one_large_query_element(palq, shape, page, dim, dtype, power):
    """One element of a query 2^power times the others, in a channel in which the keys are 0: scores come from the others."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("one large query element", shape, page, dim, dtype, power)
    g, pair, table, lens, starts, q, b = case(P, shape, page, dim, 4)
    pair.fill(g, table, lens)
    pair.ref.k[..., 5] = 0
    pair.upload()
    x = g.standard_normal(tuple(q.shape)) * 2.0 ** (-13 if dtype == "f16" else 0)
    x[..., 5] = 2.0 ** (power - (13 if dtype == "f16" else 0)) * 1.5
    q = dev(x, dtype)
    out = torch.full_like(q, 3.0)
    scale = 0.125 * 2.0 ** (13 if dtype == "f16" else 0)
    palq.attention(pair.gpu, q, out, b, scale)
    palq.sync()
    check_channels(pair, host(out), table, lens, starts, host(q), scale, dtype)


@pytest.mark.parametrize("shape", ["rows16", "rows32", "splits", "tiles"])
@pytest.mark.parametrize("scale", [1.75 * 2.0 ** 127, -1.75 * 2.0 ** 127, 2.0 ** -120])
def test_attention_scales_of_the_scores_near_the_ends(palq, shape, scale):
    """Finite scales whose product with log2(e) is none, and tiny ones, with queries and keys that bring the scores back."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("score scale", shape, scale)
    g, pair, table, lens, starts, q, b = case(P, shape, 16, 64, 6)
    pair.fill(g, table, lens)
    q = dev(g.standard_normal(tuple(q.shape)) * (2.0 ** -100 if abs(scale) > 1 else 2.0 ** 90), "bf16")
    pair.ref.ks[:] *= np.float32(2.0 ** -30 if abs(scale) > 1 else 2.0 ** 27)
    pair.upload()
    out = torch.full_like(q, 3.0)
    palq.attention(pair.gpu, q, out, b, scale)
    palq.sync()
    check_channels(pair, host(out), table, lens, starts, host(q), scale, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,dim", [(16, 64), (64, 128), (32, 96), (128, 64)])
@pytest.mark.parametrize("shape", ["rows16", "rows32", "splits", "tiles"])
def test_attention_of_one_token_is_its_value(palq, shape, page, dim, dtype):
    """A row that sees one token gives its value: the largest weight of a row is held exactly, so that the result has the
    rounding to its type and the fp32 errors of one logarithm, two powers and a division (below 2^-18) alone."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("one token", shape, page, dim, dtype)
    g, pair, table, lens, starts, q, b = case(P, shape, page, dim, 7)
    pair.fill(g, table, lens)
    q = q.to(torch.float16 if dtype == "f16" else torch.bfloat16)
    out = torch.full_like(q, 3.0)
    palq.attention(pair.gpu, q, out, b, 0.125, window=1)
    palq.sync()
    ref = pair.ref.attend(table, lens, starts, host(q), 0.125, True, 1)[0]
    err = np.abs(host(out) - ref)
    assert (err <= (EPS[dtype] * (1 + 2.0 ** -10) + 2.0 ** -18) * np.abs(ref) + TINY[dtype]).all()

"""GPU checks of head norms with rotation and of log probabilities against the numpy
oracle (oracle/step.py), within bounds derived from the roundings on the way (stated at
each); indices exactly."""
import numpy as np
import pytest

from oracle import step as S
from tests.test_gpu_serve import EPS, TINY, cumsum, dev, host, say, tdt

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def freqs(n, base=1e4):
    return base ** -(np.arange(n) / max(n, 1))


def random_masks(g, lens, starts, words, p=0.5):
    """Any bits at all, past the request's tokens too."""
    return (g.integers(0, 1 << 63, (starts[-1], words), dtype=np.uint64) * np.uint64(2) + g.integers(0, 2, (starts[-1], words), dtype=np.uint64)
            if p else np.zeros((starts[-1], words), np.uint64))


def masks_dev(m):
    return dev(m.view(np.int64))


def batch_of(lens, starts, max_new=None):
    from paper_2208_01944_amd import palq as P
    i32 = lambda v: dev(np.int32(v))  # noqa: E731
    most = max(b - a for a, b in zip(starts[:-1], starts[1:])) if max_new is None else max_new
    return P.Batch(i32(np.zeros((len(lens), 1))), i32(lens), i32(starts), most, max(max(lens), 0))


def check_rotated(got, x, pos, dtype, **kw):
    """A norm: a lane's 16 squares and up to 4 steps between lanes give the mean 20 roundings, halved by the root; mean,
    root (2 units), two products: 15 half units in all.  Sine and cosine: the angle's conversion and product, 2 half units
    of at most 0.8, and 4 of the sum.  Two products and a sum: 2 more.  Then the result's own."""
    ref, size = S.norm_rotate(x, pos, **kw)
    assert np.array_equal(np.isnan(got), np.isnan(ref.astype(np.float64)))
    ref, size = ref.astype(np.float64), size.astype(np.float64)
    ok = np.isfinite(ref)
    tol = 24 * U * size + EPS[dtype] * 1.01 * np.abs(ref) + TINY[dtype] + 1e-38
    if dtype == "f16":
        ok &= np.abs(ref) < 65000
    bad = np.abs(got - ref)[ok] > tol[ok]
    assert not bad.any(), f"{bad.sum()} of {ok.sum()} off, worst {(np.abs(got - ref)[ok] / tol[ok]).max():.3g} of the bound"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,pairs,interleaved,norm,q_heads,k_heads", [
    (64, 32, False, True, 4, 2), (64, 8, True, True, 17, 3), (64, 16, False, False, 1, 1), (96, 48, False, True, 9, 9), (96, 32, True, True, 7, 1),
    (96, 13, False, True, 5, 2), (96, 13, True, True, 5, 2), (128, 64, False, True, 32, 8), (128, 64, True, False, 8, 8), (128, 1, False, True, 3, 1),
    (128, 0, False, True, 9, 1), (256, 128, False, True, 6, 2), (256, 64, False, True, 5, 0), (256, 127, False, False, 2, 5),
])
def test_norm_rotate(palq, dtype, dim, pairs, interleaved, norm, q_heads, k_heads):
    """Requests of no token, one and many, positions from before the first to far ones."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("norm_rotate", dtype, dim, pairs, interleaved, norm, q_heads, k_heads)
    g = np.random.default_rng(dim + pairs)
    lens, new = [1, 5, 40, 3, 100003, 2 ** 31 - 1, 0], [1, 0, 17, 7, 33, 2, 3]
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], q_heads, dim)) * np.exp(g.standard_normal((starts[-1], q_heads, 1)) * 2), dtype)
    k = dev(g.standard_normal((starts[-1], k_heads, dim)), dtype) if k_heads else None
    qw, kw = (g.standard_normal(dim).astype(np.float32), None) if norm else (None, None)
    f = freqs(pairs)
    rot = P.Rotation(palq, f, interleaved) if pairs else None
    qo, ko = torch.full_like(q, 9), torch.full_like(k, 9) if k_heads else None
    b = batch_of(lens, starts)
    call = lambda x, y: palq.norm_rotate(b, x, y, k, ko, q_weight=None if qw is None else dev(qw), k_weight=kw,  # noqa: E731
                                         eps=1e-5 if norm else None, rotation=rot)
    call(q, qo)
    palq.sync()
    pos = S.positions(lens, starts)
    check_rotated(host(qo), host(q), pos, dtype, freq=f, interleaved=interleaved, weight=qw, eps=1e-5 if norm else None)
    if k_heads:
        check_rotated(host(ko), host(k), pos, dtype, freq=f, interleaved=interleaved, eps=1e-5 if norm else None)
    call(q, q)  # in place
    palq.sync()
    assert torch.equal(q, qo)


def test_norm_rotate_parts_of_a_fused_tensor(palq):
    """Queries and keys within one projection's rows, in place; the values beside them stay."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(3)
    lens, starts, dim = [70, 9], [0, 60, 69], 128
    x = dev(g.standard_normal((69, 7, dim + 6)), "bf16")
    before = x.clone()
    q, k = x[:, 1:5, 2:dim + 2], x[:, 5:6, 3:dim + 3]  # (odd places: no row is aligned to more than an element)
    rot = P.Rotation(palq, freqs(64))
    palq.norm_rotate(batch_of(lens, starts), q, q, k, k, eps=1e-6, rotation=rot)
    palq.sync()
    pos = S.positions(lens, starts)
    for got, was in ((q, before[:, 1:5, 2:dim + 2]), (k, before[:, 5:6, 3:dim + 3])):
        check_rotated(host(got), host(was), pos, "bf16", freq=freqs(64), eps=1e-6)
    q.copy_(before[:, 1:5, 2:dim + 2])
    k.copy_(before[:, 5:6, 3:dim + 3])
    assert torch.equal(x, before)


@pytest.mark.parametrize("words,new", [(1, [5, 0, 64, 1]), (1, [70, 3, 2, 65]), (3, [130, 1, 64, 192]), (16, [3, 200, 0, 7])])
def test_norm_rotate_tree(palq, words, new):
    """Positions from masks of any bits, tokens without a bit among them."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(words)
    lens, starts = [200, 300, 2000, 40], cumsum(new)
    masks = random_masks(g, lens, starts, words)
    q = dev(g.standard_normal((starts[-1], 3, 64)), "f32")
    out = torch.empty_like(q)
    palq.norm_rotate(batch_of(lens, starts), q, out, rotation=P.Rotation(palq, freqs(32)), tree=masks_dev(masks))
    palq.sync()
    check_rotated(host(out), host(q), S.positions(lens, starts, masks), "f32", freq=freqs(32))


def test_norm_rotate_values_at_the_ends(palq):
    """Squares past fp32's range and below it, infinities and NaN: each in its own head."""
    import torch
    g = np.random.default_rng(8)
    x = g.standard_normal((9, 4, 64)).astype(np.float32)
    x[0] *= 1e30
    x[1, 1] *= 3e37
    x[2] *= 1e-30
    x[3, 2] = 0
    x[4, 0, 5] = np.nan
    x[5, 1, 7] = np.inf
    x[6, 3, 60] = -np.inf
    x[7, 2] = np.inf
    for dtype in ("f32", "bf16"):
        q = dev(x, dtype)
        out = torch.empty_like(q)
        palq.norm_rotate(batch_of([9], [0, 9]), q, out, eps=1e-12)
        palq.sync()
        with np.errstate(invalid="ignore"):
            check_rotated(host(out), host(q), np.arange(9), dtype, eps=1e-12)


def test_norm_rotate_rows_left_out(palq):
    """Rows past max_new, before, between and behind the requests stay as they are; wild starts stay inside."""
    import torch
    x = torch.randn(40, 2, 64, device="cuda")
    out = torch.full_like(x, 7.0)
    b = batch_of([50, 60], [3, 20, 33], max_new=10)
    palq.norm_rotate(b, x, out, eps=1e-6)
    palq.sync()
    got = host(out)
    live = np.zeros(40, bool)
    live[3:13] = live[20:30] = True
    assert (got[~live] == 7).all()
    check_rotated(got[live], host(x)[live], np.zeros(20, np.int64), "f32", eps=1e-6)
    for lens, starts in (([9, 9], [-5, 100, 7]), ([1 << 30, -4], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]), ([-2 ** 31, 2 ** 31 - 1], [-2 ** 31, 0, 60])):
        tree = torch.full((40, 2), -1, dtype=torch.int64, device="cuda")
        wild = batch_of(lens, starts, max_new=2 ** 31 - 1)
        palq.norm_rotate(wild, x, torch.empty_like(x), eps=1e-6, tree=tree)
        palq.norm_rotate(wild, x, torch.empty_like(x), eps=1e-6)
    palq.sync()


def test_norm_rotate_many_tokens(palq):
    """Enough tokens that a wave takes all heads of one."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(11)
    lens, starts = [5000, 4000, 9000], [0, 5000, 8999, 9100]
    q, k = dev(g.standard_normal((9100, 11, 64)), "f16"), dev(g.standard_normal((9100, 3, 64)), "f16")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    palq.norm_rotate(batch_of(lens, starts), q, qo, k, ko, eps=1e-6, rotation=P.Rotation(palq, freqs(32)))
    palq.sync()
    pos = S.positions(lens, starts)
    check_rotated(host(qo), host(q), pos, "f16", freq=freqs(32), eps=1e-6)
    check_rotated(host(ko), host(k), pos, "f16", freq=freqs(32), eps=1e-6)


# ------------------------------------------------------------------ log probabilities
def check_scores(x, scale, ids, got, top):
    """t = (largest - x) scale goes into the exponential with 4 half units (difference, product, two of the constant) of
    |t|, and one more for each move of a lane's maximum (by 2^8 at least); the exponential 2 half units; a sum n / 512 + 8
    in a lane, 12 between lanes and 64 between parts.  ln S takes S's relative error and 2 half units of itself, l one
    product and difference more; the entropy the same of sum p t and, through the exponentials, of sum p t^2."""
    out, ent, top_ids, top_out = got
    ro, re, ri, rt, size = S.log_probs(x, scale, ids, top)
    ln_s, a1, a2 = size.T
    es = U * (x.shape[1] / 512 + 90 + 6 * a1)
    for g, r in ((out, ro), (top_out, rt)):
        r = np.where(r < -np.finfo(np.float32).max, -np.inf, r)  # (past fp32's range)
        assert np.array_equal(np.isnan(g), np.isnan(r))
        inf = np.isinf(r)
        assert (g[inf] == r[inf]).all()
        r = np.where(inf, 0, r)
        g = np.where(inf, 0, g)
        tol = es[:, None] + 2 * U * (np.abs(r) + ln_s[:, None]) + 2 * U * ln_s[:, None] + U * np.abs(r)
        ok = ~np.isnan(r)
        assert (np.abs(g - r)[ok] <= tol[ok]).all(), (np.abs(g - r)[ok] / tol[ok]).max()
    if ent is not None:
        assert np.array_equal(np.isnan(ent), np.isnan(re))
        tol = es * (1 + a1) + 6 * U * (a1 + a2) + 4 * U * (ln_s + a1)
        ok = np.isfinite(re)
        assert (np.abs(ent - re)[ok] <= tol[ok]).all(), (np.abs(ent - re)[ok] / tol[ok]).max()
    np.testing.assert_array_equal(top_ids, ri)


def score(palq, x, ids, top, scale=1.0, entropy=True):
    import torch
    rows = x.shape[0]
    i = dev(np.int32(ids))
    out, ent = torch.full(ids.shape, 5.0, device="cuda"), torch.full((rows,), 5.0, device="cuda") if entropy else None
    ti, to = (torch.full((rows, top), 77, dtype=torch.int32, device="cuda"), torch.full((rows, top), 5.0, device="cuda")) if top else (None, None)
    palq.log_probs(x, i, out, entropy=ent, top_ids=ti, top=to, scale=scale)
    palq.sync()
    none = np.zeros((rows, 0))
    return host(out), host(ent) if entropy else None, ti.cpu().numpy() if top else none, host(to) if top else none


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,given,top,pad", [
    (1, 1, 1, 1, 0), (3, 2, 2, 2, 1), (5, 63, 1, 5, 0), (2, 64, 1, 64, 0), (4, 65, 3, 20, 3), (7, 1000, 1, 20, 0), (333, 1000, 1, 5, 1),
    (3, 2047, 1, 7, 0), (2, 2049, 1, 64, 5), (1, 50001, 1, 20, 0), (9, 32000, 4, 64, 0), (2, 131071, 1, 20, 0), (4100, 2500, 1, 20, 3), (4097, 70, 0, 64, 0),
    (6, 5003, 100, 0, 0),
])
def test_log_probs(palq, dtype, rows, vocab, given, top, pad):
    say("log_probs", dtype, rows, vocab, given, top, pad)
    g = np.random.default_rng(rows + vocab)
    x = dev(g.standard_normal((rows, vocab + pad)).astype(np.float32) * 3, dtype)[:, :vocab]
    ids = g.integers(0, vocab, (rows, given))
    check_scores(host(x), 1.25, ids, score(palq, x, ids, top, 1.25), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [100, 6001, 70001])
def test_log_probs_orders_and_ties(palq, dtype, vocab):
    """Equal rows, rising and falling ones, few values, both zeros, a masked tail, one token left, none left."""
    g = np.random.default_rng(vocab)
    x = np.zeros((11, vocab), np.float32)
    x[1] = np.arange(vocab)
    x[2] = -np.arange(vocab)
    x[3] = g.integers(0, 3, vocab)
    x[4] = np.where(g.random(vocab) < 0.5, -0.0, 0.0)
    x[5, vocab // 2:] = -np.inf
    x[6] = -np.inf
    x[6, vocab - 3] = -4
    x[7] = -np.inf
    x[8] = np.float32(-3e38) if dtype == "f32" else -2.0 ** 127
    x[9] = g.standard_normal(vocab)
    x[9, ::7] = -3e38
    x[9, vocab // 3] = 3e38  # one certain token
    x[10] = -np.inf
    x[10, 5:30] = g.standard_normal(25)  # fewer tokens left than asked for
    x = dev(x, dtype)
    ids = np.stack([np.full(11, i) for i in (0, vocab - 1, vocab - 3, vocab // 3, -1, vocab, -2 ** 31)], 1)
    check_scores(host(x), 0.75, ids, score(palq, x, ids, 40, 0.75), 40)


@pytest.mark.parametrize("vocab", [100, 9000])
def test_log_probs_not_finite(palq, vocab):
    """NaN and +inf: their rows, whole, and no others."""
    g = np.random.default_rng(2)
    x = g.standard_normal((6, vocab)).astype(np.float32)
    x[1, 3], x[2, vocab - 1], x[3], x[4, 50:53] = np.nan, np.inf, np.nan, np.inf
    for dtype in ("f32", "f16", "bf16"):
        d = dev(x, dtype)
        ids = np.tile([3, 7], (6, 1))
        got = score(palq, d, ids, 9)
        check_scores(host(d), 1.0, ids, got, 9)
        assert (got[2][1:5] == -1).all() and (got[2][[0, 5]] >= 0).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 1e30])
def test_log_probs_scales(palq, scale):
    g = np.random.default_rng(4)
    x = dev(g.standard_normal((3, 5000)).astype(np.float32) * 5)
    ids = g.integers(0, 5000, (3, 2))
    got, want = score(palq, x, ids, 8, scale), S.log_probs(host(x), scale, ids, 8)
    np.testing.assert_array_equal(got[2], want[2])
    if scale < 100:
        check_scores(host(x), scale, ids, got, 8)
    else:  # all but the largest token past the exponential's range: l itself has 2 half units
        for a, b in ((got[0], want[0]), (got[3], want[3])):
            assert np.allclose(a, b, rtol=3 * U, atol=0)
        assert (got[1] == 0).all()


def test_log_probs_without_parts(palq):
    """Entropy alone, ids as one column, nothing asked for."""
    import torch
    x = torch.randn(5, 300, device="cuda")
    want = S.log_probs(host(x), 1.0, np.tile([[7]], (5, 1)), 0)
    ent = torch.empty(5, device="cuda")
    palq.log_probs(x, None, None, entropy=ent)
    one = torch.empty(5, device="cuda")
    palq.log_probs(x, torch.full((5,), 7, dtype=torch.int32, device="cuda"), one)
    palq.log_probs(x, None, None)
    palq.sync()
    assert np.abs(host(ent) - want[1]).max() < 1e-5 and np.abs(host(one) - want[0][:, 0]).max() < 1e-5


@pytest.mark.parametrize("dtype,rows,vocab,top", [("bf16", 600, 9001, 20), ("f32", 600, 4099, 64), ("f16", 70, 140001, 64), ("f32", 2, 200003, 33),
                                                  ("bf16", 1, 262144, 64), ("bf16", 4099, 6000, 64), ("f32", 4099, 4097, 1)])
def test_log_probs_every_kernel(palq, dtype, rows, vocab, top):
    """A wave a row, four, and parts of rows that are joined; long and short steps."""
    say("log_probs kernels", dtype, rows, vocab, top)
    g = np.random.default_rng(vocab)
    x = dev(g.standard_normal((rows, vocab)).astype(np.float32) * 3, dtype)
    x[:, vocab - vocab // 40:] = -np.inf
    some = np.unique(np.r_[0, rows - 1, g.integers(0, rows, 40)])
    ids = g.integers(0, vocab, (rows, 1))
    got = score(palq, x, ids, top, 0.8)
    check_scores(host(x[some]), 0.8, ids[some], tuple(t[some] for t in got), top)


@pytest.mark.parametrize("rows", [3, 700, 4100])
def test_log_probs_values_in_masses(palq, rows):
    """Rows of one value, of two, and rising ones, by every kernel: the first indices of equal values."""
    x = np.zeros((rows, 5000), np.float32)
    x[1, ::3] = 1
    x[2] = np.arange(5000) // 7
    d = dev(x, "bf16")
    got = score(palq, d, np.zeros((rows, 1), np.int64), 64)
    some = [0, 1, 2, rows - 1]
    check_scores(host(d[some]), 1.0, np.zeros((4, 1), np.int64), tuple(t[some] for t in got), 64)

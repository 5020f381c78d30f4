"""GPU checks of the 8-bit transformer operators against the numpy oracle
(oracle/serve.py): codes, scales and read values exactly, floating results
within bounds derived from the roundings on the way (stated at each)."""
import numpy as np
import pytest

from oracle import serve as S

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half a unit in the last place, relative
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}               # half the distance of subnormal values


def say(*a):
    print(*a, flush=True)


def tdt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(tdt(dtype))).cuda()


def host(t):
    return t.float().cpu().numpy()


# ------------------------------------------------------------------ token quantiser
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 16, 0), (3, 17, 3), (5, 64, 0), (2, 1000, 24), (7, 4096, 0), (4, 4099, 5),
                                           (3, 9000, 0), (600, 130, 6), (515, 64, 0)])
def test_quantize_rows(palq, dtype, rows, cols, pad):
    import torch
    say("quantize_rows", dtype, rows, cols, pad)
    g = np.random.default_rng(rows * 10007 + cols)
    x = dev(g.standard_normal((rows, cols + pad)) * np.exp(g.standard_normal((rows, 1)) * 3), dtype)
    x[0, :cols // 2] = 0
    if rows > 2:
        x[1] = 0
        x[2, cols // 3] = float("nan") if rows % 2 else float("inf")
    x = x[:, :cols]
    codes = torch.full((rows, cols + pad), 99, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, device="cuda")
    palq.quantize_rows(x, codes[:, :cols], scales)
    palq.sync()
    rc, rs = S.quantize_rows(host(x))
    np.testing.assert_array_equal(scales.cpu().numpy(), rs)
    np.testing.assert_array_equal(codes[:, :cols].cpu().numpy(), rc)
    assert (codes[:, cols:].cpu().numpy() == 99).all()


# ------------------------------------------------------------------ linear
def linear_case(g, rows, n_in, n_out, x_type, bias):
    w = g.integers(-127, 128, (n_out, n_in)).astype(np.int8)
    w[0] = -128
    ws = np.exp(g.standard_normal(n_out)).astype(np.float32) / 100
    b = g.standard_normal(n_out).astype(np.float32) if bias else None
    if x_type == "i8":
        x = g.integers(-128, 128, (rows, n_in)).astype(np.int8)
        x[0] = -128
        return w, ws, b, x, np.exp(g.standard_normal(rows)).astype(np.float32)
    return w, ws, b, g.standard_normal((rows, n_in)) * np.exp(g.standard_normal((rows, 1))), None


def check_linear(got, q, s, w, ws, b, y_type):
    """The int32 sum is exact; its conversion, two products and the bias round once each in fp32, the result once more."""
    ref = S.linear(q, s, w, ws, b)
    t = np.abs(S.linear(q, s, w, ws))
    bias = 0 if b is None else np.abs(b)
    tol = 5 * 2.0 ** -24 * (t + bias) + EPS[y_type] * 1.01 * np.abs(ref) + TINY[y_type]
    if y_type == "f16":  # past its range: inf
        over = np.abs(ref) >= 65520
        assert (got[over] == np.copysign(np.inf, ref[over])).all()
        got, ref, tol = got[~over], ref[~over], tol[~over]
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"{(err > tol).sum()} of {err.size} off, worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of the bound"


@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f16"), ("i8", "bf16"), ("f32", "f32"), ("i8", "f32")])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1), (1, 64, 16), (1, 4096, 256), (2, 100, 33), (15, 129, 17), (16, 256, 64),
                                             (17, 300, 100), (33, 127, 130), (50, 640, 257), (64, 192, 320), (65, 1000, 1000),
                                             (129, 65, 255), (257, 384, 513), (300, 2047, 258), (520, 130, 1030), (8, 8192, 40), (9, 8192, 40),
                                             (3, 5000, 20), (1, 70000, 18), (200, 1500, 700), (1100, 260, 300)])
def test_linear(palq, x_type, y_type, rows, n_in, n_out):
    import torch
    from paper_2208_01944_amd import palq as P
    say("linear", x_type, y_type, rows, n_in, n_out)
    g = np.random.default_rng(rows * 31 + n_in * 7 + n_out)
    bias = (rows + n_out) % 2 == 0
    w, ws, b, x, s = linear_case(g, rows, n_in, n_out, x_type, bias)
    xt = dev(x, x_type)
    st = None if s is None else dev(s)
    lin = P.Linear(palq, dev(w), dev(ws), None if b is None else dev(b), max_rows=rows)
    y = torch.full((rows, n_out + 3), 7.0, dtype=tdt(y_type), device="cuda")  # odd rows, untouched margin
    lin.run(xt, y[:, :n_out], x_scale=st)
    y2 = torch.empty(rows, n_out, dtype=tdt(y_type), device="cuda")
    lin.run(xt, y2, x_scale=st)
    palq.sync()
    q, s = (x, s) if x_type == "i8" else S.quantize_rows(host(xt))
    check_linear(host(y[:, :n_out]), q, s, w, ws, b, y_type)
    assert torch.equal(y[:, :n_out], y2)
    assert (host(y[:, n_out:]) == 7).all()


@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("i8", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("rows,n_in,n_out,kernel", [(1, 200, 50, "one"), (1, 17000, 50, "few"), (15, 700, 90, "few"), (40, 700, 90, "few"),
                                                    (70, 130, 8200, "tile"), (70, 1100, 8195, "tile"), (1100, 130, 3700, "tile"),
                                                    (1090, 900, 3701, "tile"), (2100, 200, 3900, "tile"), (2051, 650, 3899, "tile"),
                                                    (3300, 64, 3900, "tile"), (3329, 450, 3903, "tile")])
def test_linear_every_kernel(palq, x_type, y_type, rows, n_in, n_out, kernel):
    """Both sides of every size rule: one row, 16 and 32 rows of the few-row kernel, tiles of 64, 128 (two builds) and 256, with
    k of one stage and of several, ends inside tiles."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("linear", x_type, y_type, rows, n_in, n_out, kernel)
    g = np.random.default_rng(rows + n_in)
    w, ws, b, x, s = linear_case(g, rows, n_in, n_out, x_type, True)
    xt = dev(x, x_type)
    lin = P.Linear(palq, dev(w), dev(ws), dev(b), max_rows=rows)
    assert lin.kernels(rows) == f"linear_{kernel}_kernel"
    y = torch.empty(rows, n_out, dtype=tdt(y_type), device="cuda")
    lin.run(xt, y, x_scale=None if s is None else dev(s))
    palq.sync()
    q, s = (x, s) if x_type == "i8" else S.quantize_rows(host(xt))
    check_linear(host(y), q, s, w, ws, b, y_type)


def test_linear_strided_operands(palq):
    """Weights and activations as column slices of wider tensors, at odd offsets; rows and outputs in strided buffers."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(5)
    for rows, n_in, n_out in ((9, 130, 40), (300, 130, 300)):
        w, ws, b, x, _ = linear_case(g, rows, n_in, n_out, "bf16", True)
        wide = dev(np.concatenate([np.zeros((n_out, 3), np.int8), w, np.ones((n_out, 4), np.int8)], 1))
        xw = dev(np.concatenate([np.zeros((rows, 5)), x, np.full((rows, 2), np.nan)], 1), "bf16")
        lin = P.Linear(palq, wide[:, 3:3 + n_in], dev(ws), dev(b), max_rows=rows)
        y = torch.empty(rows, n_out + 9, dtype=torch.float32, device="cuda")
        lin.run(xw[:, 5:5 + n_in], y[:, 1:1 + n_out])
        palq.sync()
        q, s = S.quantize_rows(host(xw[:, 5:5 + n_in]))
        check_linear(host(y[:, 1:1 + n_out]), q, s, w, ws, b, "f32")


def test_linear_not_finite_rows(palq):
    """A row with inf or NaN gives NaN in that row and nowhere else; a row of zeros gives the bias."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(6)
    for rows in (4, 70, 300):
        w, ws, b, x, _ = linear_case(g, rows, 96, 80, "f32", True)
        x[0, 3], x[2, 95], x[1] = np.inf, np.nan, 0
        lin = P.Linear(palq, dev(w), dev(ws), dev(b), max_rows=rows)
        y = torch.empty(rows, 80, device="cuda")
        lin.run(dev(x, "f32"), y)
        palq.sync()
        y = host(y)
        assert np.isnan(y[[0, 2]]).all() and np.isfinite(np.delete(y, [0, 2], 0)).all()
        np.testing.assert_array_equal(y[1], b)


def test_linear_largest_sums(palq):
    """Sums next to 2^31: n_in = 2^17 - 1 of products 2^14."""
    import torch
    from paper_2208_01944_amd import palq as P
    n_in = (1 << 17) - 1
    w = torch.full((3, n_in), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(3, device="cuda")
    for rows in (2, 70):
        x = torch.full((rows, n_in), -128, dtype=torch.int8, device="cuda")
        lin = P.Linear(palq, w, one, max_rows=rows)
        y = torch.empty(rows, 3, device="cuda")
        lin.run(x, y, x_scale=torch.ones(rows, device="cuda"))
        palq.sync()
        np.testing.assert_array_equal(y.cpu().numpy(), np.float32([[n_in * 16384, -n_in * 16256, n_in * 16384]] * rows))


# ------------------------------------------------------------------ cache
def paged(g, lens, page, spare=2, width=None):
    """A scattered page table (unused entries out of range) and the pool's size."""
    per = [-(-n // page) for n in lens]
    pages = sum(per) + spare
    order = g.permutation(pages)
    table = np.full((len(lens), width or max(1, max(per, default=1))), -1, np.int32)
    at = 0
    for r, n in enumerate(per):
        table[r, :n] = order[at:at + n]
        at += n
    return table, pages


class Pair:
    """A cache on the GPU and the oracle's."""

    def __init__(self, P, pages, heads, page, dim):
        self.P, self.gpu, self.ref = P, P.Cache.empty(pages, heads, page, dim), S.Cache(pages, heads, page, dim)

    def batch(self, table, lens, starts, max_new=None, max_len=None):
        n = max((starts[i + 1] - starts[i] for i in range(len(lens))), default=0)
        return self.P.Batch(dev(table), dev(np.int32(lens)), dev(np.int32(starts)), n if max_new is None else max_new,
                            max(lens, default=0) if max_len is None else max_len)

    def fill(self, g, table, used, spread=0.5):
        """Random codes and scales in every block (as appends would leave them)."""
        import torch
        r = self.ref
        r.k[:] = np.clip(np.rint(g.standard_normal(r.k.shape) * 32), -127, 127)
        r.v[:] = np.clip(np.rint(g.standard_normal(r.v.shape) * 32), -127, 127)
        r.ks[:] = np.exp(g.standard_normal(r.ks.shape) * spread) / 32
        r.vs[:] = np.exp(g.standard_normal(r.vs.shape) * spread) / 32
        self.upload()

    def upload(self):
        import torch
        r, c = self.ref, self.gpu
        c.k.copy_(torch.from_numpy(r.k))
        c.v.copy_(torch.from_numpy(np.ascontiguousarray(r.v.transpose(0, 1, 3, 2))))
        c.k_scale.copy_(torch.from_numpy(r.ks))
        c.v_scale.copy_(torch.from_numpy(r.vs))

    def check(self, table, lens):
        """Scales of every block in use and codes of every token."""
        r, c = self.ref, self.gpu
        k, v = c.k.cpu().numpy(), c.v.cpu().numpy().transpose(0, 1, 3, 2)
        ks, vs = c.k_scale.cpu().numpy(), c.v_scale.cpu().numpy()
        for i, ln in enumerate(lens):
            for b in range(-(-ln // r.page)):
                p, n = table[i][b], min(r.page, ln - b * r.page)
                if not 0 <= p < len(k):
                    continue
                np.testing.assert_array_equal(ks[p], r.ks[p])
                np.testing.assert_array_equal(vs[p], r.vs[p])
                np.testing.assert_array_equal(k[p, :, :n], r.k[p, :, :n])
                np.testing.assert_array_equal(v[p, :, :n], r.v[p, :, :n])


def cumsum(n):
    return [0] + np.cumsum(n).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("page,dim,heads", [(16, 64, 2), (32, 96, 1), (64, 128, 3), (128, 256, 2), (64, 64, 1), (16, 256, 1)])
def test_cache_append_in_steps(palq, dtype, page, dim, heads):
    """Ragged requests grow in several appends (from nothing, by nothing, by one, across pages), every
    block's codes and scales equal to the oracle's after each; values of growing size, so that scales grow."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("append", dtype, page, dim, heads)
    g = np.random.default_rng(page + dim)
    steps = [[0, 1, page - 1, page, page + 1, 3], [1, 0, 1, 1, 1, 5], [1, 1, 1, 0, 2 * page + 3, 7], [2, page, 1, 1, 1, 1]]
    final = np.sum(steps, 0)
    table, pages = paged(g, final.tolist(), page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, final)  # what earlier owners left
    lens = np.zeros(6, int)
    for i, new in enumerate(steps):
        lens = lens + new
        starts = cumsum(new)
        k = dev(g.standard_normal((starts[-1], heads, dim)) * np.exp(g.standard_normal((starts[-1], heads, 1)) + i), dtype)
        v = dev(g.standard_normal((starts[-1], heads, dim)) * (0.5 + i % 2), dtype)
        pair.ref.append(table, lens.tolist(), starts, host(k), host(v))
        b = pair.batch(table, lens.tolist(), starts)
        palq.cache_append(pair.gpu, k, v, b)
        palq.sync()
        pair.check(table, lens.tolist())
        palq.cache_append(pair.gpu, k, v, b)  # again: no change
        palq.sync()
        pair.check(table, lens.tolist())
    back = np.minimum(lens, [1, 2, page, page + 1, 3 * page, 5])
    starts = cumsum(back)
    for out in ("f32", dtype):
        k = torch.zeros(starts[-1], heads, dim, dtype=tdt(out), device="cuda")
        v = torch.zeros_like(k)
        palq.cache_read(pair.gpu, k, v, pair.batch(table, lens.tolist(), starts))
        palq.sync()
        rk, rv = pair.ref.read(table, lens.tolist(), starts)
        np.testing.assert_array_equal(host(k), host(dev(rk, out)))
        np.testing.assert_array_equal(host(v), host(dev(rv, out)))


def test_cache_append_strided(palq):
    """k and v as parts of one fused projection's rows, heads in the middle, at an odd element offset; reads into such parts."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(11)
    heads, dim, page, new, lens = 2, 64, 16, [5, 17, 1], [9, 17, 33]
    table, pages = paged(g, lens, page)
    starts = cumsum(new)
    for off in (0, 3):
        pair = Pair(P, pages, heads, page, dim)
        pair.fill(g, table, lens)
        row = 3 * heads * dim + 8
        qkv = dev(g.standard_normal((starts[-1], row + off)), "bf16")
        k = qkv[:, off:off + heads * dim].unflatten(1, (heads, dim))
        v = qkv[:, off + heads * dim:off + 3 * heads * dim].unflatten(1, (heads, 2 * dim))[:, :, dim:]
        pair.ref.append(table, lens, starts, host(k), host(v))
        palq.cache_append(pair.gpu, k, v, pair.batch(table, lens, starts))
        palq.sync()
        pair.check(table, lens)
        out = torch.zeros(starts[-1], row + off, device="cuda")
        ok = out[:, off:off + heads * dim].unflatten(1, (heads, dim))
        ov = out[:, off + heads * dim:off + 3 * heads * dim].unflatten(1, (heads, 2 * dim))[:, :, dim:]
        palq.cache_read(pair.gpu, ok, ov, pair.batch(table, lens, starts))
        palq.sync()
        rk, rv = pair.ref.read(table, lens, starts)
        np.testing.assert_array_equal(host(ok), rk)
        np.testing.assert_array_equal(host(ov), rv)


def test_cache_not_finite(palq):
    """A value that is not finite makes its block's scale NaN (its head's alone) until the page starts afresh."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(12)
    page, heads, dim = 16, 2, 64
    table = np.int32([[0, 1], [2, 3]])
    pair = Pair(P, 4, heads, page, dim)
    lens = [3, 20]
    for new, bad in (([3, 20], (1, 0, 5, np.inf)), ([1, 1], None), ([2, 1], (0, 1, 0, np.nan))):
        starts = cumsum(new)
        lens = [min(a + b, 32) for a, b in zip(lens, new)] if bad is None or bad[3] != np.inf else lens
        k, v = (g.standard_normal((starts[-1], heads, dim)).astype(np.float32) for _ in range(2))
        if bad:
            k[starts[bad[0]], bad[1], bad[2]] = bad[3]
            v[starts[bad[0]], 1 - bad[1], bad[2]] = -bad[3]
        pair.ref.append(table, lens, starts, k, v)
        palq.cache_append(pair.gpu, dev(k), dev(v), pair.batch(table, lens, starts))
        palq.sync()
        pair.check(table, lens)
    assert np.isnan(pair.ref.ks).sum() == 2 and np.isnan(pair.ref.vs).sum() == 2


def test_cache_bad_tables_stay_inside(palq):
    """Page numbers out of range, lengths past the table, row starts that run backwards: nothing outside
    the tensors is touched, and what is in range is right."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(13)
    page, heads, dim = 16, 1, 64
    table = np.int32([[0, 7, 2], [1, -5, 3]])
    pair = Pair(P, 4, heads, page, dim)
    pair.fill(g, table, None)
    lens, starts = [40, 20], [0, 40, 60]
    x = g.standard_normal((60, heads, dim)).astype(np.float32)
    pair.ref.append(table, lens, starts, x, x)
    palq.cache_append(pair.gpu, dev(x), dev(x), pair.batch(table, lens, starts))
    palq.sync()
    pair.check(table, lens)
    ok, ov = torch.full((60, heads, dim), 5.0, device="cuda"), torch.full((60, heads, dim), 5.0, device="cuda")
    palq.cache_read(pair.gpu, ok, ov, pair.batch(table, lens, starts))
    palq.sync()
    rk, rv = pair.ref.read(table, lens, starts)
    np.testing.assert_array_equal(host(ok), rk)
    np.testing.assert_array_equal(host(ov), rv)
    # lengths past the table (and starts running backwards): no fault, the pool's other pages stay
    wild = pair.batch(table, [1000, 1 << 30], [0, 70, -3], max_new=60, max_len=1 << 30)
    before = pair.gpu.k_scale.clone()
    palq.cache_read(pair.gpu, ok, ov, wild)
    q = torch.zeros(60, 1, dim, dtype=torch.bfloat16, device="cuda")
    palq.attention(pair.gpu, q, torch.empty_like(q), wild, 1.0)
    palq.sync()
    assert torch.equal(before, pair.gpu.k_scale)


# ------------------------------------------------------------------ attention
def check_attend(pair, got, table, lens, starts, q, scale, dtype, **kw):
    """Bound, for each output: scores carry the fp32 rounding of dim products and of the exponent's argument
    (log2 of a weight, below 2^8 in size), a weight two such errors and its own rounding to fp16 (2^-11 relative
    or half a subnormal step of the largest weight), the result one rounding to its type."""
    ref, mass, reach, seen = pair.ref.attend(table, lens, starts, q, scale, **kw)
    dim = q.shape[2]
    es = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -15
    tol = mass * (2.0 ** -11 + 2 * es)[..., None] + (seen * 2.0 ** -25 * 127 * float(pair.ref.vs[np.isfinite(pair.ref.vs)].max()))[..., None]
    tol = tol + EPS[dtype] * (np.abs(ref) + tol) + TINY[dtype]
    err = np.abs(got - ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaN in the wrong places"
    bad = err > tol
    assert not bad.any(), f"{bad.sum()} of {err.size} off, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.3g} of the bound"
    assert (got[seen == 0] == 0).all()


def attend_case(P, ctx, seed, dtype, page, dim, heads, group, lens, new, causal=True, window=0, spread=0.5, q_mul=1.5, max_len=None,
                missing=()):
    import torch
    g = np.random.default_rng(seed)
    table, pages = paged(g, lens, page)
    for r, block in missing:
        table[r, block] = -1 if r % 2 else pages
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens, spread)
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], heads * group, dim)) * q_mul, dtype)
    out = torch.full_like(q, 3.0)
    b = pair.batch(table, lens, starts, max_len=max_len)
    ctx.attention(pair.gpu, q, out, b, dim ** -0.5, causal=causal, window=window)
    ctx.sync()
    check_attend(pair, host(out), table, lens, starts, host(q), dim ** -0.5, dtype, causal=causal, window=window)
    again = torch.empty_like(q)
    ctx.attention(pair.gpu, q, again, b, dim ** -0.5, causal=causal, window=window)
    ctx.sync()
    assert torch.equal(out, again)
    return pair, table, starts, q, out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,dim,heads,group", [(16, 64, 2, 1), (32, 96, 1, 4), (64, 128, 2, 4), (128, 256, 1, 3), (64, 64, 1, 7),
                                                  (16, 128, 1, 16), (32, 256, 2, 17)])
def test_attention_single_tokens(palq, dtype, page, dim, heads, group):
    """One new token of each request, lengths from none to several splits, empty requests among them."""
    from paper_2208_01944_amd import palq as P
    say("attention single", dtype, page, dim, heads, group)
    attend_case(P, palq, page + dim + group, dtype, page, dim, heads, group,
                [1, 0, 2, 15, 16, 17, 63, 64, 65, 130, 257, 700], [1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,dim,heads,group,lens,new,causal,window", [
    (64, 128, 1, 4, [5, 33, 100], [5, 33, 70], True, 0),        # whole prompts, and one behind cached tokens
    (16, 64, 2, 1, [70, 1, 129], [70, 1, 64], True, 0),
    (32, 96, 1, 2, [90, 40], [90, 13], True, 7),                 # windows shorter than a tile
    (64, 128, 1, 1, [200, 150], [130, 150], True, 64),
    (128, 256, 1, 2, [140, 9], [40, 9], True, 0),
    (64, 64, 1, 3, [3, 10], [9, 20], True, 0),                   # more rows than tokens: the first rows see nothing
    (64, 64, 1, 3, [3, 0, 50], [9, 20, 1], False, 0),            # cross attention, one encoder without tokens
    (16, 128, 2, 2, [150, 77], [31, 66], False, 0),
    (32, 64, 1, 1, [1, 300], [300, 5], False, 0),
    (32, 96, 1, 5, [64, 257], [40, 100], False, 0),
    (64, 256, 1, 1, [130], [129], True, 100),
])
def test_attention_many_rows(palq, dtype, page, dim, heads, group, lens, new, causal, window):
    from paper_2208_01944_amd import palq as P
    say("attention rows", dtype, page, dim, heads, group, lens, new, causal, window)
    attend_case(P, palq, page * 3 + dim + group, dtype, page, dim, heads, group, lens, new, causal, window)


# enough rows for the 128-row kernel: more than 768 blocks of 32 rows (16 for heads of 256)
@pytest.mark.parametrize("dtype,page,dim,heads,group,lens,new,causal,window,max_len,missing", [
    ("bf16", 64, 128, 16, 2, [128, 150, 131, 300, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], True, 0, None, ()),
    ("f16", 16, 64, 16, 2, [128, 150, 131, 300, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], True, 50, None, ()),
    ("bf16", 32, 96, 16, 2, [70, 150, 0, 1, 129, 64, 191], [131, 40, 5, 100, 1, 64, 120], False, 0, None, ()),
    ("f16", 128, 256, 8, 1, [100, 150, 131, 20, 129, 64, 65, 191], [200, 40, 131, 70, 1, 64, 0, 120], True, 0, None, ()),
    ("bf16", 64, 64, 16, 3, [160, 100, 130, 61, 200], [100, 100, 110, 100, 90], True, 0, 5000, ()),             # split, a part empty
    ("f16", 16, 128, 16, 3, [1300, 100, 130, 700, 200], [60, 100, 20, 31, 100], True, 700, 4000, ()),           # split, windows
    ("bf16", 16, 128, 16, 2, [128, 150, 131, 170, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], True, 0, None, ((0, 0), (1, 3), (5, 12))),
])
def test_attention_tile_kernel(palq, dtype, page, dim, heads, group, lens, new, causal, window, max_len, missing):
    from paper_2208_01944_amd import palq as P
    say("attention tiles", dtype, page, dim, heads, group, lens, new, causal, window, max_len)
    assert -(-max(new) * group // (16 if dim == 256 else 32)) * heads * len(lens) > 768
    attend_case(P, palq, page + dim, dtype, page, dim, heads, group, lens, new, causal, window, max_len=max_len, missing=missing)


def test_attention_tile_kernel_not_finite(palq):
    """As test_attention_not_finite, on the 128-row kernel, with far scales and a negative score scale."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(64)
    page, dim, heads, lens, new = 16, 64, 16, [150, 128, 131, 100, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120]
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens, 4.0)
    spare = sorted(set(range(pages)) - set(table.ravel().tolist()))
    pair.ref.ks[spare], pair.ref.vs[spare] = np.nan, np.inf
    pair.ref.ks[table[0][9], 0] = np.nan   # tokens 144 on of request 0, head 0
    pair.ref.vs[table[1][6], 1] = np.nan   # tokens 96 on of request 1, head 1
    pair.upload()
    starts = cumsum(new)
    q = g.standard_normal((starts[-1], 2 * heads, dim)).astype(np.float32)
    q[0, 0, 5], q[starts[1], 5, 3], q[starts[2], 7, 4] = np.nan, np.inf, -np.inf
    qt = dev(q, "bf16")
    out = torch.empty_like(qt)
    for scale in (0.125, -0.2):
        palq.attention(pair.gpu, qt, out, pair.batch(table, lens, starts), scale)
        palq.sync()
        with np.errstate(invalid="ignore"):
            check_attend(pair, host(out), table, lens, starts, host(qt), scale, "bf16")
        assert np.isnan(host(out)).any() and np.isfinite(host(out)).any()


@pytest.mark.parametrize("rows", [1, 5, 20, 90])
def test_attention_long(palq, rows):
    """Thousands of tokens in many splits, with a window and without, one head."""
    from paper_2208_01944_amd import palq as P
    say("attention long", rows)
    for window in (0, 1000):
        attend_case(P, palq, rows, "bf16", 64, 128, 1, 2, [5000 - rows], [rows], True, window)


def test_attention_far_scales(palq):
    """Blocks whose value scales lie many powers of two apart, sharp and flat softmaxes, large and tiny queries."""
    from paper_2208_01944_amd import palq as P
    for seed, (spread, mul) in enumerate([(8.0, 0.001), (4.0, 1.0), (0.5, 40.0), (0.1, 1e-30), (0.5, 0.0)]):
        for new in ([1, 1], [40, 3]):
            attend_case(P, palq, 50 + seed, "bf16", 16, 64, 1, 2, [130, 47], new, True, 0, spread, mul)


def test_attention_not_finite(palq):
    """Rows of q that are not finite give NaN, alone; a block with a NaN scale gives NaN to the rows that see it, alone;
    codes and scales in masked places count for nothing."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(60)
    for new in ([3, 2], [40, 33]):
        page, dim, lens = 16, 64, [50, 40]
        table, pages = paged(g, lens, page)
        pair = Pair(P, pages, 2, page, dim)
        pair.fill(g, table, lens)
        spare = sorted(set(range(pages)) - set(table.ravel().tolist()))
        pair.ref.ks[spare], pair.ref.vs[spare] = np.nan, np.inf
        pair.ref.ks[table[0][3], 0] = np.nan    # tokens 48, 49 of request 0, head 0: its last rows see them
        pair.ref.vs[table[1][2], 1] = np.nan    # request 1, head 1, tokens 32 to 39
        pair.upload()
        starts = cumsum(new)
        q = g.standard_normal((starts[-1], 2, dim)).astype(np.float32)
        q[0, 0, 5], q[starts[1], 0, 3], q[starts[1], 0, 4] = np.nan, np.inf, -np.inf
        qt = dev(q, "bf16")
        out = torch.empty_like(qt)
        palq.attention(pair.gpu, qt, out, pair.batch(table, lens, starts), 0.125)
        palq.sync()
        with np.errstate(invalid="ignore"):
            check_attend(pair, host(out), table, lens, starts, host(qt), 0.125, "bf16")
        assert np.isnan(host(out)).any() and np.isfinite(host(out)).any()


@pytest.mark.parametrize("scale", [0.125, -0.125, 0.0])
@pytest.mark.parametrize("dim,group,new", [(64, 1, [2, 17, 20]), (64, 3, [1, 1, 1]), (96, 2, [3, 1, 9]), (128, 4, [1, 1, 3]),
                                           (128, 8, [3, 4, 4]), (256, 2, [1, 7, 2])])
def test_attention_whole_tiles(palq, dim, group, new, scale):
    """Few rows over several tiles that all of them see, between tiles that some of them see: scales of either sign and
    none, a key and a value block with a NaN scale in such a tile."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("attention whole tiles", dim, group, scale)
    g = np.random.default_rng(65 + dim + group)
    page, lens = 16, [650, 400, 129]
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, 2, page, dim)
    pair.fill(g, table, lens)
    pair.ref.ks[table[1][9], 0] = np.nan   # tokens 144 on of request 1, head 0
    pair.ref.vs[table[2][5], 1] = np.nan   # tokens 80 on of request 2, head 1
    pair.upload()
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], 2 * group, dim)) * 1.5, "f16")
    out = torch.empty_like(q)
    for kw in ({"causal": True}, {"causal": True, "window": 200}, {"causal": False}):
        palq.attention(pair.gpu, q, out, pair.batch(table, lens, starts), scale, **kw)
        palq.sync()
        with np.errstate(invalid="ignore"):
            check_attend(pair, host(out), table, lens, starts, host(q), scale, "f16", **kw)
        assert np.isfinite(host(out)).any()


def test_attention_strided(palq):
    """q inside a fused row, out with its heads apart, odd element offsets."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(61)
    page, dim, heads, group = 32, 64, 2, 2
    for new, off in (([1, 1], 0), ([1, 2], 3), ([40, 30], 8), ([40, 30], 1)):
        lens = [70, 45]
        table, pages = paged(g, lens, page)
        pair = Pair(P, pages, heads, page, dim)
        pair.fill(g, table, lens)
        starts = cumsum(new)
        hq = heads * group
        q = dev(g.standard_normal((starts[-1], hq * dim + 40)), "f16")[:, off:off + hq * dim].unflatten(1, (hq, dim))
        buf = torch.full((starts[-1], hq, dim + off + 4), 9.0, dtype=torch.float16, device="cuda")
        out = buf[:, :, off:off + dim]
        palq.attention(pair.gpu, q, out, pair.batch(table, lens, starts), 0.125)
        palq.sync()
        check_attend(pair, host(out), table, lens, starts, host(q), 0.125, "f16")
        assert (host(buf[:, :, :off]) == 9).all() and (host(buf[:, :, off + dim:]) == 9).all()


def test_attention_pages_missing(palq):
    """Tokens on page numbers out of range are left out."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(62)
    lens, new = [100, 60], [2, 60]
    table, pages = paged(g, lens, 16)
    table[0, 2], table[1, 0], table[1, 3] = -1, pages, 1 << 30
    pair = Pair(P, pages, 1, 16, 64)
    pair.fill(g, table, lens)
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], 2, 64)), "bf16")
    out = torch.empty_like(q)
    palq.attention(pair.gpu, q, out, pair.batch(table, lens, starts), 0.125)
    palq.sync()
    check_attend(pair, host(out), table, lens, starts, host(q), 0.125, "bf16")


def test_large_cache_offsets(palq):
    """Pages past 2^31 bytes of k and v: append, read, attend."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(63)
    page, dim, heads = 64, 128, 1
    pages = (1 << 31) // (page * dim) + 40
    cache = P.Cache(torch.empty(pages, heads, page, dim, dtype=torch.int8, device="cuda"),
                    torch.empty(pages, heads, dim, page, dtype=torch.int8, device="cuda"),
                    torch.ones(pages, heads, device="cuda"), torch.ones(pages, heads, device="cuda"))
    real = np.int32([[pages - 1, pages - 3, 0], [pages - 2, 1, pages - 30]])
    small, lens, new = np.int32([[0, 1, 2], [3, 4, 5]]), [150, 129], [150, 129]
    pair = Pair(P, 6, heads, page, dim)
    starts = cumsum(new)
    k, v = (g.standard_normal((starts[-1], heads, dim)).astype(np.float32) for _ in range(2))
    pair.ref.append(small, lens, starts, k, v)
    b = P.Batch(dev(real), dev(np.int32(lens)), dev(np.int32(starts)), 150, 150)
    palq.cache_append(cache, dev(k), dev(v), b)
    ok, ov = torch.empty(starts[-1], heads, dim, device="cuda"), torch.empty(starts[-1], heads, dim, device="cuda")
    palq.cache_read(cache, ok, ov, b)
    q = dev(g.standard_normal((starts[-1], 2, dim)), "bf16")
    out = torch.empty_like(q)
    palq.attention(cache, q, out, b, 0.09)
    palq.sync()
    rk, rv = pair.ref.read(small, lens, starts)
    np.testing.assert_array_equal(host(ok), rk)
    np.testing.assert_array_equal(host(ov), rv)
    check_attend(pair, host(out), small, lens, starts, host(q), 0.09, "bf16")


# ------------------------------------------------------------------ streams and graphs
def test_serve_step_in_a_graph(palq):
    """Product, append and attention of one step captured on another stream and replayed with new inputs, with other
    work between the replays; every replay equals the eager calls."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(70)
    side = torch.cuda.Stream()
    ctx = P.Context(0, stream=side.cuda_stream)
    heads, dim, page, lens, new = 2, 64, 16, [40, 700], [1, 1]
    table, pages = paged(g, lens, page)
    starts = cumsum(new)
    n = 3 * heads * dim
    w = dev(g.integers(-127, 128, (n, 96)).astype(np.int8))
    lin = P.Linear(ctx, w, torch.full((n,), 1e-3, device="cuda"), max_rows=2)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens)
    start = [t.clone() for t in (pair.gpu.k, pair.gpu.v, pair.gpu.k_scale, pair.gpu.v_scale)]
    b = pair.batch(table, lens, starts)
    x = torch.empty(2, 96, dtype=torch.bfloat16, device="cuda")
    qkv = torch.empty(2, n, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(2, heads, dim, dtype=torch.bfloat16, device="cuda")

    def step():
        lin.run(x, qkv)
        q, k, v = (t.unflatten(1, (heads, dim)) for t in qkv.split(heads * dim, 1))
        ctx.cache_append(pair.gpu, k, v, b)
        ctx.attention(pair.gpu, q, out, b, 0.125)

    def reset():
        for t, s in zip((pair.gpu.k, pair.gpu.v, pair.gpu.k_scale, pair.gpu.v_scale), start):
            t.copy_(s)

    xs = [dev(g.standard_normal((2, 96)), "bf16") for _ in range(4)]
    want = []
    for xi in xs:
        reset()
        x.copy_(xi)
        torch.cuda.synchronize()
        step()
        ctx.sync()
        want.append((out.clone(), pair.gpu.k.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for xi, (o, k) in zip(xs + xs, want + want):
        reset()
        x.copy_(xi)
        _ = torch.randn(1000, device="cuda").sum().item()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(pair.gpu.k, k)


def test_workspace_of_an_earlier_graph_stays(palq):
    """A graph keeps its workspace when later, larger calls grow the context's."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(71)
    side = torch.cuda.Stream()
    ctx = P.Context(0, stream=side.cuda_stream)
    w = dev(g.integers(-127, 128, (64, 128)).astype(np.int8))
    ws = torch.full((64,), 1e-3, device="cuda")
    small = P.Linear(ctx, w, ws, max_rows=4)
    x = dev(g.standard_normal((4, 128)), "f32")
    y, ref = torch.empty(4, 64, device="cuda"), torch.empty(4, 64, device="cuda")
    small.run(x, ref)
    ctx.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        small.run(x, y)
    big = P.Linear(ctx, w, ws, max_rows=5000)
    yb = torch.empty(5000, 64, device="cuda")
    xb = dev(g.standard_normal((5000, 128)), "f32")
    torch.cuda.synchronize()
    for _ in range(3):
        big.run(xb, yb)
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)


def test_capture_of_a_larger_shape_is_refused(palq):
    """An attention whose workspace would have to grow while a graph is captured gives an error and leaves the capture whole."""
    import torch
    from paper_2208_01944_amd import palq as P
    side = torch.cuda.Stream()
    ctx = P.Context(0, stream=side.cuda_stream)
    c = P.Cache.empty(80, 1, 64, 64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    b = P.Batch(torch.arange(80, dtype=torch.int32, device="cuda")[None], i32(5000), i32(0, 1), 1, 5120)
    q = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    out, y = torch.empty_like(q), torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(P.PalqError) as e:
            ctx.attention(c, q, out, b, 1.0)
        y.add_(1.0)
    assert e.value.status == P.ERR_NOMEM
    graph.replay()
    torch.cuda.synchronize()
    assert (y.cpu() == 1).all()
    ctx.attention(c, q, out, b, 1.0)
    ctx.sync()
    assert (host(out) == 0).all()


def test_empty_calls(palq):
    """No rows, no requests, no new tokens: no launch, no error."""
    import torch
    from paper_2208_01944_amd import palq as P
    lin = P.Linear(palq, torch.ones(4, 8, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda"), max_rows=4)
    lin.run(torch.empty(0, 8, device="cuda"), torch.empty(0, 4, device="cuda"))
    c = P.Cache.empty(2, 1, 16, 64)
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    for b in (P.Batch(z(2, 1), z(2), z(3), 0, 0), P.Batch(z(0, 1), z(0), z(1), 4, 4), P.Batch(z(1, 1), z(1), z(2), 4, 16)):
        palq.cache_append(c, e, e, b)
        palq.cache_read(c, e, e, b)
        palq.attention(c, e, torch.empty_like(e), b, 1.0)
    palq.sync()

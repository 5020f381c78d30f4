"""Host-only checks of the 8-bit transformer operators: every refusal, on a
validate-only context, and pins of the numpy oracle that the GPU tests use."""
import ctypes

import numpy as np
import pytest

from oracle import serve as S


@pytest.fixture(scope="module")
def P():
    from paper_2208_01944_amd import palq
    return palq


@pytest.fixture(scope="module")
def vctx(P):
    return P.Context(-1)


def at(i, off=0):
    return 0x100000000 * (i + 1) + off


def linear(P, vctx, n_out=64, n_in=128, max_rows=8, w=at(1), w_ld=None, ws=at(2), bias=None):
    h = P.c_p()
    st = P._linear_create(vctx.h, w, n_in if w_ld is None else w_ld, ws, bias, n_out, n_in, max_rows, ctypes.byref(h))
    return st, h


def test_linear_create_refusals(P, vctx):
    st, h = linear(P, vctx)
    assert st == P.OK and P._linear_kernels(h, 1) == b""
    P._linear_destroy(h)
    for kw, want in ((dict(n_out=0), P.ERR_ARG), (dict(n_in=0), P.ERR_ARG), (dict(w_ld=127), P.ERR_ARG), (dict(max_rows=-1), P.ERR_ARG),
                     (dict(w=None), P.ERR_ARG), (dict(ws=None), P.ERR_ARG), (dict(ws=at(2, 2)), P.ERR_ARG),
                     (dict(bias=at(3, 1)), P.ERR_ARG), (dict(n_in=1 << 17), P.ERR_OVERFLOW), (dict(n_out=(1 << 24) + 1), P.ERR_UNSUPPORTED),
                     (dict(max_rows=1 << 25), P.ERR_UNSUPPORTED)):
        st, h = linear(P, vctx, **kw)
        assert st == want and not h.value, kw
        assert vctx.last_error()
    assert P._linear_create(None, at(1), 8, at(2), None, 8, 8, 1, ctypes.byref(P.c_p())) == P.ERR_ARG
    assert P._linear_create(vctx.h, at(1), 8, at(2), None, 8, 8, 1, None) == P.ERR_ARG
    assert P._linear_kernels(None, 1) is None
    P._linear_destroy(None)


def test_linear_run_refusals(P, vctx):
    _, h = linear(P, vctx)
    other = P.Context(-1)

    def run(ctx=vctx.h, lin=h, x=at(4), xt=P.BF16, x_ld=128, xs=None, rows=8, y=at(5), yt=P.BF16, y_ld=64):
        return P._linear_run(ctx, lin, x, xt, x_ld, xs, rows, y, yt, y_ld)

    assert run() == P.OK and run(rows=0, x=None, y=None) == P.OK
    assert run(xt=P.I8, xs=at(6)) == P.OK
    for kw in (dict(ctx=None), dict(lin=None), dict(ctx=other.h), dict(xt=4), dict(xt=-1), dict(yt=P.I8), dict(yt=9), dict(rows=9),
               dict(rows=-1), dict(x_ld=127), dict(y_ld=63), dict(x=None), dict(y=None), dict(xt=P.I8), dict(xs=at(6)),
               dict(x=at(4, 1)), dict(y=at(5, 1)), dict(x=at(4, 2), xt=P.F32), dict(xt=P.I8, xs=at(6, 2)),
               dict(x=at(5, 16)), dict(x=at(5, 8 * 64 * 2 - 2)), dict(x=at(5, -7 * 128 * 2 - 2)), dict(xt=P.I8, xs=at(5, 4))):
        assert run(**kw) == P.ERR_ARG, kw
    assert run(x=at(5, 8 * 64 * 2)) == P.OK and run(x=at(5, -8 * 128 * 2)) == P.OK  # next to each other
    P._linear_destroy(h)


def test_quantize_rows_refusals(P, vctx):
    def run(x=at(1), t=P.F16, rows=4, cols=100, x_ld=100, c=at(2), c_ld=100, s=at(3)):
        return P._quantize_rows(vctx.h, x, t, rows, cols, x_ld, c, c_ld, s)

    assert run() == P.OK and run(rows=0, x=None, c=None, s=None) == P.OK
    for kw in (dict(t=P.I8), dict(t=7), dict(rows=-1), dict(cols=0), dict(x_ld=99), dict(c_ld=99), dict(x=None), dict(c=None),
               dict(s=None), dict(x=at(1, 1)), dict(s=at(3, 2)), dict(c=at(1, 10)), dict(s=at(2, 396)), dict(s=at(1, 4))):
        assert run(**kw) == P.ERR_ARG, kw
    assert run(rows=1 << 31, x_ld=100) == P.ERR_UNSUPPORTED


def cache(P, **over):
    f = dict(pages=8, page_tokens=16, heads=2, head_dim=64, k=at(1), v=at(2), k_scale=at(3), v_scale=at(4)) | over
    return P.CacheDesc(*(f[n] for n, _ in P.CacheDesc._fields_))


def batch(P, **over):
    f = dict(requests=2, max_pages=4, table=at(5), lens=at(6), starts=at(7), tokens=6, max_new=4, max_len=64) | over
    return P.BatchDesc(*(f[n] for n, _ in P.BatchDesc._fields_))


BAD_CACHE = [(dict(pages=0), "ARG"), (dict(heads=0), "ARG"), (dict(page_tokens=24), "UNSUPPORTED"), (dict(page_tokens=256), "UNSUPPORTED"),
             (dict(head_dim=80), "UNSUPPORTED"), (dict(heads=65536), "UNSUPPORTED"), (dict(k=None), "ARG"), (dict(v=at(2, 8)), "ARG"),
             (dict(k_scale=None), "ARG"), (dict(v_scale=at(4, 2)), "ARG")]
BAD_BATCH = [(dict(requests=-1), "ARG"), (dict(max_pages=0), "ARG"), (dict(tokens=-1), "ARG"), (dict(max_new=-1), "ARG"),
             (dict(max_len=-1), "ARG"), (dict(table=None), "ARG"), (dict(lens=at(6, 2)), "ARG"), (dict(starts=None), "ARG"),
             (dict(requests=32768), "UNSUPPORTED")]


def calls(P, vctx):
    """The three calls that take a cache and a batch, with good tensors."""
    def append(c, b, k=at(8), kr=128, kh=64, v=at(9), vr=128, vh=64, t=P.BF16):
        return P._cache_append(vctx.h, c, b, k, kr, kh, v, vr, vh, t)

    def read(c, b, k=at(8), kr=128, kh=64, v=at(9), vr=128, vh=64, t=P.F32):
        return P._cache_read(vctx.h, c, b, k, kr, kh, v, vr, vh, t)

    def attend(c, b, q=at(8), qr=256, qh=64, n=4, o=at(9), r=256, oh=64, t=P.BF16, scale=0.125, causal=1, window=0):
        return P._attention(vctx.h, c, b, q, qr, qh, n, o, r, oh, t, scale, causal, window)

    return append, read, attend


def ref(x):
    return None if x is None else ctypes.byref(x)


@pytest.mark.parametrize("which", [0, 1, 2])
def test_cache_and_batch_refusals(P, vctx, which):
    call = calls(P, vctx)[which]
    assert call(ref(cache(P)), ref(batch(P))) == P.OK
    assert call(ref(cache(P)), ref(batch(P, requests=0, table=None, lens=None, starts=None))) == P.OK
    assert call(None, ref(batch(P))) == P.ERR_ARG and call(ref(cache(P)), None) == P.ERR_ARG
    for over, err in BAD_CACHE:
        assert call(ref(cache(P, **over)), ref(batch(P))) == getattr(P, "ERR_" + err), over
    for over, err in BAD_BATCH:
        assert call(ref(cache(P)), ref(batch(P, **over))) == getattr(P, "ERR_" + err), over


def test_append_and_read_refusals(P, vctx):
    c, b = ref(cache(P)), ref(batch(P))
    for call in calls(P, vctx)[:2]:
        for kw in (dict(t=P.I8), dict(t=-1), dict(k=None), dict(v=None), dict(k=at(8, 1)), dict(kh=63), dict(vr=63), dict(kr=-128),
                   dict(vh=-64), dict(kr=1 << 60)):
            assert call(c, b, **kw) == P.ERR_ARG, kw


def test_attention_refusals(P, vctx):
    attend = calls(P, vctx)[2]
    c, b = ref(cache(P)), ref(batch(P))
    assert attend(c, b, window=5) == P.OK and attend(c, b, causal=0) == P.OK
    for kw in (dict(t=P.F32), dict(t=P.I8), dict(n=3), dict(n=0), dict(q=None), dict(o=None), dict(q=at(8, 1)), dict(qh=63),
               dict(r=63), dict(scale=float("inf")), dict(scale=float("nan")), dict(causal=2), dict(window=-1),
               dict(causal=0, window=4), dict(o=at(8)), dict(o=at(8, 2 * (5 * 256 + 255)))):
        assert attend(c, b, **kw) == P.ERR_ARG, kw
    assert attend(c, b, o=at(8, 2 * 6 * 256)) == P.OK
    assert attend(c, ref(batch(P, max_new=(1 << 30) - 1))) == P.ERR_UNSUPPORTED


def test_binding_refusals(P):
    import torch
    z = lambda *s, d=torch.int8: torch.zeros(*s, dtype=d)  # noqa: E731
    f = torch.float32
    ok = (z(2, 1, 16, 64), z(2, 1, 64, 16), z(2, 1, d=f), z(2, 1, d=f))
    c = P.Cache(*ok)
    for i, bad in ((0, z(2, 1, 64, 16)), (1, z(2, 1, 16, 64)), (0, z(2, 1, 16, 64, d=f)), (2, z(2, 2, d=f)), (3, z(2, 1)),
                   (0, z(2, 1, 16, 128)[..., ::2])):
        with pytest.raises(P.PalqError):
            P.Cache(*(bad if j == i else t for j, t in enumerate(ok)))
    i32 = torch.int32
    args = (z(2, 3, d=i32), z(2, d=i32), z(3, d=i32))
    b = P.Batch(*args, 4, 32)
    for i, bad in ((0, z(2, 3)), (1, z(3, d=i32)), (2, z(2, d=i32)), (0, z(3, 2, d=i32).t())):
        with pytest.raises(P.PalqError):
            P.Batch(*(bad if j == i else t for j, t in enumerate(args)), 4, 32)
    ctx = P.Context(-1)
    x = z(4, 1, 64, d=torch.bfloat16)
    for k, v in ((x, x[:3]), (x, x.float()), (x[..., :32], x), (z(4, 2, 64, d=torch.bfloat16),) * 2, (z(4, 1, 64, d=torch.float64),) * 2,
                 (z(4, 1, 128, d=torch.bfloat16)[..., ::2],) * 2):
        with pytest.raises(P.PalqError):
            ctx.cache_append(c, k, v, b)
    with pytest.raises(P.PalqError):
        ctx.attention(c, x, x[:2], b, 1.0)
    lin = P.Linear(ctx, z(8, 16), z(8, d=f), max_rows=4)
    for xx, y, s in ((z(4, 15, d=f), z(4, 8, d=f), None), (z(4, 16, d=f), z(3, 8, d=f), None), (z(4, 16, d=f), z(4, 9, d=f), None),
                     (z(4, 16), z(4, 8, d=f), z(3, d=f)), (z(4, 32, d=f)[:, ::2], z(4, 8, d=f), None), (z(5, 16, d=f), z(5, 8, d=f), None)):
        with pytest.raises(P.PalqError):
            lin.run(xx, y, x_scale=s)
    with pytest.raises(P.PalqError):
        P.Linear(ctx, z(8, 16, d=f), z(8, d=f))
    with pytest.raises(P.PalqError):
        ctx.quantize_rows(z(4, 16, d=f), z(4, 15), z(4, d=f))


# ------------------------------------------------------------------ pins of the oracle
def test_oracle_quantiser():
    s = S.scale_of(np.float32([-254.0, 3.0]))
    assert abs(s - 2.0) < 1e-6
    np.testing.assert_array_equal(S.codes_of(np.float32([-254, 127, 1, 3, 5, 0]), np.float32(2)), [-127, 64, 0, 2, 2, 0])  # ties to even
    assert S.scale_of(np.zeros(3)) == np.float32(2.0 ** -100) and not S.codes_of(np.zeros(3), S.scale_of(np.zeros(3))).any()
    g = np.random.default_rng(1)
    x = g.standard_normal(4000).astype(np.float32) * 7
    s = S.scale_of(x)
    q = S.codes_of(x, s)
    assert np.abs(q).max() == 127 and np.abs(q * np.float64(s) - x).max() <= 0.5 * s * (1 + 1e-5)
    assert np.isnan(S.scale_of(np.float32([1, np.inf]))) and not S.codes_of(np.float32([1, np.inf]), np.float32(np.nan)).any()


def test_oracle_cache_round_trip():
    """Values read back lie within half a step of the block's scale of what was appended (one step more for each rescaling)."""
    g = np.random.default_rng(2)
    c = S.Cache(6, 2, 16, 8)
    table, x = [[4, 0, 2], [1, 5, 3]], g.standard_normal((60, 2, 8)).astype(np.float32)
    c.append(table, [20, 40], [0, 20, 60], x, 3 * x)
    k, v = c.read(table, [20, 40], [0, 20, 60])
    for got, want, sc in ((k, x, c.ks), (v, 3 * x, c.vs)):
        for r, (a, n) in enumerate(((0, 20), (20, 40))):
            for j in range(n):
                assert (np.abs(got[a + j] - want[a + j]) <= 0.5001 * sc[table[r][j // 16]][:, None]).all()


def test_oracle_attention_against_torch():
    import torch
    g = np.random.default_rng(3)
    c = S.Cache(5, 1, 16, 8)
    x, y = g.standard_normal((2, 40, 1, 8)).astype(np.float32)
    table = [[3, 1, 4]]
    c.append(table, [40], [0, 40], x, y)
    q = g.standard_normal((40, 2, 8)).astype(np.float32)
    k, v = (torch.from_numpy(np.concatenate([z[table[0][b], 0] * np.float64(s[table[0][b], 0]) for b in range(3)])[:40])
            for z, s in ((c.k, c.ks), (c.v, c.vs)))
    for causal, window in ((True, 0), (True, 5), (False, 0)):
        out = c.attend(table, [40], [0, 40], q, 0.3, causal, window)[0]
        z = torch.from_numpy(q).double().transpose(0, 1) @ k.T * 0.3
        i = torch.arange(40)
        if causal:
            z = z.masked_fill(i[None, :] > i[:, None], -np.inf)
        if window:
            z = z.masked_fill(i[None, :] <= i[:, None] - window, -np.inf)
        np.testing.assert_allclose(out, (z.softmax(-1) @ v).transpose(0, 1).numpy(), rtol=1e-10, atol=1e-12)

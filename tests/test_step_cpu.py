"""Host-only checks of head norms with rotation, attention with sinks and over trees, and
log probabilities: every refusal, on a validate-only context, and pins of the numpy oracle that
the GPU tests use."""
import ctypes

import numpy as np
import pytest

from oracle import serve as S
from oracle import step as T
from tests.test_serve_cpu import BAD_BATCH, BAD_CACHE, P, at, batch, cache, ref, vctx  # noqa: F401


def tree(P, **over):  # noqa: F811
    f = dict(mask=at(20), words=1) | over
    return P.TreeDesc(f["mask"], f["words"])


BAD_TREE = [(dict(words=0), "ARG"), (dict(words=17), "UNSUPPORTED"), (dict(mask=None), "ARG"), (dict(mask=at(20, 4)), "ARG")]


def rotation(P, ctx, freq=(1.0, 0.5), pairs=2, interleaved=0):  # noqa: F811
    h = P.c_p()
    f = None if freq is None else (ctypes.c_double * max(len(freq), 1))(*freq)
    return P._rotation_create(ctx.h, f, pairs, interleaved, ctypes.byref(h)), h


def test_rotation_refusals(P, vctx):  # noqa: F811
    st, h = rotation(P, vctx)
    assert st == P.OK and h.value
    P._rotation_destroy(h)
    for kw in (dict(freq=None), dict(pairs=0), dict(freq=(1.0,) * 200, pairs=129), dict(interleaved=2), dict(freq=(1.0, float("nan"))),
               dict(freq=(float("inf"), 1.0))):
        st, h = rotation(P, vctx, **kw)
        assert st == P.ERR_ARG and not h.value and vctx.last_error(), kw
    assert P._rotation_create(vctx.h, (ctypes.c_double * 1)(1.0), 1, 0, None) == P.ERR_ARG
    P._rotation_destroy(None)
    for bad in ([], [[1.0]], [1.0] * 129, [np.nan]):
        with pytest.raises(P.PalqError):
            P.Rotation(vctx, bad)


def rotate(P, vctx):  # noqa: F811
    """The call with good tensors: queries of 4 heads and keys of 2 within rows of 8 heads, in tensors of their own."""
    def run(rot=None, b=None, t=None, q=at(8), qr=512, qh=64, qn=4, qo=at(9), qor=256, qoh=64, qw=at(10), k=at(8, 512), kr=512, kh=64, kn=2,
            ko=at(11), kor=128, koh=64, kw=at(12), dim=64, type=P.BF16, eps=1e-6, no_q=False,
            no_k=False):
        h = [P.HeadsDesc(*f) for f in ((q, qr, qh, qo, qor, qoh, qw, qn), (k, kr, kh, ko, kor, koh, kw, kn))]
        at_q, at_k = (None if none else ctypes.addressof(x) for x, none in zip(h, (no_q, no_k)))
        return P._norm_rotate(vctx.h, rot, ref(batch(P)) if b is None else b, t, at_q, at_k, dim, type, eps)
    return run


def test_norm_rotate_refusals(P, vctx):  # noqa: F811
    run = rotate(P, vctx)
    _, rot = rotation(P, vctx, [1.0] * 32, 32)
    _, wide = rotation(P, vctx, [1.0] * 33, 33)
    other = P.Context(-1)
    _, foreign = rotation(P, other)
    assert run() == run(rot=rot) == run(t=ref(tree(P))) == P.OK
    assert run(no_k=True) == run(no_q=True) == run(qw=None, kw=None) == run(eps=0.0, qw=None, kw=None) == run(no_k=True, k=None) == P.OK
    assert run(type=P.F32, q=at(8), k=at(8, 1024)) == P.OK
    in_place = dict(qo=at(8), qor=512, qoh=64, ko=at(8, 512), kor=512, koh=64)
    assert run(**in_place) == P.OK
    for kw in (dict(rot=wide), dict(rot=foreign), dict(type=P.I8), dict(type=9), dict(no_q=True, no_k=True), dict(qn=0), dict(kn=0), dict(qn=-1), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(eps=1e-40), dict(eps=0.0), dict(eps=0.0, qw=None), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None),
               dict(q=at(8, 1)), dict(ko=at(11, 1)), dict(qw=at(10, 2)), dict(qh=63), dict(qor=63), dict(koh=32), dict(kor=-128),
               dict(qor=1 << 60), dict(qoh=64, qor=64),                            # rows of an output over each other
               dict(qo=at(8, 2)), dict(qo=at(8), qor=256), dict(in_place, qo=at(8, 128)),  # over its input, but not in place
               dict(qo=at(8, 512)), dict(ko=at(8), kor=512),                       # over the other's input
               dict(ko=at(9, 64)), dict(qo=at(11, -64)),                           # over the other output
               dict(qw=at(9, 100)), dict(kw=at(9)), dict(t=ref(tree(P, mask=at(9, 8))))):
        assert run(**kw) == P.ERR_ARG, kw
    for kw in (dict(dim=80), dict(dim=32), dict(dim=512), dict(qn=65536, qor=1 << 23, qr=1 << 23)):
        assert run(**kw) == P.ERR_UNSUPPORTED, kw
    for over, err in BAD_TREE:
        assert run(t=ref(tree(P, **over))) == getattr(P, "ERR_" + err), over
    for over, err in BAD_BATCH:
        assert run(b=ref(batch(P, **over))) == getattr(P, "ERR_" + err), over
    empty = ref(batch(P, tokens=0))
    assert run(b=empty, q=None, qo=None, k=None, ko=None) == P.OK
    P._rotation_destroy(rot)
    P._rotation_destroy(wide)
    P._rotation_destroy(foreign)


@pytest.mark.parametrize("form", ["sinks", "tree"])
def test_attention_refusals(P, vctx, form):  # noqa: F811
    def attend(c=None, b=None, t=None, q=at(8), qr=256, qh=64, n=4, o=at(9), r=256, oh=64, type=P.BF16, scale=0.125, window=0, sinks=0):
        c, b = ref(cache(P)) if c is None else c, ref(batch(P)) if b is None else b
        if form == "sinks":
            return P._attention_sinks(vctx.h, c, b, q, qr, qh, n, o, r, oh, type, scale, window, sinks)
        return P._attention_tree(vctx.h, c, b, ref(tree(P)) if t is None else t, q, qr, qh, n, o, r, oh, type, scale, window, sinks)

    assert attend() == attend(window=5) == attend(window=5, sinks=2) == attend(sinks=2) == attend(window=2 ** 31 - 1, sinks=2 ** 31 - 1) == P.OK
    for kw in (dict(type=P.F32), dict(type=P.I8), dict(n=3), dict(n=0), dict(q=None), dict(o=None), dict(q=at(8, 1)), dict(qh=63), dict(r=63),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(window=-1), dict(sinks=-1), dict(o=at(8)), dict(o=at(8, 2 * (5 * 256 + 255))),
               dict(o=at(1)), dict(o=at(3))):
        assert attend(**kw) == P.ERR_ARG, kw
    assert attend(b=ref(batch(P, max_new=(1 << 30) - 1))) == P.ERR_UNSUPPORTED
    for over, err in BAD_CACHE:
        assert attend(c=ref(cache(P, **over))) == getattr(P, "ERR_" + err), over
    for over, err in BAD_BATCH:
        assert attend(b=ref(batch(P, **over))) == getattr(P, "ERR_" + err), over
    if form == "tree":
        for over, err in BAD_TREE:
            assert attend(t=ref(tree(P, **over))) == getattr(P, "ERR_" + err), over
        assert attend(t=ref(tree(P, mask=at(9, 8)))) == P.ERR_ARG
        assert P._attention_tree(vctx.h, ref(cache(P)), ref(batch(P)), None, at(8), 256, 64, 4, at(9), 256, 64, P.BF16, 0.1, 0, 0) == P.ERR_ARG


def test_log_probs_refusals(P, vctx):  # noqa: F811
    def run(x=at(1), type=P.BF16, rows=4, vocab=100, ld=100, scale=1.0, ids=at(2), given=2, out=at(3), ent=at(4), top=5, ti=at(5), to=at(6)):
        return P._log_probs(vctx.h, x, type, rows, vocab, ld, scale, ids, given, out, ent, top, ti, to)

    assert run() == run(ent=None) == run(given=0, ids=None, out=None) == run(top=0, ti=None, to=None) == P.OK
    assert run(rows=0, x=None, ids=None, out=None, ti=None, to=None) == run(vocab=5, ld=5) == run(top=64) == P.OK
    for kw in (dict(type=P.I8), dict(type=-1), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(given=-1), dict(top=-1), dict(top=6, vocab=5, ld=5),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.0 ** 120), dict(scale=2.0 ** -120),
               dict(x=None), dict(ids=None), dict(out=None), dict(ti=None), dict(to=None), dict(x=at(1, 1)), dict(ids=at(2, 2)), dict(out=at(3, 1)),
               dict(ent=at(4, 2)), dict(ti=at(5, 3)), dict(to=at(6, 1)), dict(out=at(1, 796)), dict(ent=at(2, 28)), dict(ti=at(3, 28)), dict(to=at(5, 76)),
               dict(to=at(4, 12)), dict(ld=1 << 60)):
        assert run(**kw) == P.ERR_ARG, kw
    assert run(out=at(1, 800)) == P.OK  # next to each other
    for kw in (dict(top=65), dict(rows=1 << 31), dict(vocab=(1 << 30) + 1, ld=1 << 31)):
        assert run(**kw) == P.ERR_UNSUPPORTED, kw


def test_binding_refusals(P):  # noqa: F811
    import torch
    i32, f, bf = torch.int32, torch.float32, torch.bfloat16
    z = lambda *s, d=f: torch.zeros(*s, dtype=d)  # noqa: E731
    ctx, other = P.Context(-1), P.Context(-1)
    b = P.Batch(z(2, 3, d=i32), z(2, d=i32), z(3, d=i32), 4, 32)
    q, k = z(6, 4, 64, d=bf), z(6, 2, 64, d=bf)
    ctx.norm_rotate(b, q, q, k, k, q_weight=z(64), eps=1e-6, rotation=P.Rotation(ctx, [1.0] * 32), tree=z(6, 1, d=torch.int64))
    ctx.norm_rotate(b, q, torch.zeros_like(q), eps=1e-6)
    for args, kw in (((q, q, k), {}), ((q, q, None, k), {}), ((q, k), {}), ((q, q.float()), {}), ((q, q, k.float(), k.float()), {}),
                     ((q, q, k[:5], k[:5]), {}), ((q, q, k[..., :32], k[..., :32]), {}), ((q[..., ::2], q[..., ::2]), {}),
                     ((z(6, 4, 64, d=torch.float64),) * 2, {}), ((q, q), dict(eps=0)), ((q, q), dict(eps=-1.0)), ((q, q), dict(eps=1e-6, q_weight=z(63))),
                     ((q, q), dict(eps=1e-6, q_weight=z(64, d=bf))), ((q, q), dict(q_weight=z(64))), ((q, q), dict(rotation=P.Rotation(other, [1.0]))),
                     ((q, q), dict(tree=z(6, 1, d=i32))), ((q, q), dict(tree=z(5, 1, d=torch.int64))), ((q, q), dict(tree=z(6, 2, d=torch.int64)[:, ::2])),
                     ((q, q), dict(tree=z(6, 17, d=torch.int64)))):
        with pytest.raises(P.PalqError):
            ctx.norm_rotate(b, *args, **kw)
    i8 = torch.int8
    c = P.Cache(z(2, 2, 16, 64, d=i8), z(2, 2, 64, 16, d=i8), z(2, 2), z(2, 2))
    o = torch.zeros_like(q)
    ctx.attention(c, q, o, b, 1.0, window=4, sinks=2, tree=z(6, 1, d=torch.int64))
    for kw in (dict(sinks=-1), dict(sinks=1, causal=False), dict(tree=z(6, 1, d=i32)), dict(tree=z(6, 1, d=torch.int64), causal=False),
               dict(tree=z(5, 1, d=torch.int64)), dict(tree=z(6, d=torch.int64)), dict(window=-1, sinks=1)):
        with pytest.raises(P.PalqError):
            ctx.attention(c, q, o, b, 1.0, **kw)
    x, ids, out = z(6, 50), z(6, 2, d=i32), z(6, 2)
    top = dict(top_ids=z(6, 3, d=i32), top=z(6, 3))
    ctx.log_probs(x, ids, out, entropy=z(6), **top)
    ctx.log_probs(x, ids[:, 0].contiguous(), out[:, 0].contiguous())
    ctx.log_probs(x, None, None, **top)
    for args, kw in (((x, ids, z(6, 1)), {}), ((x, ids, None), {}), ((x, ids.long(), out), {}), ((x, ids, out.double()), {}), ((x, ids[:5], out[:5]), {}),
                     ((x, z(6, 4, d=i32)[:, ::2], out), {}), ((x[:, ::2], ids, out), {}), ((x.double(), ids, out), {}), ((x, ids, out), dict(entropy=z(5))),
                     ((x, ids, out), dict(top=z(6, 3))), ((x, ids, out), dict(top_ids=z(6, 3, d=i32))), ((x, ids, out), dict(top, top=z(6, 2))),
                     ((x, ids, out), dict(top_ids=z(5, 3, d=i32), top=z(5, 3))), ((x, ids, out), dict(top_ids=z(6, 51, d=i32), top=z(6, 51))),
                     ((x, ids, out), dict(scale=0.0))):
        with pytest.raises(P.PalqError):
            ctx.log_probs(*args, **kw)


def test_tensors_off_the_context_device_are_refused(P):  # noqa: F811
    import torch
    i32, bf = torch.int32, torch.bfloat16
    z = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d)  # noqa: E731
    ctx = P.Context(-1)
    ctx.device = 0  # (to the binding)
    b = P.Batch(z(2, 3, d=i32), z(2, d=i32), z(3, d=i32), 4, 32)
    q = z(6, 4, 64, d=bf)
    c = P.Cache(z(2, 2, 16, 64, d=torch.int8), z(2, 2, 64, 16, d=torch.int8), z(2, 2), z(2, 2))
    for call in (lambda: ctx.norm_rotate(b, q, q, eps=1e-6), lambda: ctx.log_probs(z(4, 50), z(4, d=i32), z(4)),
                 lambda: ctx.attention(c, q, q.clone(), b, 1.0, window=3, sinks=1),
                 lambda: ctx.attention(c, q, q.clone(), b, 1.0, tree=z(6, 1, d=torch.int64))):
        with pytest.raises(P.PalqError, match="device|cuda:0"):
            call()


# ------------------------------------------------------------------ pins of the oracle
def test_oracle_positions():
    assert T.positions([5, 3, 2], [0, 2, 2, 6]).tolist() == [3, 4, -2, -1, 0, 1]
    mask = np.uint64([[0b1], [0b11], [0b101], [0b1000]])  # a root, two children of it, one that sees only itself
    assert T.positions([10], [0, 4], mask).tolist() == [6, 7, 7, 6]
    assert T.positions([10], [0, 3], np.uint64([[0xf8], [0], [0b111]])).tolist() == [7, 7, 9]  # bits past the new tokens count nothing


def test_oracle_rotation():
    """Quarter turns by hand, the complex plane, and that a norm has the mean square of its weights."""
    x = np.arange(1.0, 9.0)[None, None]
    pos = np.array([1])
    out, _ = T.norm_rotate(x, pos, [np.pi / 2, 0.0])
    np.testing.assert_allclose(out[0, 0].astype(float), [-3, 2, 1, 4, 5, 6, 7, 8], atol=1e-15)
    out, _ = T.norm_rotate(x, pos, [np.pi / 2, np.pi], interleaved=True)
    np.testing.assert_allclose(out[0, 0].astype(float), [-2, 1, -3, -4, 5, 6, 7, 8], atol=1e-15)
    g = np.random.default_rng(0)
    x, pos, f = g.standard_normal((20, 3, 16)), np.arange(20) * 1000, 1e3 ** -(np.arange(8) / 8)
    out, _ = T.norm_rotate(x, pos, f)
    z = (x[..., :8] + 1j * x[..., 8:]) * np.exp(1j * pos[:, None] * f)[:, None]
    np.testing.assert_allclose(out.astype(float), np.concatenate([z.real, z.imag], -1), atol=1e-10)
    w = g.standard_normal(16).astype(np.float32)
    y, _ = T.norm_rotate(x, pos, (), weight=w, eps=1e-12)
    np.testing.assert_allclose(((y / w).astype(float) ** 2).mean(-1), 1, atol=1e-10)


def test_oracle_log_probs():
    from scipy.special import log_softmax
    g = np.random.default_rng(1)
    x = g.standard_normal((4, 30)) * 3
    x[1, 3:20] = -np.inf
    x[2] = -np.inf
    ids = np.array([[0, 29], [4, -1], [0, 1], [30, 7]])
    out, ent, ti, to, _ = T.log_probs(x, 0.5, ids, 4)
    l = log_softmax(x[[0, 1, 3]] * 0.5, axis=1)
    np.testing.assert_allclose(out[0], l[0, [0, 29]], rtol=1e-12)
    assert out[1, 0] == -np.inf and np.isnan(out[1, 1]) and (out[2] == -np.inf).all() and ent[2] == 0 and np.isnan(out[3, 0])
    p = np.exp(l)
    np.testing.assert_allclose(ent[[0, 1, 3]], -np.where(p > 0, p * np.where(p > 0, l, 0), 0).sum(1), rtol=1e-12)
    assert ti[0].tolist() == np.argsort(-x[0])[:4].tolist() and ti[2].tolist() == [0, 1, 2, 3]
    np.testing.assert_allclose(to[0], l[0, ti[0]], rtol=1e-12)


def test_oracle_attention_with_sinks_and_trees():
    """Without either it is the plain oracle; a mask of ancestors is plain attention of the branch alone."""
    g = np.random.default_rng(2)
    c = S.Cache(4, 1, 16, 8)
    x, y = g.standard_normal((2, 40, 1, 8)).astype(np.float32)
    table = [[3, 1, 2]]
    c.append(table, [40], [0, 40], x, y)
    q = g.standard_normal((6, 2, 8))
    for window in (0, 5):
        np.testing.assert_allclose(T.attend(c, table, [40], [0, 6], q, 0.3, window)[0], c.attend(table, [40], [0, 6], q, 0.3, True, window)[0])
    np.testing.assert_allclose(T.attend(c, table, [40], [0, 6], q, 0.3, 5, 40)[0], c.attend(table, [40], [0, 6], q, 0.3)[0])
    seen = T.attend(c, table, [40], [0, 6], q, 0.3, 5, 3)[3]
    assert (seen == 8).all()
    mask = np.uint64([[1], [3], [5], [0b1101], [0], [0b100000]])
    out, _, _, seen = T.attend(c, table, [40], [0, 6], q, 0.3, mask=mask)
    assert seen[:, 0].tolist() == [35, 36, 36, 37, 34, 35]
    k, v = (c.values(table, 0, 40, 0, w)[0] for w in "kv")
    rows = np.r_[0:34, 34, 36, 37]
    s = q[3, 1] @ k[rows].T * 0.3
    np.testing.assert_allclose(out[3, 1], np.exp(s - s.max()) @ v[rows] / np.exp(s - s.max()).sum(), rtol=1e-10)

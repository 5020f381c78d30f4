"""Host-only checks: tensors that the cache's calls write, laid over themselves, each
other or the cache, are refused; every layout without an overlap is taken."""
import itertools

import pytest

from tests.test_serve_cpu import at, batch, cache, ref


@pytest.fixture(scope="module")
def P():
    from paper_2208_01944_amd import palq
    return palq


def rows(base, tokens, row, heads, head, dim):
    return [set(range(base + t * row + h * head, base + t * row + h * head + dim)) for t in range(tokens) for h in range(heads)]


def disjoint(sets):
    return sum(len(s) for s in sets) == len(set().union(*sets))


TOKENS, HEADS, DIM = 5, 3, 64
STRIDES = [64, 65, 96, 128, 130, 160, 191, 192, 193, 200, 256, 320, 384, 64 * 15 + 7]


def test_attention_outputs_of_every_layout(P):
    """Row and head strides in every order: refused exactly where two rows share an element."""
    ctx, c, b = P.Context(-1), cache(P, heads=HEADS, head_dim=DIM), batch(P, tokens=TOKENS)
    kinds = set()
    for row, head in itertools.product(STRIDES, STRIDES):
        good = disjoint(rows(0, TOKENS, row, HEADS, head, DIM))
        kinds.add(good)
        st = P._attention(ctx.h, ref(c), ref(b), at(8), HEADS * DIM, DIM, HEADS, at(9), row, head, P.BF16, 1.0, 1, 0)
        assert st == (P.OK if good else P.ERR_ARG), (row, head)
    assert kinds == {True, False}


def test_read_outputs_of_every_layout(P):
    ctx, c, b = P.Context(-1), cache(P, heads=HEADS, head_dim=DIM), batch(P, tokens=TOKENS)
    kinds = set()
    for row, head, apart in itertools.product([192, 200, 256, 384, 448], [64, 128, 65], [0, 1, 63, 64, 65, 128, 192, 200, 384, 1000, 5000, -64, -63]):
        k = rows(0, TOKENS, row, HEADS, head, DIM)
        good = disjoint(k + rows(apart, TOKENS, row, HEADS, head, DIM))
        kinds.add(good)
        st = P._cache_read(ctx.h, ref(c), ref(b), at(8, 4096), row, head, at(8, 4096 + 2 * apart), row, head, P.BF16)
        assert st == (P.OK if good else P.ERR_ARG), (row, head, apart)
    assert kinds == {True, False}
    # different strides: at least their first rows are apart
    assert P._cache_read(ctx.h, ref(c), ref(b), at(8), 192, 64, at(8, 2 * 63), 256, 64, P.BF16) == P.ERR_ARG
    assert P._cache_read(ctx.h, ref(c), ref(b), at(8), 192, 64, at(9), 256, 64, P.BF16) == P.OK


def test_outputs_over_the_cache(P):
    ctx, c, b = P.Context(-1), cache(P), batch(P)  # 8 pages of 16 tokens, 2 heads of 64
    codes, scales = 8 * 2 * 16 * 64, 8 * 2 * 4
    for i, size in ((1, codes), (2, codes), (3, scales), (4, scales)):
        out = 6 * 128 * 2
        for off, want in ((0, P.ERR_ARG), (size - 2, P.ERR_ARG), (2 - out, P.ERR_ARG), (size, P.OK), (-out, P.OK)):
            assert P._attention(ctx.h, ref(c), ref(b), at(8), 128, 64, 2, at(i, off), 128, 64, P.BF16, 1.0, 1, 0) == want, (i, off)
            assert P._cache_read(ctx.h, ref(c), ref(b), at(i, off), 128, 64, at(9), 128, 64, P.BF16) == want, (i, off)
            assert P._cache_read(ctx.h, ref(c), ref(b), at(9), 128, 64, at(i, off), 128, 64, P.BF16) == want, (i, off)


def test_one_row_or_none(P):
    """Strides of a tensor with one token or one head do not count; no tokens, no tensor."""
    ctx = P.Context(-1)
    one, c = batch(P, tokens=1), cache(P)
    assert P._cache_read(ctx.h, ref(c), ref(one), at(8), 0, 64, at(8, 256), 0, 64, P.BF16) == P.OK
    assert P._cache_read(ctx.h, ref(c), ref(one), at(8), 0, 64, at(8, 254), 0, 64, P.BF16) == P.ERR_ARG
    h1 = cache(P, heads=1)
    assert P._attention(ctx.h, ref(h1), ref(batch(P)), at(8), 64, 0, 1, at(9), 64, 0, P.BF16, 1.0, 1, 0) == P.OK
    assert P._cache_read(ctx.h, ref(c), ref(batch(P, tokens=0)), None, 128, 64, None, 128, 64, P.F32) == P.OK

"""GPU checks of attention with sinks and over trees where requests are longer than max_len or
their table: tokens past the bound are left out, and the rows' positions stay, so that a window
may begin behind the last token that is there and only the first ones are seen."""
import numpy as np
import pytest

from oracle import step as S
from tests.test_gpu_serve import Pair, check_attend, cumsum, dev, host, paged, say
from tests.test_gpu_sight import SHAPES
from tests.test_gpu_step import masks_dev, random_masks

pytestmark = pytest.mark.gpu


class Sees:
    """A pair whose oracle leaves out what lies past `limit` tokens."""

    def __init__(self, ref, mask, limit):
        self.cache, self.vs, self.mask, self.limit, self.ref = ref, ref.vs, mask, limit, self

    def attend(self, table, lens, starts, q, scale, **kw):
        return S.attend(self.cache, table, lens, starts, q, scale, mask=self.mask, limit=self.limit, **kw)


def run_bounded(P, ctx, seed, dtype, page, dim, heads, group, lens, new, limit, window, sinks, words, by_table):
    """limit: max_len, or (by_table, then whole pages) what the table holds.  out lies inside a larger tensor, whose other
    elements stay."""
    import torch
    g = np.random.default_rng(seed)
    assert not by_table or limit % page == 0
    table, pages = paged(g, [min(n, limit) for n in lens], page, width=-(-limit // page))
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens)
    starts = cumsum(new)
    masks = random_masks(g, lens, starts, words) if words else None
    q = dev(g.standard_normal((starts[-1], heads * group, dim)) * 1.5, dtype)
    big = torch.full((starts[-1] + 2, heads * group + 2, dim), 3.0, dtype=q.dtype, device="cuda")
    out = big[1:-1, 1:-1]
    b = pair.batch(table, lens, starts, max_len=max(lens) if by_table else limit)
    ctx.attention(pair.gpu, q, out, b, dim ** -0.5, window=window, sinks=sinks, tree=masks_dev(masks) if words else None)
    ctx.sync()
    check_attend(Sees(pair.ref, masks, limit), host(out), table, lens, starts, host(q), dim ** -0.5, dtype, window=window, sinks=sinks)
    out.fill_(3.0)
    assert (big == 3.0).all()


# bounds inside the sinks' last tile, at its end and past it; windows that begin in the bound's tile and far behind it
BOUNDS = [(48, 10, 4), (96, 1, 100), (128, 2, 200), (144, 30, 65), (192, 100, 1000), (48, 10, 2 ** 31 - 1), (64, 3, 64)]


@pytest.mark.parametrize("words", [0, 1])
@pytest.mark.parametrize("by_table", [False, True])
@pytest.mark.parametrize("page,dim,heads,group", SHAPES)
@pytest.mark.parametrize("limit,window,sinks", BOUNDS)
def test_single_rows_past_the_bound(palq, page, dim, heads, group, limit, window, sinks, by_table, words):
    from paper_2208_01944_amd import palq as P
    say("bound single", page, dim, heads, group, limit, window, sinks, by_table, words)
    limit = -(-limit // page) * page if by_table else limit - 3
    lens = [1, limit - 1, limit, limit + 1, limit + 2, limit + window, limit + window + 1, limit + 63, limit + 400, 2 ** 31 - 1]
    run_bounded(P, palq, page + dim, "bf16", page, dim, heads, group, lens, [1] * len(lens), limit, window, sinks, words, by_table)


@pytest.mark.parametrize("words", [0, 2])
@pytest.mark.parametrize("dtype,page,dim,heads,group,limit,new,window,sinks", [
    ("bf16", 64, 128, 1, 4, 100, [5, 33, 70, 1], 17, 30),
    ("f16", 16, 64, 2, 1, 270, [70, 1, 64, 90], 30, 270),
    ("bf16", 32, 96, 1, 2, 85, [90, 13, 40, 2], 7, 5),
    ("f16", 128, 256, 1, 2, 200, [40, 9, 60, 3], 100, 140),
    # the kernel of 128 rows
    ("f16", 16, 64, 16, 2, 150, [128, 40, 131, 100, 1, 64, 120], 33, 140),
    ("bf16", 64, 128, 16, 2, 120, [128, 40, 131, 100, 1, 64, 120], 10, 70),
    ("bf16", 32, 96, 16, 2, 90, [131, 40, 5, 100, 1, 64, 120], 50, 5),
    ("f16", 128, 256, 8, 1, 140, [200, 40, 131, 70, 1, 64, 0, 120], 20, 130),
])
def test_rows_across_the_bound(palq, dtype, page, dim, heads, group, limit, new, window, sinks, words):
    """Requests that end before, at and behind the bound, so that rows of one block differ in whether their window reaches it."""
    from paper_2208_01944_amd import palq as P
    say("bound rows", dtype, page, dim, heads, group, limit, window, sinks, words)
    past = [10, 0, 60, 200, -30, 1000, window, 2 ** 20]
    lens = [max(n, limit + p) for n, p in zip(new, past)]
    run_bounded(P, palq, page * 3 + dim, dtype, page, dim, heads, group, lens, new, limit, window, sinks, words, False)


@pytest.mark.parametrize("words", [0, 1])
@pytest.mark.parametrize("rows", [1, 20])
def test_long_rows_past_the_bound(palq, rows, words):
    """Parts that are joined: requests whose windows lie past 9000 tokens see 4990 first ones, others both."""
    from paper_2208_01944_amd import palq as P
    say("bound long", rows, words)
    run_bounded(P, palq, rows, "bf16", 32, 64, 1, 2, [9000, 2 ** 30, 12005, 8000], [rows, rows, rows, rows], 9000, 3000, 4990, words, False)

"""GPU checks of attention with sinks and over trees of drafted tokens against the numpy
oracle, under the bound that plain attention has (tests/test_gpu_serve.py)."""
import numpy as np
import pytest

from oracle import step as S
from tests.test_gpu_serve import Pair, check_attend, cumsum, dev, host, paged, say
from tests.test_gpu_step import masks_dev, random_masks

pytestmark = pytest.mark.gpu


class Sees:
    """A pair whose oracle is the one with sinks and trees."""

    def __init__(self, ref, mask):
        self.cache, self.vs, self.mask, self.ref = ref, ref.vs, mask, self

    def attend(self, table, lens, starts, q, scale, **kw):
        return S.attend(self.cache, table, lens, starts, q, scale, mask=self.mask, **kw)


def chains(starts, words):
    """Masks by which every row sees the new tokens up to itself: the order that plain attention takes."""
    m = np.zeros((starts[-1], words), np.uint64)
    for a, b in zip(starts[:-1], starts[1:]):
        for t in range(b - a):
            for w in range(words):
                m[a + t, w] = (1 << max(0, min(64, t + 1 - 64 * w))) - 1
    return m


def run_case(P, ctx, seed, dtype, page, dim, heads, group, lens, new, window=0, sinks=0, words=0, masks=None, max_len=None, spread=0.5,
             missing=(), most=None):
    import torch
    g = np.random.default_rng(seed)
    table, pages = paged(g, lens, page)
    for r, block in missing:
        table[r, block] = -1 if r % 2 else pages
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens, spread)
    starts = cumsum(new)
    if words and masks is None:
        masks = random_masks(g, lens, starts, words)
    q = dev(g.standard_normal((starts[-1], heads * group, dim)) * 1.5, dtype)
    out = torch.full_like(q, 3.0)
    b = pair.batch(table, lens, starts, max_len=max_len)
    tree = masks_dev(masks) if words else None
    ctx.attention(pair.gpu, q, out, b, dim ** -0.5, window=window, sinks=sinks, tree=tree)
    ctx.sync()
    check_attend(Sees(pair.ref, masks), host(out), table, lens, starts, host(q), dim ** -0.5, dtype, window=window, sinks=sinks)
    again = torch.empty_like(q)
    ctx.attention(pair.gpu, q, again, b, dim ** -0.5, window=window, sinks=sinks, tree=tree)
    ctx.sync()
    assert torch.equal(out, again)
    return pair, table, starts, q, out, b


SHAPES = [(16, 64, 2, 1), (32, 96, 1, 4), (64, 128, 2, 4), (128, 256, 1, 3), (64, 64, 1, 7), (16, 128, 1, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,dim,heads,group", SHAPES)
@pytest.mark.parametrize("window,sinks", [(1, 1), (40, 4), (64, 64), (100, 200), (300, 1000)])
def test_sinks_single_tokens(palq, dtype, page, dim, heads, group, window, sinks):
    from paper_2208_01944_amd import palq as P
    say("sinks single", dtype, page, dim, heads, group, window, sinks)
    run_case(P, palq, page + dim, dtype, page, dim, heads, group, [1, 0, 2, 15, 16, 17, 63, 64, 65, 130, 257, 700],
             [1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1, 1], window, sinks)


@pytest.mark.parametrize("dtype,page,dim,heads,group,lens,new,window,sinks", [
    ("bf16", 64, 128, 1, 4, [5, 33, 100], [5, 33, 70], 17, 3),
    ("f16", 16, 64, 2, 1, [270, 1, 129], [70, 1, 64], 30, 70),
    ("bf16", 32, 96, 1, 2, [290, 40], [90, 13], 7, 5),
    ("f16", 64, 128, 1, 1, [400, 150], [130, 150], 64, 128),
    ("bf16", 128, 256, 1, 2, [440, 9], [40, 9], 100, 1),
    ("f16", 64, 64, 1, 3, [3, 10], [9, 20], 2, 1),         # more rows than tokens
    ("bf16", 16, 128, 2, 2, [550, 1077], [31, 66], 200, 33),
])
def test_sinks_many_rows(palq, dtype, page, dim, heads, group, lens, new, window, sinks):
    from paper_2208_01944_amd import palq as P
    say("sinks rows", dtype, page, dim, heads, group, lens, new, window, sinks)
    run_case(P, palq, page * 3 + dim, dtype, page, dim, heads, group, lens, new, window, sinks)


# enough rows for the 128-row kernel: more than 768 blocks of 32 rows (16 for heads of 256)
TILES = [
    ("bf16", 64, 128, 16, 2, [128, 350, 131, 300, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], None, ()),
    ("f16", 16, 64, 16, 2, [128, 150, 131, 300, 129, 500, 140], [128, 40, 131, 100, 1, 64, 120], None, ()),
    ("bf16", 32, 96, 16, 2, [70, 150, 0, 1, 129, 64, 291], [131, 40, 5, 100, 1, 64, 120], None, ()),
    ("f16", 128, 256, 8, 1, [300, 150, 131, 20, 129, 64, 65, 191], [200, 40, 131, 70, 1, 64, 0, 120], None, ()),
    ("bf16", 64, 64, 16, 3, [160, 100, 130, 61, 1200], [100, 100, 110, 100, 90], 5000, ()),
    ("f16", 16, 128, 16, 3, [1300, 100, 130, 700, 200], [60, 100, 20, 31, 100], 4000, ()),
    ("bf16", 16, 128, 16, 2, [128, 150, 131, 170, 129, 400, 140], [128, 40, 131, 100, 1, 64, 120], None, ((0, 0), (1, 3), (5, 12))),
    ("bf16", 16, 256, 8, 1, [300, 150, 131, 20, 129, 64, 65, 191], [200, 40, 131, 70, 1, 64, 0, 120], None, ((1, 0),)),
]


@pytest.mark.parametrize("dtype,page,dim,heads,group,lens,new,max_len,missing", TILES)
@pytest.mark.parametrize("window,sinks", [(33, 5), (100, 64)])
def test_sinks_tile_kernel(palq, dtype, page, dim, heads, group, lens, new, max_len, missing, window, sinks):
    from paper_2208_01944_amd import palq as P
    say("sinks tiles", dtype, page, dim, heads, group, lens, new, max_len, window, sinks)
    run_case(P, palq, page + dim, dtype, page, dim, heads, group, lens, new, window, sinks, max_len=max_len, missing=missing)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,dim,heads,group", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 0), (50, 3), (5000, 9)])
def test_tree(palq, dtype, page, dim, heads, group, window, sinks):
    """Any masks, rows that see nothing among them; drafts that end inside a page, drafts alone, without a bit."""
    from paper_2208_01944_amd import palq as P
    say("tree", dtype, page, dim, heads, group, window, sinks)
    lens, new = [1, 0, 7, 15, 33, 64, 200, 700, 130], [1, 3, 7, 0, 12, 33, 5, 25, 66]
    g = np.random.default_rng(page)
    starts = cumsum(new)
    masks = random_masks(g, lens, starts, 1)
    masks[starts[2]:starts[2] + 3] = 0
    masks[starts[7] + 1] = 0
    run_case(P, palq, page + dim, dtype, page, dim, heads, group, lens, new, window, sinks, 1, masks)


@pytest.mark.parametrize("words,new,lens", [(2, [100, 3], [400, 90]), (3, [130, 192], [131, 1000]), (16, [40, 90], [300, 95]), (1, [100, 70], [300, 70])])
def test_tree_words(palq, words, new, lens):
    from paper_2208_01944_amd import palq as P
    say("tree words", words, new, lens)
    run_case(P, palq, words, "bf16", 32, 128, 1, 2, lens, new, 60, 4, words)
    run_case(P, palq, words, "f16", 64, 64, 1, 3, lens, new, 0, 0, words)


@pytest.mark.parametrize("dtype,page,dim,heads,group,lens,new,max_len,missing", TILES)
@pytest.mark.parametrize("window,sinks,words", [(0, 0, 3), (90, 7, 2)])
def test_tree_tile_kernel(palq, dtype, page, dim, heads, group, lens, new, max_len, missing, window, sinks, words):
    from paper_2208_01944_amd import palq as P
    say("tree tiles", dtype, page, dim, heads, group, lens, new, max_len, window, sinks, words)
    run_case(P, palq, page + dim, dtype, page, dim, heads, group, lens, new, window, sinks, words, max_len=max_len, missing=missing)


@pytest.mark.parametrize("page,dim,heads,group,lens,new", [(64, 128, 2, 4, [5, 33, 100, 900], [5, 33, 60, 17]),
                                                          (16, 64, 16, 2, [128, 350, 131, 300, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120])])
def test_tree_of_chains_is_plain_attention(palq, page, dim, heads, group, lens, new):
    """Masks in the tokens' order: plain attention's outputs, within the bound.  Sinks without a window: the same bits."""
    import torch
    from paper_2208_01944_amd import palq as P
    words = -(-max(new) // 64)
    starts = cumsum(new)
    pair, table, starts, q, out, b = run_case(P, palq, 5, "bf16", page, dim, heads, group, lens, new, 0, 0, words, chains(starts, words))
    check_attend(pair, host(out), table, lens, starts, host(q), dim ** -0.5, "bf16")
    plain = torch.empty_like(q)
    palq.attention(pair.gpu, q, plain, b, dim ** -0.5)
    palq.attention(pair.gpu, q, out, b, dim ** -0.5, sinks=7)
    palq.sync()
    assert torch.equal(out, plain)


@pytest.mark.parametrize("words,window", [(0, 100), (1, 100), (1, 0)])
@pytest.mark.parametrize("rows", [1, 5, 20])
def test_long(palq, rows, words, window):
    """Thousands of tokens in parts that are joined."""
    from paper_2208_01944_amd import palq as P
    say("long", rows, words, window)
    window = window and 3000
    run_case(P, palq, rows, "bf16", 32, 64, 1, 2, [9000, 4100, 1], [rows, rows, 1], window, 700 if window else 0, words, max_len=16000)


def test_not_finite_outside_the_sight(palq):
    """Blocks with NaN or inf scales between sinks and window, behind the draft and under tokens that no bit names: seen by no
    row, they change nothing; those that a row sees make it NaN, and no other."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(21)
    page, dim, lens, new = 16, 64, [300, 180], [4, 20]
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, 1, page, dim)
    pair.fill(g, table, lens, 0.5)
    for block in range(3, 10):  # tokens 48 to 159 of request 0: past sinks of 40, before a window of 100
        pair.ref.ks[table[0][block]], pair.ref.vs[table[0][block]] = np.nan, np.inf
    pair.ref.vs[table[1][11]] = np.nan  # tokens 176 to 179 of request 1: its new tokens 16 to 19
    for n in ("k_scale", "v_scale"):
        getattr(pair.gpu, n).copy_(dev(pair.ref.ks if n == "k_scale" else pair.ref.vs))
    starts = cumsum(new)
    masks = chains(starts, 1)
    masks[starts[1]:] &= np.uint64(0xffff)  # (as first written: nobody sees the last four)
    q = dev(g.standard_normal((24, 2, dim)), "bf16")
    out = torch.empty_like(q)
    b = pair.batch(table, lens, starts)
    palq.attention(pair.gpu, q, out, b, 0.125, window=100, sinks=40, tree=masks_dev(masks))
    palq.sync()
    assert torch.isfinite(out).all()
    check_attend(Sees(pair.ref, masks), host(out), table, lens, starts, host(q), 0.125, "bf16", window=100, sinks=40)
    masks[starts[1] + 3] |= np.uint64(1 << 17)
    palq.attention(pair.gpu, q, out, b, 0.125, window=100, sinks=40, tree=masks_dev(masks))
    palq.sync()
    bad = torch.isnan(out).all(-1).all(-1).cpu().numpy()
    assert bad[starts[1] + 3] and bad.sum() == 1
    palq.attention(pair.gpu, q[:4], out[:4], pair.batch(table[:1], lens[:1], starts[:2]), 0.125, window=100, sinks=40)
    palq.sync()
    assert torch.isfinite(out[:4]).all()


def test_wild_batches_stay_inside(palq):
    """Lengths past the table, starts that run backwards or outside, all bits set: nothing outside the tensors."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(5)
    table, pages = paged(g, [60, 60], 16)
    pair = Pair(P, pages, 1, 16, 64)
    pair.fill(g, table, [60, 60], 0.5)
    q = torch.randn(40, 2, 64, device="cuda").to(torch.bfloat16)
    tree = torch.full((40, 2), -1, dtype=torch.int64, device="cuda")
    for lens, starts in (([9, 9], [-5, 100, 7]), ([1 << 30, -4], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]),
                         ([2 ** 31 - 1, 2 ** 31 - 1], [0, 20, 40]), ([3, 2 ** 31 - 1], [-2 ** 31, 0, 60]), ([-9, 5], [0, 30, 40])):
        b = P.Batch(dev(np.int32(table)), dev(np.int32(lens)), dev(np.int32(starts)), 2 ** 31 - 1, 2 ** 31 - 1)
        for window, sinks in ((0, 0), (7, 3), (2 ** 31 - 1, 2 ** 31 - 1)):
            out = torch.empty_like(q)
            b.desc.max_new = 1 << 20
            palq.attention(pair.gpu, q, out, b, 0.1, window=window, sinks=sinks)
            palq.attention(pair.gpu, q, out, b, 0.1, window=window, sinks=sinks, tree=tree)
    palq.sync()


@pytest.mark.parametrize("scale", [-0.1, 0.0])
@pytest.mark.parametrize("words", [0, 1])
@pytest.mark.parametrize("page,dim,heads,group,lens,new", [(16, 64, 2, 2, [90, 300], [5, 20]), (64, 128, 2, 4, [90, 300], [12, 60]),
                                                          (32, 256, 1, 2, [200], [30]), (16, 128, 16, 2, [128, 350, 131, 300, 129, 200, 140],
                                                                                         [64, 40, 64, 60, 1, 64, 60]),
                                                          (32, 64, 16, 2, [128, 350, 131, 300, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120])])
def test_scales_of_scores_and_blocks(palq, page, dim, heads, group, lens, new, scale, words):
    """Negative and zero score scales, blocks of scales far apart and of 0, in every kernel."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("scales", page, dim, heads, group, scale, words)
    g = np.random.default_rng(dim + words)
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens, 2.0)
    pair.ref.ks[table[0][1]], pair.ref.vs[table[-1][0]] = 0, 0
    pair.upload()
    starts = cumsum(new)
    masks = random_masks(g, lens, starts, words) if words else None
    q = dev(g.standard_normal((starts[-1], heads * group, dim)) * 0.3, "bf16")
    out = torch.empty_like(q)
    palq.attention(pair.gpu, q, out, pair.batch(table, lens, starts), scale, window=50, sinks=5, tree=masks_dev(masks) if words else None)
    palq.sync()
    check_attend(Sees(pair.ref, masks), host(out), table, lens, starts, host(q), scale, "bf16", window=50, sinks=5)

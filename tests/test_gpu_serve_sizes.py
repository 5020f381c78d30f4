"""GPU checks of the 8-bit transformer operators over every page and head size that
they take, and at the edges of their ranges, against the numpy oracle."""
import numpy as np
import pytest

from oracle import serve as S  # noqa: F401
from tests.test_gpu_serve import Pair, attend_case, check_attend, cumsum, dev, host, paged, say, tdt  # noqa: F401

pytestmark = pytest.mark.gpu

PAIRS = [(page, dim) for page in (16, 32, 64, 128) for dim in (64, 96, 128, 256)]


@pytest.mark.parametrize("page,dim", PAIRS)
def test_append_and_read_every_size(palq, page, dim):
    """Whole blocks, parts of blocks and single tokens, new and behind others, in every page and head size: codes and scales
    equal to the oracle's, values that grow so that old codes are rescaled."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("append sizes", page, dim)
    g = np.random.default_rng(page * 7 + dim)
    heads, steps = 2, [[page, 1, 3 * page // 4, 2 * page + 3], [1, page - 1, page // 4 + 1, page], [page + 2, 3, 1, page - 5]]
    final = np.sum(steps, 0)
    table, pages = paged(g, final.tolist(), page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, final)
    lens = np.zeros(4, int)
    for i, new in enumerate(steps):
        lens = lens + new
        starts = cumsum(new)
        k, v = (dev(g.standard_normal((starts[-1], heads, dim)) * np.exp(g.standard_normal((starts[-1], heads, dim)) + i), "bf16")
                for _ in range(2))
        pair.ref.append(table, lens.tolist(), starts, host(k), host(v))
        palq.cache_append(pair.gpu, k, v, pair.batch(table, lens.tolist(), starts))
        palq.sync()
        pair.check(table, lens.tolist())
    starts = cumsum(lens.tolist())
    k, v = torch.zeros(starts[-1], heads, dim, device="cuda"), torch.zeros(starts[-1], heads, dim, device="cuda")
    palq.cache_read(pair.gpu, k, v, pair.batch(table, lens.tolist(), starts))
    palq.sync()
    rk, rv = pair.ref.read(table, lens.tolist(), starts)
    np.testing.assert_array_equal(host(k), rk)
    np.testing.assert_array_equal(host(v), rv)


@pytest.mark.parametrize("page,dim", PAIRS)
def test_attention_tiles_every_size(palq, page, dim):
    """The 128-row kernel in every page and head size, rows and tokens that end inside tiles."""
    from paper_2208_01944_amd import palq as P
    say("attention tiles, sizes", page, dim)
    lens, new, heads, group = [128, 150, 131, 260, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120], 16, 2
    assert -(-max(new) * group // (16 if dim == 256 else 32)) * heads * len(lens) > 768
    for causal, window in ((True, 0), (True, 70), (False, 0)):
        attend_case(P, palq, page * 5 + dim, "bf16", page, dim, heads, group, lens, new, causal, window)


@pytest.mark.parametrize("page,dim", PAIRS)
def test_attention_rows_every_size(palq, page, dim):
    """The kernels of 16 and 32 rows in every page and head size."""
    from paper_2208_01944_amd import palq as P
    say("attention rows, sizes", page, dim)
    for lens, new, group, window in (([1, 130, 64, 300], [1, 1, 1, 1], 4, 0), ([9, 130, 200], [9, 11, 5], 3, 50)):
        attend_case(P, palq, page * 3 + dim, "f16", page, dim, 2, group, lens, new, True, window)


# lens, rows of the request, bounds: the position of its first row in the tensors, and how many rows are in both bounds
LEFT_OUT = [
    ("one past the table", 33, (0, 1), {}, 32, 1),
    ("rows past the table", 34, (0, 3), {}, 31, 3),
    ("past max_len", 23, (0, 5), dict(max_len=20), 18, 5),
    ("rows past max_new", 30, (0, 5), dict(max_new=3), 25, 3),
    ("rows past the tensors", 30, (0, 9), dict(max_new=9), 21, 6),
    ("starts below 0", 30, (-2, 3), dict(max_new=5), 27, 3),
    ("more rows than tokens", 2, (0, 5), {}, -3, 5),
]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("what,length,rows,bounds,pos,n", LEFT_OUT, ids=[c[0] for c in LEFT_OUT])
def test_rows_left_out_move_no_others(palq, what, length, rows, bounds, pos, n, dim):
    """Rows and tokens past the bounds are left out, and the others keep their positions: append, read and attention
    of a request beside an ordinary one, six rows in the tensors."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("left out", what, dim)
    g = np.random.default_rng(length)
    page, heads, tokens = 16, 2, 6
    table, room = np.int32([[3, 1]]), 32
    top = min(room, bounds.get("max_len", room), length)  # its tokens
    pair = Pair(P, 4, heads, page, dim)
    pair.fill(g, table, None)
    b = P.Batch(dev(table), dev(np.int32([length])), dev(np.int32(rows)), bounds.get("max_new", rows[1] - rows[0]), bounds.get("max_len", 64))
    x, y = (g.standard_normal((tokens, heads, dim)).astype(np.float32) for _ in range(2))
    # what is left: tensor row i at position first + i, for i in [0, n), of which those in [0, top) have a place
    first, end = pos - rows[0] if rows[0] > 0 else pos, min(pos + n, top)
    live = [i for i in range(n) if 0 <= first + i < end]
    if live:
        part = slice(live[0], live[-1] + 1)
        pair.ref.append(table, [first + live[-1] + 1], [0, len(live)], x[part], y[part])
    before = [t.clone() for t in (pair.gpu.k, pair.gpu.v, pair.gpu.k_scale, pair.gpu.v_scale)]
    palq.cache_append(pair.gpu, dev(x), dev(y), b)
    palq.sync()
    done = first + live[-1] + 1 if live else top
    pair.check(table, [done])
    for t, was in zip((pair.gpu.k, pair.gpu.v, pair.gpu.k_scale, pair.gpu.v_scale), before):
        assert torch.equal(t[[0, 2]], was[[0, 2]])
        if not live:
            assert torch.equal(t, was)
    pair.fill(g, table, None)
    k, v = torch.full((tokens, heads, dim), 5.0, device="cuda"), torch.full((tokens, heads, dim), 5.0, device="cuda")
    palq.cache_read(pair.gpu, k, v, b)
    palq.sync()
    for out, which in ((k, "k"), (v, "v")):
        want = np.full((tokens, heads, dim), 5.0, np.float32)
        for h in range(heads):
            vals = pair.ref.values(table, 0, top, h, which)[0]
            for i in live:
                want[i, h] = vals[first + i]
        np.testing.assert_array_equal(host(out), want)
    # attention: each row alone, as the last of a request that ends with it (the oracle's table without what is past `top`)
    for causal, window in ((True, 0), (True, 4), (False, 0)):
        q = dev(g.standard_normal((tokens, heads * 2, dim)), "f16")
        out = torch.full_like(q, 3.0)
        palq.attention(pair.gpu, q, out, b, 0.125, causal=causal, window=window)
        palq.sync()
        assert (host(out[n:]) == 3).all()
        for i in range(n):
            p = first + i
            if causal and p < 0:
                assert (host(out[i]) == 0).all()
                continue
            sees = [j for j in range(top) if not causal or (j <= p and (not window or j > p - window))]
            if not sees:
                assert (host(out[i]) == 0).all()
                continue
            # the same tokens, all seen by one row that ends with the last of them
            span = sees[-1] + 1
            check_attend(pair, host(out[i:i + 1]), table, [span], [0, 1], host(q[i:i + 1]), 0.125, "f16", causal=True,
                         window=span - sees[0])


@pytest.mark.parametrize("max_new,max_len", [(100, None), (None, 144), (90, 128)])
def test_rows_left_out_of_tiles(palq, max_new, max_len):
    """The same on the 128-row kernel: rows past max_new stay as they are, tokens past max_len are not seen, positions stay."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("left out of tiles", max_new, max_len)
    g = np.random.default_rng(5)
    page, dim, heads, lens, new = 16, 64, 16, [128, 150, 131, 260, 129, 200, 140], [128, 40, 131, 100, 1, 64, 120]
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens)
    starts = cumsum(new)
    q = dev(g.standard_normal((starts[-1], 2 * heads, dim)) * 1.5, "bf16")
    b = pair.batch(table, lens, starts, max_new=max_new, max_len=max_len)
    seen = table.copy()
    if max_len:
        seen[:, max_len // page:] = -1
    for causal, window in ((True, 0), (True, 70), (False, 0)):
        out = torch.full_like(q, 3.0)
        palq.attention(pair.gpu, q, out, b, 0.125, causal=causal, window=window)
        palq.sync()
        got = host(out)
        # the rows left out: replaced by what the oracle says, once they are seen to be as they were
        left = np.zeros(starts[-1], bool)
        for r, n in enumerate(new):
            left[starts[r] + min(n, max_new or n):starts[r + 1]] = True
        assert (got[left] == 3).all() and left.any() == bool(max_new)
        got[left] = pair.ref.attend(seen, lens, starts, host(q), 0.125, causal, window)[0][left]
        check_attend(pair, got, seen, lens, starts, host(q), 0.125, "bf16", causal=causal, window=window)


@pytest.mark.parametrize("window", [1, 5, (1 << 31) - 1, (1 << 31) - 2, (1 << 31) - 40])
def test_window_of_any_size_before_the_first_token(palq, window):
    """More rows than tokens under a window: the rows before position 0 see nothing and take nothing from the others,
    however large the window is (16, 32 and 128 rows a workgroup)."""
    from paper_2208_01944_amd import palq as P
    say("window", window)
    for heads, group, lens, new in ((1, 1, [3, 30], [9, 5]), (2, 3, [10, 50], [33, 20]), (16, 4, [100, 30, 7, 60], [130, 100, 90, 60])):
        attend_case(P, palq, heads, "bf16", 16, 64, heads, group, lens, new, True, window)


@pytest.mark.parametrize("length", [(1 << 31) - 1024 - 5, (1 << 31) - 1024, (1 << 31) - 900, (1 << 31) - 1])
@pytest.mark.parametrize("heads,group,new", [(2, 2, 3), (16, 4, 400)])
def test_lengths_near_the_limit(palq, length, heads, group, new):
    """Append, read and attention (rows and tiles) of the last positions next to 2^31 - 1024 tokens, and past it, where
    tokens are left out: as the same rows and tokens 2^31 - 2048 places earlier."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("long", length, heads)
    g = np.random.default_rng(3)
    page, dim, room, base = 128, 64, 1 << 24, (1 << 31) - 2048
    near = np.arange(1, 17, dtype=np.int32)[None]  # the pages of the last 2048 tokens
    pair = Pair(P, 17, heads, page, dim)
    pair.fill(g, near, None)
    table = torch.zeros(1, room, dtype=torch.int32, device="cuda")
    table[:, -16:] = dev(near)
    starts, short, top = [0, new], length - base, 1024
    b = P.Batch(table, dev(np.int32([length])), dev(np.int32(starts)), new, (1 << 31) - 1)
    x, y = (g.standard_normal((new, heads, dim)).astype(np.float32) for _ in range(2))
    left = max(0, min(top, short) - (short - new))  # rows with a place below the limit
    if left:
        pair.ref.append(near, [short - new + left], [0, left], x[:left], y[:left])
    palq.cache_append(pair.gpu, dev(x), dev(y), b)
    palq.sync()
    pair.check(near, [min(top, short)])
    k, v = torch.full((new, heads, dim), 5.0, device="cuda"), torch.full((new, heads, dim), 5.0, device="cuda")
    palq.cache_read(pair.gpu, k, v, b)
    palq.sync()
    assert (host(k[left:]) == 5).all() and (host(v[left:]) == 5).all()
    if left:
        rk, rv = pair.ref.read(near, [short - new + left], [0, left])
        np.testing.assert_array_equal(host(k[:left]), rk)
        np.testing.assert_array_equal(host(v[:left]), rv)
    seen = near.copy()
    seen[:, top // page:] = -1
    q = dev(g.standard_normal((new, heads * group, dim)), "bf16")
    for window in (1, 300):
        out = torch.full_like(q, 3.0)
        palq.attention(pair.gpu, q, out, b, 0.125, window=window)
        palq.sync()
        check_attend(pair, host(out), seen, [short], starts, host(q), 0.125, "bf16", causal=True, window=window)


# ------------------------------------------------------------------ sizes of launches
def test_quantize_rows_past_one_launch(palq):
    """More rows than one launch has waves for."""
    import torch
    rows = (1 << 26) + 5
    x = torch.randn(rows, 1, device="cuda", dtype=torch.float16)
    x[::1000] = 0
    codes, scales = torch.full((rows, 1), 99, dtype=torch.int8, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    palq.quantize_rows(x, codes, scales)
    palq.sync()
    v = x.cpu().numpy()[:, 0].astype(np.float32)
    s = np.maximum(np.abs(v) * S.C127, S.FLOOR)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy()[:, 0], np.clip(np.rint(v * (np.float32(1) / s)), -127, 127).astype(np.int8))


def test_linear_codes_past_one_grid(palq):
    """More codes to lay out than the grid has waves: each takes several pieces."""
    import torch
    from paper_2208_01944_amd import palq as P
    rows, n_in, n_out = 4200, 65500, 20
    x = torch.randint(-128, 128, (rows, n_in), dtype=torch.int8, device="cuda")
    w = torch.randint(-128, 128, (n_out, n_in), dtype=torch.int8, device="cuda")
    lin = P.Linear(palq, w, torch.ones(n_out, device="cuda"), max_rows=rows)
    y = torch.empty(rows, n_out, device="cuda")
    lin.run(x, y, x_scale=torch.ones(rows, device="cuda"))
    palq.sync()
    want = torch.cat([torch.mm(part.double(), w.double().t().contiguous()) for part in x.split(600)]).float()  # (sums below 2^53)
    assert torch.equal(y, want)


def test_attention_bounds_past_one_launch(palq):
    """A bound for a request's rows so loose that its workgroups, nearly all of them without rows, are more than one launch
    takes: the same results as with the close bound, for wide and narrow pages."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(8)
    heads, dim, requests, new = 64, 64, 600, 100
    for page in (16, 64):
        per = -(-(new + 30) // page)
        table, pages = g.permutation(requests * per).astype(np.int32).reshape(requests, per), requests * per
        cache = P.Cache(*(torch.randint(-127, 128, s, dtype=torch.int8, device="cuda") for s in ((pages, heads, page, dim), (pages, heads, dim, page))),
                        torch.rand(pages, heads, device="cuda") / 64, torch.rand(pages, heads, device="cuda") / 64)
        lens, starts = g.integers(1, new + 30, requests).astype(np.int32), (np.arange(requests + 1) * new).astype(np.int32)
        starts[1:] -= np.cumsum(g.integers(0, 2, requests)).astype(np.int32)
        tokens = int(starts[-1])
        assert -(-tokens // 128) * heads * requests > 1 << 24
        q = torch.randn(tokens, heads, dim, device="cuda", dtype=torch.bfloat16)
        outs = []
        for max_new in (new, 1 << 29):
            out = torch.full_like(q, 3.0)
            palq.attention(cache, q, out, P.Batch(dev(table), dev(lens), dev(starts), max_new, per * page), 0.125)
            palq.sync()
            outs.append(out)
        assert torch.equal(*outs) and torch.isfinite(outs[0]).all() and not (outs[0] == 3.0).all(2).any()


def test_cache_bounds_past_one_launch(palq):
    """Append and read of three tokens under bounds of 2^31 - 1 rows and tokens and a table of 2^24 pages."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(9)
    page, dim, room, length, new = 16, 64, 1 << 24, 35, 3
    pair = Pair(P, 4, 2, page, dim)
    small = np.int32([[2, 0, 3]])
    pair.fill(g, small, None)
    table = torch.full((1, room), -1, dtype=torch.int32, device="cuda")
    table[:, :3] = dev(small)
    b = P.Batch(table, dev(np.int32([length])), dev(np.int32([0, new])), (1 << 31) - 1, (1 << 31) - 1)
    k, v = (g.standard_normal((new, 2, dim)).astype(np.float32) for _ in range(2))
    pair.ref.append(small, [length], [0, new], k, v)
    palq.cache_append(pair.gpu, dev(k), dev(v), b)
    ok, ov = torch.zeros(new, 2, dim, device="cuda"), torch.zeros(new, 2, dim, device="cuda")
    palq.cache_read(pair.gpu, ok, ov, b)
    palq.sync()
    pair.check(small, [length])
    rk, rv = pair.ref.read(small, [length], [0, new])
    np.testing.assert_array_equal(host(ok), rk)
    np.testing.assert_array_equal(host(ov), rv)

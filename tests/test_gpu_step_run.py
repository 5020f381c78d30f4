"""GPU checks of a generation step's operators as they are run: together, captured and replayed, on
several streams, at offsets past 32 bits, and with nothing to do."""
import numpy as np
import pytest

from oracle import step as S
from tests.test_gpu_serve import Pair, check_attend, cumsum, dev, host, paged
from tests.test_gpu_sight import Sees
from tests.test_gpu_step import batch_of, check_rotated, check_scores, freqs, masks_dev, random_masks, score

pytestmark = pytest.mark.gpu


class Step:
    """A step of drafted tokens over one layer: product, norms and rotation in place, append, attention of the tree, a
    second product to logits, their log probabilities."""

    def __init__(self, P, stream, seed, lens=(40, 5000, 300), new=(7, 5, 12), page=32, heads=2, group=2, dim=64, vocab=50001, window=0, sinks=0):
        import torch
        g = np.random.default_rng(seed)
        self.torch, self.stream, self.ctx = torch, stream, P.Context(0, stream=stream.cuda_stream)
        self.dim, self.heads, self.group, self.window, self.sinks = dim, heads, group, window, sinks
        table, pages = paged(g, list(lens), page)
        starts = cumsum(list(new))
        t = starts[-1]
        n = heads * (group + 2) * dim
        w = lambda a, b: dev(g.integers(-127, 128, (a, b)).astype(np.int8))  # noqa: E731
        self.lin = P.Linear(self.ctx, w(n, 96), torch.full((n,), 1e-3, device="cuda"), max_rows=t)
        self.head = P.Linear(self.ctx, w(vocab, heads * group * dim), torch.full((vocab,), 1e-3, device="cuda"), max_rows=t)
        self.pair = Pair(P, pages, heads, page, dim)
        self.pair.fill(g, table, list(lens))
        c = self.pair.gpu
        self.state = (c.k, c.v, c.k_scale, c.v_scale)
        self.start = [x.clone() for x in self.state]
        self.b = self.pair.batch(table, list(lens), starts)
        self.rot = P.Rotation(self.ctx, freqs(dim // 2))
        self.tree = masks_dev(random_masks(g, lens, starts, 1))
        self.weight = torch.rand(dim, device="cuda") + 0.5
        e = lambda *s, d=torch.bfloat16: torch.empty(*s, dtype=d, device="cuda")  # noqa: E731
        self.x, self.qkv, self.out, self.logits = e(t, 96), e(t, n), e(t, heads * group, dim), e(t, vocab)
        self.ids = torch.randint(0, vocab, (t, 2), dtype=torch.int32, device="cuda")
        self.logp, self.ent, self.top, self.top_ids = e(t, 2, d=torch.float32), e(t, d=torch.float32), e(t, 9, d=torch.float32), e(t, 9, d=torch.int32)
        torch.cuda.synchronize()

    def __call__(self):
        c = self.ctx
        self.lin.run(self.x, self.qkv)
        q, k, v = self.qkv.unflatten(1, (self.heads * (self.group + 2), self.dim)).split([self.heads * self.group, self.heads, self.heads], 1)
        c.norm_rotate(self.b, q, q, k, k, q_weight=self.weight, eps=1e-6, rotation=self.rot, tree=self.tree)
        c.cache_append(self.pair.gpu, k, v, self.b)
        c.attention(self.pair.gpu, q, self.out, self.b, 0.125, window=self.window, sinks=self.sinks, tree=self.tree)
        self.head.run(self.out.flatten(1), self.logits)
        c.log_probs(self.logits, self.ids, self.logp, entropy=self.ent, top_ids=self.top_ids, top=self.top)

    def reset(self, x):
        for t, s in zip(self.state, self.start):
            t.copy_(s)
        self.x.copy_(x)
        self.torch.cuda.synchronize()

    def results(self):
        return [t.clone() for t in (self.qkv, self.out, self.logits, self.logp, self.ent, self.top, self.top_ids, *self.state)]

    def inputs(self, n, seed):
        g = np.random.default_rng(seed)
        return [dev(g.standard_normal(tuple(self.x.shape)), "bf16") for _ in range(n)]


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5)])
def test_step_in_a_graph(palq, window, sinks):
    """Captured and replayed with new inputs, other work between the replays: every replay equals the eager calls, whose log
    probabilities are the oracle's."""
    import torch
    from paper_2208_01944_amd import palq as P
    side = torch.cuda.Stream()
    s = Step(P, side, 80, window=window, sinks=sinks)
    xs, want = s.inputs(3, 81), []
    for x in xs:
        s.reset(x)
        s()
        s.ctx.sync()
        want.append(s.results())
    check_scores(host(s.logits), 1.0, s.ids.cpu().numpy(), (host(s.logp), host(s.ent), s.top_ids.cpu().numpy(), host(s.top)), 9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s()
    for x, w in zip(xs + xs, want + want):
        s.reset(x)
        _ = torch.randn(1000, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(s.results(), w))


def test_steps_on_two_streams(palq):
    """Two contexts, their graphs replayed at the same time and their eager calls between: each has a workspace of its own."""
    import torch
    from paper_2208_01944_amd import palq as P
    steps = [Step(P, torch.cuda.Stream(), 90), Step(P, torch.cuda.Stream(), 91, lens=(9000, 64, 2000), new=(20, 20, 1), window=3000, sinks=4)]
    xs = [s.inputs(1, 92 + i)[0] for i, s in enumerate(steps)]
    want, graphs = [], []
    for s, x in zip(steps, xs):
        s.reset(x)
        s()
        s.ctx.sync()
        want.append(s.results())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s.stream):
            s()
    for turn in range(4):
        for s, x in zip(steps, xs):
            s.reset(x)
        for i, (s, g) in enumerate(zip(steps, graphs)):
            with torch.cuda.stream(s.stream):
                if (turn + i) % 2:
                    s()
                else:
                    g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(s.results(), w))


def test_workspace_in_a_capture(palq):
    """Rows that are split need workspace: refused in a capture that would have to allocate it, taken once it is there; a later,
    larger call leaves the graph its own."""
    import torch
    from paper_2208_01944_amd import palq as P
    side = torch.cuda.Stream()
    ctx = P.Context(0, stream=side.cuda_stream)
    x = dev(np.random.default_rng(3).standard_normal((2, 100000)), "bf16")
    ids = torch.tensor([[5], [99999]], dtype=torch.int32, device="cuda")
    out, y = torch.empty(2, 1, device="cuda"), torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(P.PalqError) as e:
            ctx.log_probs(x, ids, out)
        y.add_(1.0)
    assert e.value.status == P.ERR_NOMEM
    graph.replay()
    torch.cuda.synchronize()
    assert (y.cpu() == 1).all()
    ctx.log_probs(x, ids, out)
    ctx.sync()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.log_probs(x, ids, out)
    big = torch.randn(40, 100000, device="cuda")
    for _ in range(3):
        t = torch.empty(40, 64, dtype=torch.int32, device="cuda"), torch.empty(40, 64, device="cuda")
        torch.cuda.synchronize()
        ctx.log_probs(big, None, None, top_ids=t[0], top=t[1])
        ctx.sync()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_offsets_past_32_bits(palq):
    """Rows 2^30 elements and more apart."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(5)
    room = torch.empty(5 << 30, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((5, 3001), (1 << 30, 1))
    x.copy_(dev(g.standard_normal((5, 3001)), "bf16"))
    ids = g.integers(0, 3001, (5, 2))
    check_scores(host(x), 1.0, ids, score(palq, x, ids, 7), 7)
    q = room.as_strided((5, 2, 64), (1 << 30, 1 << 28, 1))
    q.copy_(dev(g.standard_normal((5, 2, 64)), "bf16"))
    want = host(q)
    palq.norm_rotate(batch_of([9], [0, 5]), q, q, eps=1e-6, rotation=P.Rotation(palq, freqs(32)))
    palq.sync()
    check_rotated(host(q), want, np.arange(4, 9), "bf16", freq=freqs(32), eps=1e-6)


def test_large_cache_offsets(palq):
    """Pages past 2^31 bytes: sinks on one end of the pool, the window on the other, a tree across."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(64)
    page, dim, heads = 64, 128, 1
    pages = (1 << 31) // (page * dim) + 40
    cache = P.Cache(torch.empty(pages, heads, page, dim, dtype=torch.int8, device="cuda"),
                    torch.empty(pages, heads, dim, page, dtype=torch.int8, device="cuda"),
                    torch.ones(pages, heads, device="cuda"), torch.ones(pages, heads, device="cuda"))
    real = np.int32([[pages - 1, 2, 0, pages - 3], [pages - 2, 1, pages - 30, 4]])
    small, lens, new = np.int32([[0, 1, 2, 3], [4, 5, 6, 7]]), [250, 229], [250, 229]
    pair = Pair(P, 8, heads, page, dim)
    k, v = (g.standard_normal((479, heads, dim)).astype(np.float32) for _ in range(2))
    pair.ref.append(small, lens, cumsum(new), k, v)
    palq.cache_append(cache, dev(k), dev(v), P.Batch(dev(real), dev(np.int32(lens)), dev(np.int32(cumsum(new))), 250, 250))
    starts = [0, 9, 17]
    q = dev(g.standard_normal((17, 2, dim)), "bf16")
    out = torch.empty_like(q)
    b = P.Batch(dev(real), dev(np.int32(lens)), dev(np.int32(starts)), 9, 250)
    for masks in (None, random_masks(g, lens, starts, 1)):
        palq.attention(cache, q, out, b, 0.09, window=50, sinks=70, tree=None if masks is None else masks_dev(masks))
        palq.sync()
        check_attend(Sees(pair.ref, masks), host(out), small, lens, starts, host(q), 0.09, "bf16", window=50, sinks=70)


def test_strided_heads_and_rows_left_out(palq):
    """Queries and outputs as parts of wider tensors; rows past max_new and between requests stay as they are."""
    import torch
    from paper_2208_01944_amd import palq as P
    g = np.random.default_rng(66)
    page, dim, heads, group, lens, starts = 16, 96, 2, 3, [90, 200], [2, 9, 30]
    table, pages = paged(g, lens, page)
    pair = Pair(P, pages, heads, page, dim)
    pair.fill(g, table, lens)
    wide = dev(g.standard_normal((33, heads * group + 3, dim + 8)), "f16")
    q = wide[:, 2:2 + heads * group, 5:5 + dim]
    room = torch.full((33, heads * group + 1, dim + 2), 7.0, dtype=torch.float16, device="cuda")
    out = room[:, 1:, 1:1 + dim]
    masks = random_masks(g, lens, [0, 33], 1)
    b = P.Batch(dev(table), dev(np.int32(lens)), dev(np.int32(starts)), 20, 200)
    palq.attention(pair.gpu, q, out, b, 0.1, window=60, sinks=3, tree=masks_dev(masks))
    palq.sync()
    got = host(out)
    live = np.zeros(33, bool)
    live[2:9] = live[9:29] = True  # (row 29 is past max_new)
    assert (got[~live] == 7).all() and (host(room[:, 0]) == 7).all() and (host(room[..., 0]) == 7).all() and (host(room[..., -1]) == 7).all()
    # the oracle takes all 21 rows of the second request, as their positions and bits are
    rm, rstarts = masks[2:30], [0, 7, 28]
    ref = S.attend(pair.ref, table, lens, rstarts, host(q)[2:30], 0.1, 60, 3, rm)
    err = np.abs(got[2:29] - ref[0][:27])
    mass, reach = ref[1][:27], ref[2][:27]
    es = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -15  # (as check_attend)
    tol = mass * (2.0 ** -11 + 2 * es)[..., None] + (ref[3][:27] * 2.0 ** -25 * 127 * float(pair.ref.vs.max()))[..., None]
    assert (err <= tol + 2.0 ** -11 * (np.abs(ref[0][:27]) + tol) + 2.0 ** -25).all()


def test_empty_calls(palq):
    """No rows, no requests, no new tokens: no launch, no error."""
    import torch
    from paper_2208_01944_amd import palq as P
    c = P.Cache.empty(2, 1, 16, 64)
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    t = torch.empty(0, 1, dtype=torch.int64, device="cuda")
    for b in (P.Batch(z(2, 1), z(2), z(3), 0, 0), P.Batch(z(0, 1), z(0), z(1), 4, 4), P.Batch(z(1, 1), z(1), z(2), 4, 16)):
        palq.norm_rotate(b, e, e, eps=1e-6, tree=t)
        palq.attention(c, e, torch.empty_like(e), b, 1.0, window=3, sinks=1)
        palq.attention(c, e, torch.empty_like(e), b, 1.0, tree=t)
    palq.log_probs(torch.empty(0, 9, device="cuda"), z(0, 2), torch.empty(0, 2, device="cuda"))
    palq.sync()

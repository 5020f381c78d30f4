"""Generation with drafted tokens in 8 bits: a decoder whose heads are normed and
rotated by position, over paged 8-bit caches of which every other layer keeps a window
and the first tokens of a request; trees of drafted tokens are checked in one step by the
log probabilities of the decoder's head, and the branch that it agrees with is kept.

    python examples/draft_tree_int8.py [--layers 4] [--width 1024] [--steps 16]

Weights and drafts are random, so drafts are hardly ever right: what counts is the time of a
step.  Embedding, residual sums and the gate are plain torch.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2208_01944_amd import palq  # noqa: E402

EPS = 1e-6


def quantized(w):
    """fp32 [n_out, n_in] -> int8 codes and a scale for each channel."""
    s = w.abs().amax(1) / 127
    return (w / s[:, None]).round().to(torch.int8), s


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def masks(parents):
    """Masks of trees: parents[r][i] is the index of new token i's parent among the request's new tokens, or -1."""
    words = -(-max(len(p) for p in parents) // 64)
    rows = []
    for p in parents:
        sees = []
        for i, a in enumerate(p):
            sees.append((sees[a] if a >= 0 else 0) | 1 << i)
        rows += [[(s >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for s in sees]
    return torch.from_numpy(np.array(rows, dtype=np.uint64).view(np.int64)).cuda()


class Layer:
    NAMES = ("qkv", "out", "up", "down")

    def __init__(self, ctx, width, heads, kv_heads, dim, hidden, pages, page, max_rows, window, sinks, rotation, gen):
        self.ctx, self.heads, self.kv, self.dim, self.window, self.sinks, self.rotation = ctx, heads, kv_heads, dim, window, sinks, rotation
        shapes = dict(qkv=((heads + 2 * kv_heads) * dim, width), out=(width, heads * dim), up=(2 * hidden, width), down=(width, hidden))
        self.codes = {n: quantized(torch.randn(*shapes[n], generator=gen, device="cuda") * shapes[n][1] ** -0.5) for n in self.NAMES}
        self.lin = {n: palq.Linear(ctx, *self.codes[n], max_rows=max_rows) for n in self.NAMES}
        self.q_weight, self.k_weight = (1 + 0.1 * torch.randn(dim, generator=gen, device="cuda") for _ in range(2))
        self.cache = palq.Cache.empty(pages, kv_heads, page, dim)

    def product(self, name, x):
        y = torch.empty(x.shape[0], self.lin[name].n_out, dtype=torch.bfloat16, device="cuda")
        self.lin[name].run(x, y)
        return y

    def __call__(self, x, batch, tree):
        """x [tokens, width], the requests' new tokens; their keys and values stay at hand until it is known which are kept."""
        q, k, v = self.product("qkv", norm(x)).unflatten(1, (self.heads + 2 * self.kv, self.dim)).split([self.heads, self.kv, self.kv], 1)
        self.ctx.norm_rotate(batch, q, q, k, k, q_weight=self.q_weight, k_weight=self.k_weight, eps=EPS, rotation=self.rotation, tree=tree)
        self.ctx.cache_append(self.cache, k, v, batch)
        self.new = k, v
        o = torch.empty(x.shape[0], self.heads, self.dim, dtype=torch.bfloat16, device="cuda")
        self.ctx.attention(self.cache, q, o, batch, self.dim ** -0.5, window=self.window, sinks=self.sinks, tree=tree)
        x = x + self.product("out", o.flatten(1))
        a, b = self.product("up", norm(x)).chunk(2, 1)
        return x + self.product("down", (torch.nn.functional.silu(a.float()) * b.float()).to(torch.bfloat16))


class Session:
    """Requests with their page tables: prompts first, then trees of drafted tokens."""

    def __init__(self, prompts, room, layers=2, width=256, heads=4, kv_heads=2, dim=64, hidden=512, vocab=1000, page=16, window=24, sinks=4,
                 seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ctx = palq.Context(0)
        n, per = len(prompts), -(-(max(prompts) + room) // page)
        rows = max(sum(prompts), n * room)
        self.lens, self.vocab, self.pages, self.page = [0] * n, vocab, n * per, page
        self.table = torch.randperm(n * per, generator=gen, device="cuda").to(torch.int32).view(n, per)
        rotation = palq.Rotation(self.ctx, 10000.0 ** -(np.arange(dim // 2) / (dim // 2)))
        self.layers = [Layer(self.ctx, width, heads, kv_heads, dim, hidden, n * per, page, rows, window if i % 2 else 0, sinks if i % 2 else 0,
                             rotation, gen) for i in range(layers)]
        self.embedding = torch.randn(vocab, width, generator=gen, device="cuda").to(torch.bfloat16)
        self.codes = quantized(torch.randn(vocab, width, generator=gen, device="cuda") * width ** -0.5)
        self.head = palq.Linear(self.ctx, *self.codes, max_rows=rows)

    def run(self, tokens, new, tree=None):
        """Logits of `new` tokens of each request, which lie behind its present ones (they are cached, not yet counted)."""
        starts = [0]
        for t in new:
            starts.append(starts[-1] + t)
        lens = [a + b for a, b in zip(self.lens, new)]
        batch = palq.Batch(self.table, ints(lens), ints(starts), max(new), max(lens))
        x = self.embedding[tokens.long()]
        for layer in self.layers:
            x = layer(x, batch, tree)
        logits = torch.empty(len(tokens), self.vocab, dtype=torch.bfloat16, device="cuda")
        self.head.run(norm(x), logits)
        return logits

    def prompt(self, tokens, prompts):
        """The most probable token behind each prompt."""
        last = self.run(tokens, prompts)[torch.tensor(prompts).cumsum(0).cuda() - 1].contiguous()
        self.lens = list(prompts)
        return self.score(last, None)[1][:, 0]

    def score(self, logits, tokens):
        """Log probabilities of given tokens, and the most probable ones."""
        out = None if tokens is None else torch.empty(len(logits), 1, device="cuda")
        ids, top = torch.empty(len(logits), 5, dtype=torch.int32, device="cuda"), torch.empty(len(logits), 5, device="cuda")
        self.ctx.log_probs(logits, tokens, out, top_ids=ids, top=top)
        return out, ids

    def check(self, tokens, parents):
        """One step of trees: tokens int32 [sum of their sizes], node 0 of each its request's next token.  Keeps the branch that the
        decoder agrees with; returns the rows that were kept, the next tokens, and the log probability of every node's
        token given its parent."""
        new = [len(p) for p in parents]
        logits = self.run(tokens, new, masks(parents))
        starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        above = [starts[r] + max(a, 0) for r, p in enumerate(parents) for a in p]
        logp, _ = self.score(logits[torch.tensor(above, device="cuda")], tokens[:, None].contiguous())
        best = self.score(logits, None)[1][:, 0]
        said, drafted = best.cpu().tolist(), tokens.cpu().tolist()
        kept, following = [], []
        for r, p in enumerate(parents):
            at, rows = 0, [starts[r]]
            while True:
                children = [i for i, a in enumerate(p) if i and a == at and drafted[starts[r] + i] == said[starts[r] + at]]
                if not children:
                    break
                at = children[0]
                rows.append(starts[r] + at)
            kept.append(rows)
            following.append(said[rows[-1]])
        self.keep(kept)
        return kept, ints(following), logp

    def keep(self, kept):
        """Of the new tokens those rows, in order: appended again behind the present ones."""
        starts = [0]
        for rows in kept:
            starts.append(starts[-1] + len(rows))
        self.lens = [a + len(rows) for a, rows in zip(self.lens, kept)]
        batch = palq.Batch(self.table, ints(self.lens), ints(starts), max(map(len, kept)), max(self.lens))
        at = torch.tensor([i for rows in kept for i in rows], device="cuda")
        for layer in self.layers:
            k, v = layer.new
            self.ctx.cache_append(layer.cache, k[at], v[at], batch)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=16)
    args = ap.parse_args()
    prompts, nodes, vocab = [1000, 37, 512, 801, 1, 300, 640, 129], 25, 32000
    rng = np.random.default_rng(0)
    s = Session(prompts, nodes * (args.steps + 1), args.layers, args.width, args.width // 64, args.width // 256, 64, 4 * args.width, vocab, 64, 256)
    following = s.prompt(ints(rng.integers(0, vocab, sum(prompts)).tolist()), prompts)
    torch.cuda.synchronize()
    t, kept = time.perf_counter(), 0
    for _ in range(args.steps):
        parents = [[-1] + [int(rng.integers(0, i)) for i in range(1, nodes)] for _ in prompts]
        tokens = ints(rng.integers(0, vocab, nodes * len(prompts)).tolist())
        tokens[::nodes] = following
        rows, following, _ = s.check(tokens, parents)
        kept += sum(map(len, rows))
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / args.steps
    print(f"{len(prompts)} trees of {nodes} tokens a step: {t * 1e3:.2f} ms, {kept / args.steps:.1f} tokens kept")


if __name__ == "__main__":
    main()

"""The example of drafted trees against the same decoder in numpy (sums in 64 bits, bf16 where
the example rounds): prompts, a tree step, the branch that is kept, and the step after it."""
import os
import sys

import numpy as np
import pytest

from oracle import serve as S
from oracle import step as T
from tests.test_gpu_serve_example import bf16, norm

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Layer:
    def __init__(self, layer, pages, page, freq):
        self.w = {n: (c.cpu().numpy(), s.cpu().numpy()) for n, (c, s) in layer.codes.items()}
        self.qw, self.kw = layer.q_weight.cpu().numpy(), layer.k_weight.cpu().numpy()
        self.h, self.kv, self.d, self.window, self.sinks, self.freq = layer.heads, layer.kv, layer.dim, layer.window, layer.sinks, freq
        self.cache = S.Cache(pages, self.kv, page, self.d)

    def product(self, name, x):
        q, s = S.quantize_rows(x)
        return bf16(S.linear(q, s, *self.w[name]))

    def __call__(self, x, table, lens, starts, mask):
        t, h, kv, d = len(x), self.h, self.kv, self.d
        y = self.product("qkv", norm(x)).reshape(t, h + 2 * kv, d)
        pos = T.positions(lens, starts, mask)
        q, k = (bf16(T.norm_rotate(z, pos, self.freq, weight=w, eps=1e-6)[0]) for z, w in ((y[:, :h], self.qw), (y[:, h:h + kv], self.kw)))
        self.new = k, y[:, h + kv:]
        self.cache.append(table, lens, starts, *self.new)
        o = bf16(T.attend(self.cache, table, lens, starts, q, d ** -0.5, self.window, self.sinks, mask)[0])
        x = bf16(x + self.product("out", o.reshape(t, -1)))
        a, b = np.split(self.product("up", norm(x)), 2, 1)
        return bf16(x + self.product("down", bf16(a / (1 + np.exp(-a.astype(np.float64))) * b)))


def test_draft_tree_example():
    """Quantisation to 127 steps leaves about 1 % of noise in each product, and where the two sides round apart a code may
    fall on the other side of a step: at most that noise again.  Four products in each of two layers and the head: 1 %
    sqrt(18) = 4.2 % of the logits."""
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import draft_tree_int8 as E
    prompts, page = [39, 1, 50], 16
    s = E.Session(prompts, 40, page=page)
    table = s.table.cpu().numpy()
    freq = 10000.0 ** -(np.arange(32) / 32)
    ref = [Layer(layer, s.pages, page, freq) for layer in s.layers]
    embedding, head = s.embedding.float().cpu().numpy(), tuple(t.cpu().numpy() for t in s.codes)
    g = np.random.default_rng(4)

    def compare(what, tokens, new, lens, mask, logits):
        starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        x = embedding[tokens]
        for r in ref:
            x = r(x, table, [a + b for a, b in zip(lens, new)], starts, mask)
        q, sc = S.quantize_rows(norm(x))
        want = bf16(S.linear(q, sc, *head))
        err = np.linalg.norm(logits - want) / np.linalg.norm(want)
        print(what, "relative difference", err, flush=True)
        assert err < 0.05

    seen = []
    run = s.run
    s.run = lambda tokens, new, tree=None: seen.append(run(tokens, new, tree)) or seen[-1]
    tokens = g.integers(0, s.vocab, sum(prompts))
    following = s.prompt(E.ints(tokens.tolist()), prompts)
    compare("prompts", tokens, prompts, [0] * 3, None, seen[-1].float().cpu().numpy())
    for step in range(3):
        lens = list(s.lens)
        parents = [[-1, 0, 0, 1, 1, 2, 5], [-1, 0, 1, 2], [-1] + [0] * 5 + [3, 3]]
        new = [len(p) for p in parents]
        starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        tokens = g.integers(0, s.vocab, sum(new))
        tokens[starts[:-1]] = following.cpu().numpy()
        if step:  # a branch that is right: what the decoder says behind the first token, as one of its children
            probe = s.run(E.ints(tokens.tolist()), new, E.masks(parents)).float().cpu().numpy()
            s.keep([[a] for a in starts[:-1]])
            s.lens = list(lens)
            for r in range(3):
                tokens[starts[r] + 1] = probe[starts[r]].argmax()
        kept, following, logp = s.check(E.ints(tokens.tolist()), parents)
        logits = seen[-1].float().cpu().numpy()
        mask = E.masks(parents).cpu().numpy().view(np.uint64)
        if step == 0:
            compare("tree", tokens, new, lens, mask, logits)
        above = [starts[r] + max(a, 0) for r, p in enumerate(parents) for a in p]
        want = T.log_probs(logits[above], 1.0, tokens[:, None], 0)[0]
        assert np.abs(logp.cpu().numpy() - want).max() < 1e-5
        said = logits.argmax(1)  # (the lowest index of equal ones, as the library's)
        for r, rows in enumerate(kept):
            assert rows[0] == starts[r] and len(rows) >= (2 if step else 1)
            for a, b in zip(rows, rows[1:]):
                assert parents[r][b - starts[r]] == a - starts[r] and tokens[b] == said[a]
            assert following[r] == said[rows[-1]] and s.lens[r] == lens[r] + len(rows)
        if step == 0:
            at = [i for rows in kept for i in rows]
            kstarts = np.concatenate([[0], np.cumsum([len(r) for r in kept])]).tolist()
            for r in ref:
                r.cache.append(table, s.lens, kstarts, r.new[0][at], r.new[1][at])
            # the next token of each alone, behind what was kept
            one = g.integers(0, s.vocab, 3)
            logits = s.run(E.ints(one.tolist()), [1] * 3).float().cpu().numpy()
            compare("after it", one, [1] * 3, s.lens, None, logits)

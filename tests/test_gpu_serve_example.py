"""The decoder example, prompts and steps, against the same layers in numpy
(sums in 64 bits, bf16 where the example rounds)."""
import os
import sys

import numpy as np
import pytest

from oracle import serve as S

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def norm(x):
    return bf16(x / np.sqrt((x.astype(np.float64) ** 2).mean(-1, keepdims=True) + 1e-6))


class Layer:
    def __init__(self, layer, pages, enc_pages, page):
        self.w = {n: (c.cpu().numpy(), s.cpu().numpy()) for n, (c, s) in layer.codes.items()}
        self.h, self.kv, self.d = layer.heads, layer.kv, layer.dim
        self.cache, self.enc = S.Cache(pages, self.kv, page, self.d), S.Cache(enc_pages, self.kv, page, self.d)

    def product(self, name, x):
        q, s = S.quantize_rows(x)
        return bf16(S.linear(q, s, *self.w[name]))

    def __call__(self, x, table, lens, starts, enc_table, enc_lens):
        t, h, kv, d = len(x), self.h, self.kv, self.d
        y = self.product("qkv", norm(x)).reshape(t, h + 2 * kv, d)
        self.cache.append(table, lens, starts, y[:, h:h + kv], y[:, h + kv:])
        o = bf16(self.cache.attend(table, lens, starts, y[:, :h], d ** -0.5)[0])
        x = bf16(x + self.product("out", o.reshape(t, -1)))
        q = self.product("cross_q", norm(x)).reshape(t, h, d)
        o = bf16(self.enc.attend(enc_table, enc_lens, starts, q, d ** -0.5, causal=False)[0])
        x = bf16(x + self.product("cross_out", o.reshape(t, -1)))
        a, b = np.split(self.product("up", norm(x)), 2, 1)
        return bf16(x + self.product("down", bf16(a / (1 + np.exp(-a.astype(np.float64))) * b)))


def test_decoder_example():
    """Quantisation to 127 steps leaves about 1 % of noise in each of a layer's seven products, and where the two sides round
    apart a code may fall on the other side of a step: at most that noise again, 1 % sqrt(14) = 4 % of the change over two
    layers, which is smaller than the outputs themselves (they carry the inputs)."""
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decode_int8 as E
    prompts, encoders, page = [19, 1, 34], [21, 40, 3], 16
    s = E.Session(prompts, encoders, 4, page=page)
    per, enc = s.table.shape[1], s.enc_table.shape[1]
    table, enc_table = s.table.cpu().numpy(), s.enc_table.cpu().numpy()
    ref = [Layer(layer, 3 * per, 3 * enc, page) for layer in s.layers]
    starts = np.concatenate([[0], np.cumsum(encoders)]).tolist()
    states = s.states.float().cpu().numpy()
    for r in ref:
        y = r.product("cross_kv", states).reshape(len(states), 2 * r.kv, r.d)
        r.enc.append(enc_table, encoders, starts, y[:, :r.kv], y[:, r.kv:])
    g = np.random.default_rng(9)
    lens = list(prompts)
    for step in range(4):
        new = prompts if step == 0 else [1] * 3
        x = bf16(g.standard_normal((sum(new), s.width)))
        xt = torch.from_numpy(x).to(torch.bfloat16).cuda()
        if step:
            lens = [n + 1 for n in lens]
        got = (s.step(xt) if step else s.prompt(xt)).float().cpu().numpy()
        starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        for r in ref:
            x = r(x, table, lens, starts, enc_table, encoders)
        err = np.linalg.norm(got - x) / np.linalg.norm(x)
        print("step", step, "relative difference", err, flush=True)
        assert err < 0.04

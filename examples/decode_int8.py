"""A transformer decoder layer served in 8 bits with the library's operators:
products with scales for each token and channel, a paged 8-bit cache, causal
attention for prompts and single tokens, and cross attention to an encoder's
states of another length.

    python examples/decode_int8.py [--layers 4] [--width 1024] [--steps 32]

Weights and inputs are random.  Prints the time of the prompts and of a step of
all requests; norms, the gate and residual sums are plain torch.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2208_01944_amd import palq  # noqa: E402


def quantized(w):
    """fp32 [n_out, n_in] -> int8 codes and a scale for each channel."""
    s = w.abs().amax(1) / 127
    return (w / s[:, None]).round().to(torch.int8), s


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Layer:
    """One decoder layer: self attention over its cache, cross attention over the encoder's, a gated MLP."""

    NAMES = ("qkv", "out", "cross_q", "cross_kv", "cross_out", "up", "down")

    def __init__(self, ctx, width, heads, kv_heads, dim, hidden, pages, page, enc_pages, max_rows, gen):
        self.ctx, self.heads, self.kv, self.dim = ctx, heads, kv_heads, dim
        shapes = dict(qkv=((heads + 2 * kv_heads) * dim, width), out=(width, heads * dim), cross_q=(heads * dim, width),
                      cross_kv=(2 * kv_heads * dim, width), cross_out=(width, heads * dim), up=(2 * hidden, width), down=(width, hidden))
        self.codes = {n: quantized(torch.randn(*shapes[n], generator=gen, device="cuda") * shapes[n][1] ** -0.5) for n in self.NAMES}
        self.lin = {n: palq.Linear(ctx, *self.codes[n], max_rows=max_rows) for n in self.NAMES}
        self.cache = palq.Cache.empty(pages, kv_heads, page, dim)
        self.encoder = palq.Cache.empty(enc_pages, kv_heads, page, dim)

    def product(self, name, x):
        y = torch.empty(x.shape[0], self.lin[name].n_out, dtype=torch.bfloat16, device="cuda")
        self.lin[name].run(x, y)
        return y

    def remember(self, states, batch):
        """Caches the encoder's keys and values, once for a batch of requests."""
        k, v = self.product("cross_kv", states).unflatten(1, (2 * self.kv, self.dim)).split(self.kv, 1)
        self.ctx.cache_append(self.encoder, k, v, batch)

    def __call__(self, x, batch, cross):
        """x [tokens, width]; batch: the requests' tokens with these at their ends; cross: the same rows over the encoder's tokens."""
        q, k, v = self.product("qkv", norm(x)).unflatten(1, (self.heads + 2 * self.kv, self.dim)).split([self.heads, self.kv, self.kv], 1)
        self.ctx.cache_append(self.cache, k, v, batch)
        o = torch.empty(x.shape[0], self.heads, self.dim, dtype=torch.bfloat16, device="cuda")
        self.ctx.attention(self.cache, q, o, batch, self.dim ** -0.5)
        x = x + self.product("out", o.flatten(1))
        q = self.product("cross_q", norm(x)).unflatten(1, (self.heads, self.dim))
        self.ctx.attention(self.encoder, q, o, cross, self.dim ** -0.5, causal=False)
        x = x + self.product("cross_out", o.flatten(1))
        a, b = self.product("up", norm(x)).chunk(2, 1)
        return x + self.product("down", (torch.nn.functional.silu(a.float()) * b.float()).to(torch.bfloat16))


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Session:
    """Requests with their page tables: prompts first, then one token of each at a time."""

    def __init__(self, prompts, encoders, room, layers=2, width=256, heads=4, kv_heads=2, dim=64, hidden=512, page=16, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ctx = palq.Context(0)
        n = len(prompts)
        per, enc = -(-(max(prompts) + room) // page), -(-max(encoders) // page)
        self.lens, self.width = list(prompts), width
        self.table = torch.randperm(n * per, generator=gen, device="cuda").to(torch.int32).view(n, per)
        self.enc_table = torch.arange(n * enc, dtype=torch.int32, device="cuda").view(n, enc)
        self.enc_lens = ints(encoders)
        rows = max(sum(prompts), sum(encoders), n)
        self.layers = [Layer(self.ctx, width, heads, kv_heads, dim, hidden, n * per, page, n * enc, rows, gen) for _ in range(layers)]
        starts = [0]
        for e in encoders:
            starts.append(starts[-1] + e)
        self.states = torch.randn(starts[-1], width, generator=gen, device="cuda").to(torch.bfloat16)
        batch = palq.Batch(self.enc_table, self.enc_lens, ints(starts), max(encoders), max(encoders))
        for layer in self.layers:
            layer.remember(self.states, batch)
        self.encoders = encoders

    def run(self, x, new):
        """x: the rows of `new` tokens of each request, one after the other; self.lens counts them already."""
        starts = [0]
        for t in new:
            starts.append(starts[-1] + t)
        starts = ints(starts)
        batch = palq.Batch(self.table, ints(self.lens), starts, max(new), max(self.lens))
        cross = palq.Batch(self.enc_table, self.enc_lens, starts, max(new), max(self.encoders))
        for layer in self.layers:
            x = layer(x, batch, cross)
        return x

    def prompt(self, x):
        return self.run(x, list(self.lens))

    def step(self, x):
        self.lens = [t + 1 for t in self.lens]
        return self.run(x, [1] * len(self.lens))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=32)
    args = ap.parse_args()
    prompts, encoders = [1000, 37, 512, 801, 1, 300, 640, 129], [1500, 750, 900, 1500, 333, 1200, 64, 1111]
    s = Session(prompts, encoders, args.steps, args.layers, args.width, args.width // 64, args.width // 256, 64, 4 * args.width, 64)
    x = torch.randn(sum(prompts), args.width, device="cuda").to(torch.bfloat16)
    for label, call, rows in (("prompts", lambda: s.prompt(x), len(x)),
                              ("steps", lambda: [s.step(x[:len(prompts)]) for _ in range(args.steps)], len(prompts) * args.steps)):
        torch.cuda.synchronize()
        t = time.perf_counter()
        call()
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"{label}: {rows} tokens in {t * 1e3:.2f} ms, {rows / t:.0f} tokens/s")


if __name__ == "__main__":
    main()

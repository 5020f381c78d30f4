"""The 8-bit transformer operators under measurement, over the range of
sizes, types and layouts that the library takes, and their plain forms.

Kinds of cases:
  linear : y = (codes of x) W^T with a scale for each token and channel, x
           quantised within the call (or given as codes and scales);
  append : new keys and values quantised into the pages of an 8-bit cache with
           a scale for each block of tokens and head, then the touched blocks
           read back as the values they stand for;
  attend : attention of ragged queries over such a cache: causal prompts,
           single tokens, windows, and cross attention (causal = False).

Cache layout: k [pages, heads, page, dim], v [pages, heads, dim, page], int8;
scales [pages, heads]; a request's token j lies on page table[r, j // page],
place j % page.  The queries of request r are rows starts[r] .. starts[r + 1]
and belong to its last positions; lens[r] counts its cached tokens.

Quantisation is part of the definition, in 32-bit arithmetic: s = max(max|x| *
fl(1/127), 2^-100), code = clamp(rint(x * fl(1/s)), -127, 127).
"""
import math

import numpy as np
import torch

own = False

C127 = float(np.float32(1.0) / np.float32(127.0))
FLOOR = 2.0 ** -100
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
DEV = "cuda"


def listed():
    return [
        # one token of one request through a projection: the latency of generation
        dict(name="linear_1x4096x4096_bf16", kind="linear", rows=1, n_in=4096, n_out=4096, x="bf16", y="bf16", bias=False),
        # a batch of generating requests through an up projection
        dict(name="linear_48x4096x16384_bf16", kind="linear", rows=48, n_in=4096, n_out=16384, x="bf16", y="bf16", bias=False),
        # a classifier head of the image networks on fp32 features, sizes that fill no tile
        dict(name="linear_333x2047x1000_f32", kind="linear", rows=333, n_in=2047, n_out=1000, x="f32", y="f32", bias=True),
        # a chunk of prompts whose codes the previous operator left
        dict(name="linear_1024x4096x4096_i8", kind="linear", rows=1024, n_in=4096, n_out=4096, x="i8", y="f16", bias=True),
        # the largest: a batch of long prompts through a wide layer
        dict(name="linear_4096x8192x8192_bf16", kind="linear", rows=4096, n_in=8192, n_out=8192, x="bf16", y="bf16", bias=False),
        # one new token for each of 64 generating requests, somewhere inside their blocks
        dict(name="append_64x1_d128_bf16", kind="append", requests=64, new_lo=1, new_hi=1, old_lo=65, old_hi=4000, page=64,
             heads=8, dim=128, dtype="bf16"),
        # prompts of different lengths, the first ones of their requests or continued ones
        dict(name="append_8xprompt_d128_bf16", kind="append", requests=8, new_lo=113, new_hi=2048, old_lo=0, old_hi=301,
             page=64, heads=8, dim=128, dtype="bf16"),
        # a single generating request with a short history
        dict(name="attend_1x1_300_d64_f16", kind="attend", requests=1, new_lo=1, new_hi=1, len_lo=300, len_hi=300, page=16,
             heads=8, group=1, dim=64, causal=True, window=0, dtype="f16"),
        # a large batch of generating requests with long histories of different lengths
        dict(name="attend_32x1_16k_d128_bf16", kind="attend", requests=32, new_lo=1, new_hi=1, len_lo=2047, len_hi=16384,
             page=64, heads=8, group=4, dim=128, causal=True, window=0, dtype="bf16"),
        # a few drafted tokens checked at once behind one very long history, the older part outside a window
        dict(name="attend_4x5_window_d128_bf16", kind="attend", requests=4, new_lo=5, new_hi=5, len_lo=20001, len_hi=32768,
             page=32, heads=8, group=4, dim=128, causal=True, window=8191, dtype="bf16"),
        # ragged chunks of prompts behind cached parts
        dict(name="attend_4xprompt_d128_bf16", kind="attend", requests=4, new_lo=1531, new_hi=2048, len_lo=2100, len_hi=4096,
             page=64, heads=8, group=4, dim=128, causal=True, window=0, dtype="bf16"),
        # decoder tokens attending an encoder's states of another length
        dict(name="attend_8xcross_d64_f16", kind="attend", requests=8, new_lo=17, new_hi=131, len_lo=750, len_hi=1500,
             page=32, heads=16, group=1, dim=64, causal=False, window=0, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "append", "attend", "attend"])
    while True:
        if kind == "linear":
            c = dict(kind=kind, rows=_log(rng, 1, 4096), n_in=_log(rng, 64, 8192), n_out=_log(rng, 64, 8192),
                     x=rng.choice(["bf16", "bf16", "f16", "f32", "i8"]), y=rng.choice(["bf16", "f16", "f32"]),
                     bias=rng.random() < 0.5)
            if rng.random() < 0.5:  # half of the widths as models have them, the others odd
                c["n_in"], c["n_out"] = -(-c["n_in"] // 128) * 128, -(-c["n_out"] // 128) * 128
            if 3072 not in c.values():  # no width of this library's configurations
                return c
            continue
        page, dim = rng.choice([16, 32, 64, 128]), rng.choice([64, 96, 128, 256])
        if kind == "append":
            hi = _log(rng, 1, 2048)
            old = _log(rng, 1, 4000)
            c = dict(kind=kind, requests=_log(rng, 1, 64), new_lo=rng.randint(1, hi), new_hi=hi, old_lo=rng.randint(0, old),
                     old_hi=old, page=page, heads=_log(rng, 1, 16), dim=dim, dtype=rng.choice(["bf16", "f16", "f32"]))
            most = listed()[6]
        else:
            hi = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 16, 2048)])
            new_lo = rng.randint(1, hi)
            length = _log(rng, 32, 32768)
            causal = rng.random() < 0.75
            if causal:
                length = max(length, hi)
            c = dict(kind=kind, requests=_log(rng, 1, 32), new_lo=new_lo, new_hi=hi,
                     len_lo=rng.randint(max(1, hi if causal else 1, length // 8), length), len_hi=length, page=page,
                     heads=rng.choice([1, 2, 4, 8, 16]), group=rng.choice([1, 2, 4, 7, 8]), dim=dim, causal=causal,
                     window=rng.choice([0, 0, 0, _log(rng, 16, 8192)]) if causal else 0, dtype=rng.choice(["bf16", "f16"]))
            # the plain form holds every score and the values in 32 bits
            scores = c["requests"] * c["heads"] * c["group"] * hi * length
            if scores > 4 * 32 * 2048 * 4096 or c["requests"] * c["heads"] * length * dim > 32 * 8 * 16384 * 128:
                continue
            most = listed()[10]
        if work(c)["flops"] <= work(most)["flops"] and work(c)["bytes"] <= max(work(m)["bytes"] for m in listed() if m["kind"] == kind):
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi in a mixed order, the same for every seed."""
    at = [(7 * i + 3) % n for i in range(n)] if n % 7 else [(5 * i + 1) % n for i in range(n)] if n % 5 else list(range(n))
    return [hi if n == 1 else lo + (hi - lo) * a // (n - 1) for a in at]


def _shape(c):
    """Tokens cached and tokens new of each request (host lists)."""
    new = _spread(c["new_lo"], c["new_hi"], c["requests"])
    if c["kind"] == "append":
        lens = [o + t for o, t in zip(_spread(c["old_lo"], c["old_hi"], c["requests"])[::-1], new)]
    else:
        lens = _spread(c["len_lo"], c["len_hi"], c["requests"])[::-1]
    return lens, new


def _seen(c, length, new):
    """(query, token) pairs that the mask leaves of one request, and the tokens that any query sees."""
    if not c["causal"]:
        return new * length, length
    pos = np.arange(length - new, length, dtype=np.int64)
    lo = np.maximum(0, pos - c["window"] + 1) if c["window"] else np.zeros_like(pos)
    return int(np.sum(pos + 1 - lo)), int(length - lo[0])


def work(case):
    c = case
    if c["kind"] == "linear":
        m, k, n = c["rows"], c["n_in"], c["n_out"]
        b = m * k * SIZE[c["x"]] + n * k + 4 * n * (1 + c["bias"]) + m * n * SIZE[c["y"]] + (4 * m if c["x"] == "i8" else 0)
        return {"bytes": b, "flops": 2 * m * k * n}
    lens, new = _shape(c)
    if c["kind"] == "append":
        h, d, p = c["heads"], c["dim"], c["page"]
        read = sum(2 * h * d * SIZE[c["dtype"]] * t for t in new)
        code = sum(2 * h * d * t for t in new)
        back = sum(ln - (ln - t) // p * p for ln, t in zip(lens, new))  # tokens of the touched blocks
        scales = sum(2 * 4 * h * (-(-ln // p) - (ln - t) // p) for ln, t in zip(lens, new))
        # new values in, their codes out; the touched blocks' codes in, their values out in 32 bits
        return {"bytes": read + code + scales + 2 * h * d * back * 5, "flops": 2 * h * d * (sum(new) * 3 + back)}
    pairs = [_seen(c, ln, t) for ln, t in zip(lens, new)]
    h, d = c["heads"], c["dim"]
    b = sum(t * 2 * h * d + -(-t // c["page"]) * (8 * h + 4) for _, t in pairs) + 2 * sum(new) * h * c["group"] * d * 2
    return {"bytes": b, "flops": 4 * d * h * c["group"] * sum(p for p, _ in pairs)}


def _context():
    from paper_2208_01944_amd import palq
    if not hasattr(_context, "ctx"):
        _context.ctx = palq.Context(0)
    return palq, _context.ctx


def _paged(c, lens, g):
    """A page table that scatters every request's pages over the pool; the pool has some pages to spare."""
    per = [-(-ln // c["page"]) for ln in lens]
    pages = sum(per) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(len(lens), max(per), dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(per):
        table[r, :n] = order[at:at + n]
        at += n
    return table, pages


def _codes(shape, g):
    """Codes as blocks of normal values have them: the largest of a block near 127."""
    out = torch.empty(shape, dtype=torch.int8, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = (torch.randn(n, generator=g, device=DEV) * 32).round_().clamp_(-127, 127).to(torch.int8)
    return out


def _scales(pages, heads, g):
    """Scales of normal values, some blocks several times larger than others."""
    return torch.exp(torch.randn(pages, heads, generator=g, device=DEV) * 0.4) / 32.0


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    if c["kind"] == "linear":
        m, k, n = c["rows"], c["n_in"], c["n_out"]
        s = dict(case=c, w=torch.randint(-127, 128, (n, k), generator=g, device=DEV, dtype=torch.int8),
                 w_scale=torch.exp(rnd(n) * 0.3) / (74.0 * math.sqrt(k)), bias=rnd(n) if c["bias"] else None, x_scale=None)
        if c["x"] == "i8":
            s["x"] = _codes((m, k), g)
            s["x_scale"] = torch.exp(rnd(m) * 0.3) / 32.0
        else:  # activations with a few large channels
            s["x"] = (rnd(m, k) * torch.exp(rnd(1, k) * 0.7)).to(DT[c["x"]])
        s["y"] = torch.empty(m, n, dtype=DT[c["y"]], device=DEV)
        if own:
            palq, ctx = _context()
            s["plan"] = palq.Linear(ctx, s["w"], s["w_scale"], s["bias"], max_rows=m)
        return s
    lens, new = _shape(c)
    table, pages = _paged(c, lens, g)
    h, d, p = c["heads"], c["dim"], c["page"]
    s = dict(case=c, k=_codes((pages, h, p, d), g), v=_codes((pages, h, d, p), g), ks=_scales(pages, h, g),
             vs=_scales(pages, h, g), table=table, lens=_ints(lens), starts=_ints(np.concatenate([[0], np.cumsum(new)]).tolist()),
             max_new=max(new), max_len=max(lens))
    tokens = sum(new)
    if c["kind"] == "append":
        dt = DT[c["dtype"]]
        s["new_k"], s["new_v"] = (rnd(tokens, h, d) * 1.3).to(dt), (rnd(tokens, h, d) * 0.9).to(dt)
        back = [ln - (ln - t) // p * p for ln, t in zip(lens, new)]
        s["back"] = _ints(np.concatenate([[0], np.cumsum(back)]).tolist())
        s["max_back"] = max(back)
        s["out_k"] = torch.empty(sum(back), h, d, dtype=torch.float32, device=DEV)
        s["out_v"] = torch.empty_like(s["out_k"])
    else:
        s["q"] = (rnd(tokens, h * c["group"], d) * 1.5).to(DT[c["dtype"]])
        s["out"] = torch.empty_like(s["q"])
    if own:
        palq, ctx = _context()
        s["cache"] = palq.Cache(s["k"], s["v"], s["ks"], s["vs"])
        s["batch"] = palq.Batch(table, s["lens"], s["starts"], s["max_new"], s["max_len"])
        if c["kind"] == "append":
            s["read"] = palq.Batch(table, s["lens"], s["back"], s["max_back"], s["max_len"])
    return s


def run(state):
    s = state
    c = s["case"]
    if own:
        _, ctx = _context()
        if c["kind"] == "linear":
            s["plan"].run(s["x"], s["y"], x_scale=s["x_scale"])
            return s["y"]
        if c["kind"] == "append":
            ctx.cache_append(s["cache"], s["new_k"], s["new_v"], s["batch"])
            ctx.cache_read(s["cache"], s["out_k"], s["out_v"], s["read"])
            return s["out_k"], s["out_v"]
        ctx.attention(s["cache"], s["q"], s["out"], s["batch"], c["dim"] ** -0.5, causal=c["causal"], window=c["window"])
        return s["out"]
    return {"linear": _linear, "append": _append, "attend": _attend}[c["kind"]](s)


# ------------------------------------------------------------------ plain forms
def _linear(s):
    if s["x_scale"] is None:
        x = s["x"].float()
        sx = (x.abs().amax(1) * C127).clamp_min(FLOOR)
        q = (x * sx.reciprocal()[:, None]).round().clamp(-127, 127)
    else:
        q, sx = s["x"].float(), s["x_scale"]
    y = torch.matmul(q, s["w"].float().t()) * sx[:, None] * s["w_scale"][None, :]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["y"].dtype)


def _rows(starts, tokens):
    """Request and index within it of every ragged row."""
    at = torch.arange(tokens, device=DEV)
    r = (at[:, None] >= starts[None, 1:]).sum(1)
    return r, at - starts.long()[r]


def _append(s):
    c = s["case"]
    p, table, lens = c["page"], s["table"].long(), s["lens"].long()
    tokens, heads = s["new_k"].shape[:2]
    r, i = _rows(s["starts"], tokens)
    old = lens - (s["starts"][1:] - s["starts"][:-1])  # tokens before the new ones
    pos = old[r] + i
    page, place = table[r, pos // p], pos % p
    pages = s["k"].shape[0]
    head = torch.gather(table, 1, (old // p).clamp(max=table.shape[1] - 1)[:, None])[:, 0]  # the block where each request goes on
    kept = (old % p > 0)[:, None]
    for x, codes, scale in ((s["new_k"], s["k"], s["ks"]), (s["new_v"], s["v"].transpose(2, 3), s["vs"])):
        x = x.float()
        a = torch.zeros(pages, heads, device=DEV).scatter_reduce_(0, page[:, None].expand(-1, heads), x.abs().amax(2), "amax")
        now = (a * C127).clamp_min(FLOOR)
        had = scale[head]
        now[head] = torch.where(kept, torch.maximum(now[head], had), now[head])
        ratio = torch.where(kept & (now[head] > had), had / now[head], 1.0)
        codes[head] = (codes[head].float() * ratio[:, :, None, None]).round().to(torch.int8)
        codes[page, :, place] = (x * now.reciprocal()[page][:, :, None]).round().clamp(-127, 127).to(torch.int8)
        scale[page] = now[page]
    n = s["out_k"].shape[0]
    r, i = _rows(s["back"], n)
    pos = lens[r] - (s["back"][1:] - s["back"][:-1]).long()[r] + i
    page, place = table[r, pos // p], pos % p
    return s["k"][page, :, place].float() * s["ks"][page][:, :, None], s["v"][page, :, :, place].float() * s["vs"][page][:, :, None]


def _attend(s):
    c = s["case"]
    p, d, h, group = c["page"], c["dim"], c["heads"], c["group"]
    requests, most, longest = c["requests"], s["max_new"], s["max_len"]
    table, lens, starts = s["table"].long(), s["lens"].long(), s["starts"].long()
    kt = (s["k"][table].float() * s["ks"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(requests, h, -1, d)[:, :, :longest]
    vt = (s["v"][table].float() * s["vs"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(requests, h, -1, d)[:, :, :longest]
    new = starts[1:] - starts[:-1]
    i = torch.arange(most, device=DEV)
    at = (starts[:-1, None] + i[None, :]).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[at].reshape(requests, most, h, group, d).permute(0, 2, 1, 3, 4).reshape(requests, h, most * group, d)
    score = torch.matmul(q, kt.transpose(2, 3)).mul_(d ** -0.5).view(requests, h, most, group, longest)
    j = torch.arange(longest, device=DEV)
    sees = (j[None, None, :] < lens[:, None, None]).expand(-1, most, -1)
    if c["causal"]:
        pos = (lens - new)[:, None, None] + i[None, :, None]
        sees = sees & (j <= pos)
        if c["window"]:
            sees = sees & (j > pos - c["window"])
    score.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(requests, h, most * group, longest), vt).view(requests, h, most, group, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(requests, most, h * group, d)
    r, t = _rows(starts, s["q"].shape[0])
    return o[r, t].to(s["q"].dtype)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The definitions in 64 bits, request by request and block by block; codes and scales, which the definition
    forms in 32-bit arithmetic, are formed so."""
    s = prepare(case, seed)
    c = case
    one = torch.tensor(1.0, device=DEV)
    low, c127 = torch.tensor(FLOOR, device=DEV), torch.tensor(C127, device=DEV)
    if c["kind"] == "linear":
        if c["x"] == "i8":
            q, sx = s["x"].double(), s["x_scale"].double()
        else:
            x = s["x"].float()
            sx = torch.maximum(torch.max(x.abs(), dim=1).values * c127, low)
            q = torch.clamp(torch.round(x * (one / sx)[:, None]), -127, 127).double()
            sx = sx.double()
        w = s["w"].double() * s["w_scale"].double()[:, None]
        y = torch.cat([torch.mm(part, w.t()) for part in q.split(1024)]) * sx[:, None]
        return y + s["bias"].double() if s["bias"] is not None else y
    lens, starts, table = s["lens"].tolist(), s["starts"].tolist(), s["table"].tolist()
    p = c["page"]
    if c["kind"] == "append":
        if sum(-(-ln // p) for ln in lens) > 40000:
            return None
        out = []
        for name, codes, scale in (("new_k", s["k"], s["ks"]), ("new_v", s["v"].transpose(2, 3), s["vs"])):
            x, vals = s[name].float(), []
            for r, ln in enumerate(lens):
                n = starts[r + 1] - starts[r]
                for b in range((ln - n) // p, -(-ln // p)):
                    lo, hi = max(b * p, ln - n), min(b * p + p, ln)
                    page, kept = table[r][b], lo - b * p
                    part = x[starts[r] + lo - (ln - n):starts[r] + hi - (ln - n)].transpose(0, 1)  # [heads, tokens, dim]
                    now = torch.maximum(torch.amax(part.abs(), dim=(1, 2)) * c127, low)
                    block = codes[page, :, :kept].float()
                    if kept:
                        had = scale[page]
                        now = torch.maximum(now, had)
                        block = torch.where((now > had)[:, None, None], torch.round(block * (had / now)[:, None, None]), block)
                    fresh = torch.clamp(torch.round(part * (one / now)[:, None, None]), -127, 127)
                    vals.append((torch.cat([block, fresh], 1).double() * now.double()[:, None, None]).transpose(0, 1))
            out.append(torch.cat(vals))
        return out[0], out[1]
    if work(c)["flops"] > 2e12:
        return None
    h, group, d = c["heads"], c["group"], c["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for r, ln in enumerate(lens):
        n = starts[r + 1] - starts[r]
        pages = s["table"][r, :-(-ln // p)].long()
        pos = torch.arange(ln - n, ln, device=DEV)[:, None, None]
        j = torch.arange(ln, device=DEV)[None, None, :]
        sees = torch.ones(n, 1, ln, dtype=torch.bool, device=DEV)
        if c["causal"]:
            sees = sees & (j <= pos)
            if c["window"]:
                sees = sees & (pos - j < c["window"])
        for g in range(h):
            k = (s["k"][pages, g].double() * s["ks"][pages, g].double()[:, None, None]).reshape(-1, d)[:ln]
            v = (s["v"][pages, g].double() * s["vs"][pages, g].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:ln]
            q = s["q"][starts[r]:starts[r + 1], g * group:(g + 1) * group].double()
            z = torch.mm(q.reshape(n * group, d), k.t()).reshape(n, group, ln) / math.sqrt(d)
            z = torch.where(sees, z, torch.full_like(z, -math.inf))
            z = torch.exp(z - z.max(-1, keepdim=True).values.nan_to_num(neginf=0.0))
            z = z / z.sum(-1, keepdim=True).clamp_min(1e-300)
            out[starts[r]:starts[r + 1], g * group:(g + 1) * group] = torch.mm(z.reshape(n * group, ln), v).reshape(n, group, d)
    return out

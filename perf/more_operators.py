"""Operators of a generation step with drafted tokens under measurement, over
the range of sizes, types and layouts that the library takes, and their plain
forms.

Kinds of cases:
  rotate : RMS norm of each head of queries and keys and the rotation by their
           positions, from a fused projection into tensors of their own;
  sinks  : attention of ragged queries over an 8-bit paged cache, through a
           window and the first tokens of each request, which stay visible;
  tree   : the same for drafted tokens that form a tree: a row sees the cached
           tokens before the draft and the drafted ones whose bit its mask has;
  logp   : log probabilities of given tokens, entropy and the most probable
           tokens of each row of logits.

Cache layout: k [pages, heads, page, dim], v [pages, heads, dim, page], int8;
scales [pages, heads]; a request's token j lies on page table[r, j // page],
place j % page.  The rows of request r are starts[r] .. starts[r + 1] of the
tensors and belong to its last positions; lens[r] counts its cached tokens.  Of
a tree's rows, bit b of the mask stands for the request's b-th new token, and a
row's position is the first new one's plus the number of other tokens it sees.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
DEV = "cuda"
EPS = 1e-6
BASE = 500000.0


def listed():
    return [
        # one token of one request at a far position: the latency of generation
        dict(name="rotate_1x1_d128_bf16", kind="rotate", requests=1, new_lo=1, new_hi=1, old_lo=200000, old_hi=200000, q_heads=32,
             k_heads=8, dim=128, pairs=64, interleaved=False, norm=True, tree=False, dtype="bf16"),
        # drafted trees of a batch; a quarter of each head rotates, in neighbouring pairs
        dict(name="rotate_48x25_tree_d64_f16", kind="rotate", requests=48, new_lo=9, new_hi=25, old_lo=300, old_hi=30000, q_heads=16,
             k_heads=4, dim=64, pairs=8, interleaved=True, norm=True, tree=True, dtype="f16"),
        # a batch of long prompts
        dict(name="rotate_8xprompt_d128_bf16", kind="rotate", requests=8, new_lo=1531, new_hi=4096, old_lo=0, old_hi=8191, q_heads=32,
             k_heads=8, dim=128, pairs=64, interleaved=False, norm=True, tree=False, dtype="bf16"),
        # a single generating request, most of its history outside the window
        dict(name="sinks_1x1_5000_d64_f16", kind="sinks", requests=1, new_lo=1, new_hi=1, len_lo=5000, len_hi=5000, page=16,
             heads=8, group=1, dim=64, window=512, sinks=4, dtype="f16"),
        # a large batch of generating requests, histories of different lengths
        dict(name="sinks_32x1_32k_d128_bf16", kind="sinks", requests=32, new_lo=1, new_hi=1, len_lo=2047, len_hi=32768, page=64,
             heads=8, group=4, dim=128, window=4096, sinks=4, dtype="bf16"),
        # ragged chunks of long prompts behind cached parts
        dict(name="sinks_4xprompt_d128_bf16", kind="sinks", requests=4, new_lo=1531, new_hi=2048, len_lo=4100, len_hi=8192, page=32,
             heads=8, group=4, dim=128, window=1024, sinks=100, dtype="bf16"),
        # a few drafted tokens behind a short history
        dict(name="tree_1x7_700_d64_f16", kind="tree", requests=1, new_lo=7, new_hi=7, len_lo=700, len_hi=700, page=16, heads=8,
             group=1, dim=64, window=0, sinks=0, dtype="f16"),
        # small drafts behind long histories, heads in groups of seven, a window with sinks
        dict(name="tree_8x25_window_d96_bf16", kind="tree", requests=8, new_lo=11, new_hi=25, len_lo=5001, len_hi=20000, page=32,
             heads=4, group=7, dim=96, window=4095, sinks=4, dtype="bf16"),
        # large drafts of a batch
        dict(name="tree_16x64_d128_bf16", kind="tree", requests=16, new_lo=48, new_hi=64, len_lo=1000, len_hi=16384, page=64,
             heads=8, group=4, dim=128, window=0, sinks=0, dtype="bf16"),
        # the logits of one generated token
        dict(name="logp_1x131071_bf16", kind="logp", rows=1, vocab=131071, given=1, top=20, scale=1.0, masked=True, dtype="bf16"),
        # classes of a batch of images
        dict(name="logp_333x1000_f32", kind="logp", rows=333, vocab=1000, given=1, top=5, scale=1.0, masked=False, dtype="f32"),
        # the tokens of long prompts scored
        dict(name="logp_4096x131071_bf16", kind="logp", rows=4096, vocab=131071, given=1, top=20, scale=1.25, masked=True,
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "sinks", "tree", "logp"])
    most = [work(m) for m in listed() if m["kind"] == kind]
    flops, moved = max(m["flops"] for m in most), max(m["bytes"] for m in most)
    while True:
        if kind == "logp":
            vocab = _log(rng, 100, 262144)
            c = dict(kind=kind, rows=_log(rng, 1, 8192), vocab=vocab, given=rng.choice([0, 1, 1, 4]),
                     top=rng.choice([0, 1, 5, 20, 64]), scale=rng.choice([1.0, 1.25, 0.7]), masked=rng.random() < 0.5,
                     dtype=rng.choice(["bf16", "f16", "f32"]))
        elif kind == "rotate":
            dim, hi, old = rng.choice([64, 96, 128, 256]), rng.choice([1, _log(rng, 2, 64), _log(rng, 16, 4096)]), _log(rng, 1, 1 << 20)
            pairs = rng.choice([dim // 2, dim // 2, dim // 4, dim // 8, rng.randint(1, dim // 2)])
            k_heads = rng.choice([1, 2, 4, 8, 16])
            c = dict(kind=kind, requests=_log(rng, 1, 64), new_lo=rng.randint(1, hi), new_hi=hi, old_lo=rng.randint(0, old), old_hi=old,
                     q_heads=k_heads * rng.choice([1, 2, 4, 7, 8]), k_heads=k_heads, dim=dim, pairs=pairs, interleaved=rng.random() < 0.3,
                     norm=rng.random() < 0.8, tree=hi <= 64 and rng.random() < 0.5, dtype=rng.choice(["bf16", "f16", "f32"]))
        else:
            hi = _log(rng, 2, 256) if kind == "tree" else rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 16, 2048)])
            length = max(hi, _log(rng, 32, 32768))
            window = _log(rng, 16, 8192) if kind == "sinks" or rng.random() < 0.4 else 0
            c = dict(kind=kind, requests=_log(rng, 1, 32), new_lo=rng.randint(1, hi), new_hi=hi,
                     len_lo=rng.randint(max(hi, length // 8), length), len_hi=length, page=rng.choice([16, 32, 64, 128]),
                     heads=rng.choice([1, 2, 4, 8, 16]), group=rng.choice([1, 2, 4, 7, 8]), dim=rng.choice([64, 96, 128, 256]),
                     window=window, sinks=rng.choice([1, 4, _log(rng, 1, 512)]) if window else 0, dtype=rng.choice(["bf16", "f16"]))
            # the plain form holds every score and the values in 32 bits
            scores = c["requests"] * c["heads"] * c["group"] * hi * length
            if scores > 4 * 32 * 2048 * 8192 or c["requests"] * c["heads"] * length * c["dim"] > 32 * 8 * 32768 * 128:
                continue
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= moved:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi in a mixed order, the same for every seed."""
    at = [(7 * i + 3) % n for i in range(n)] if n % 7 else [(5 * i + 1) % n for i in range(n)] if n % 5 else list(range(n))
    return [hi if n == 1 else lo + (hi - lo) * a // (n - 1) for a in at]


def _shape(c):
    """Tokens cached and tokens new of each request (host lists)."""
    new = _spread(c["new_lo"], c["new_hi"], c["requests"])
    if c["kind"] == "rotate":
        return [o + t for o, t in zip(_spread(c["old_lo"], c["old_hi"], c["requests"])[::-1], new)], new
    return _spread(c["len_lo"], c["len_hi"], c["requests"])[::-1], new


def _seen(c, length, new):
    """(query, token) pairs that the mask leaves of one request, and the tokens that any query sees."""
    old = length - new
    pos = np.arange(old, length, dtype=np.int64)
    if c["kind"] == "tree":  # a random tree's token is about ln(new) deep
        depth = int(math.log(new))
        pos = np.minimum(pos, old + depth)
    lo = np.maximum(0, pos - c["window"] + 1) if c["window"] else np.zeros_like(pos)
    kept = np.minimum(lo, c["sinks"])
    return int(np.sum(pos + 1 - lo + kept)), int(length - lo[0] + kept[0])


def work(case):
    c = case
    if c["kind"] == "logp":
        n = c["rows"]
        b = n * c["vocab"] * SIZE[c["dtype"]] + n * (8 * c["given"] + 4 + 8 * c["top"])
        return {"bytes": b, "flops": 6 * n * c["vocab"]}
    lens, new = _shape(c)
    if c["kind"] == "rotate":
        rows = sum(new) * (c["q_heads"] + c["k_heads"])
        b = 2 * rows * c["dim"] * SIZE[c["dtype"]] + 8 * c["dim"] * c["norm"] + 8 * c["pairs"]
        return {"bytes": b, "flops": rows * (4 * c["dim"] * c["norm"] + 6 * c["pairs"])}
    pairs = [_seen(c, ln, t) for ln, t in zip(lens, new)]
    h, d = c["heads"], c["dim"]
    b = sum(t * 2 * h * d + -(-t // c["page"]) * (8 * h + 4) for _, t in pairs) + 2 * sum(new) * h * c["group"] * d * 2
    if c["kind"] == "tree":
        b += sum(new) * 8 * -(-c["new_hi"] // 64)
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


def _trees(new, seed):
    """Masks of random trees, int64 [tokens, words]: a token sees itself and its ancestors."""
    most, words = max(new), -(-max(new) // 64)
    rng = np.random.default_rng(seed)
    sees = np.zeros((len(new), most, words * 64), dtype=np.uint8)
    for i in range(most):
        parent = rng.integers(-1, i, size=len(new)) if i else np.full(len(new), -1)
        if i:
            sees[:, i] = np.where((parent >= 0)[:, None], sees[np.arange(len(new)), parent], 0)
        sees[:, i, i] = 1
    rows = np.concatenate([sees[r, :n] for r, n in enumerate(new)])
    packed = np.packbits(rows, axis=1, bitorder="little").view(np.int64)
    return torch.from_numpy(packed.copy()).to(DEV)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    dt = DT[c["dtype"]]
    if c["kind"] == "logp":
        n, vocab = c["rows"], c["vocab"]
        x = torch.empty(n, vocab, dtype=dt, device=DEV)
        for part in x.split(256):
            part.copy_(rnd(*part.shape) * 2.5)
        allowed = vocab - vocab // 50 if c["masked"] else vocab  # a padded vocabulary's tail is masked
        x[:, allowed:] = -math.inf
        s = dict(case=c, x=x, ids=torch.randint(0, allowed, (n, c["given"]), generator=g, device=DEV).to(torch.int32),
                 out=torch.empty(n, c["given"], device=DEV), entropy=torch.empty(n, device=DEV),
                 top_ids=torch.empty(n, c["top"], dtype=torch.int32, device=DEV), top=torch.empty(n, c["top"], device=DEV))
        if own:
            _context()
        return s
    lens, new = _shape(c)
    tokens = sum(new)
    s = dict(case=c, lens=_ints(lens), starts=_ints(np.concatenate([[0], np.cumsum(new)]).tolist()), max_new=max(new), max_len=max(lens),
             tree=_trees(new, seed) if c["kind"] == "tree" or c.get("tree") else None)
    if c["kind"] == "rotate":
        q, k, d = c["q_heads"], c["k_heads"], c["dim"]
        fused = torch.empty(tokens, q + 2 * k, d, dtype=dt, device=DEV)  # queries, keys and values as one projection leaves them
        for part in fused.split(1024):
            part.copy_(rnd(*part.shape) * 1.7)
        s["q"], s["k"] = fused[:, :q], fused[:, q:q + k]
        s["q_out"], s["k_out"] = torch.empty(tokens, q, d, dtype=dt, device=DEV), torch.empty(tokens, k, d, dtype=dt, device=DEV)
        s["q_weight"], s["k_weight"] = (1 + 0.2 * rnd(d), 1 + 0.2 * rnd(d)) if c["norm"] else (None, None)
        s["freq"] = BASE ** -(np.arange(c["pairs"], dtype=np.float64) / c["pairs"])
        s["angles"] = torch.from_numpy(s["freq"]).to(DEV)
        if own:
            palq, ctx = _context()
            s["rotation"] = palq.Rotation(ctx, s["freq"], interleaved=c["interleaved"])
            table = torch.zeros(len(lens), 1, dtype=torch.int32, device=DEV)
            s["batch"] = palq.Batch(table, s["lens"], s["starts"], s["max_new"], s["max_len"])
        return s
    table, pages = _paged(c, lens, g)
    h, d, p = c["heads"], c["dim"], c["page"]
    s.update(k=_codes((pages, h, p, d), g), v=_codes((pages, h, d, p), g), ks=_scales(pages, h, g), vs=_scales(pages, h, g), table=table)
    s["q"] = (rnd(tokens, h * c["group"], d) * 1.5).to(dt)
    s["out"] = torch.empty_like(s["q"])
    if own:
        palq, ctx = _context()
        s["cache"] = palq.Cache(s["k"], s["v"], s["ks"], s["vs"])
        s["batch"] = palq.Batch(table, s["lens"], s["starts"], s["max_new"], s["max_len"])
    return s


def run(state):
    s = state
    c = s["case"]
    if own:
        _, ctx = _context()
        if c["kind"] == "logp":
            ctx.log_probs(s["x"], s["ids"], s["out"], entropy=s["entropy"], top_ids=s["top_ids"], top=s["top"], scale=c["scale"])
            return s["out"], s["entropy"], s["top_ids"], s["top"]
        if c["kind"] == "rotate":
            ctx.norm_rotate(s["batch"], s["q"], s["q_out"], s["k"], s["k_out"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                            eps=EPS if c["norm"] else None, rotation=s["rotation"], tree=s["tree"])
            return s["q_out"], s["k_out"]
        ctx.attention(s["cache"], s["q"], s["out"], s["batch"], c["dim"] ** -0.5, window=c["window"], sinks=c["sinks"], tree=s["tree"])
        return s["out"]
    return {"logp": _logp, "rotate": _rotate, "sinks": _attend, "tree": _attend}[c["kind"]](s)


# ------------------------------------------------------------------ plain forms
def _logp(s):
    c = s["case"]
    raw = s["x"].float()
    x = raw * c["scale"]
    low = x.amax(1, keepdim=True)
    x.sub_(low)
    p = x.exp()
    total = p.sum(1, keepdim=True)
    shift = total.log()
    entropy = shift[:, 0] - p.mul_(x.clamp_min(-1e30)).sum(1) / total[:, 0]
    out = torch.gather(x, 1, s["ids"].long()) - shift
    # the largest in turn, ties to the lowest index: bits of the values in their order as integers
    key = (raw + 0.0).view(torch.int32)
    key = torch.where(key < 0, key ^ 0x7fffffff, key)
    at = torch.arange(c["vocab"], dtype=torch.int32, device=DEV)
    ids = torch.empty(c["rows"], c["top"], dtype=torch.int32, device=DEV)
    for i in range(c["top"]):
        best = key.amax(1, keepdim=True)
        ids[:, i] = torch.where(key == best, at, c["vocab"]).amin(1)
        key.scatter_(1, ids[:, i:i + 1].long(), -(1 << 31))
    return out, entropy, ids, torch.gather(x, 1, ids.long()) - shift


def _rows(starts, tokens):
    """Request and index within it of every ragged row."""
    at = torch.arange(tokens, device=DEV)
    r = (at[:, None] >= starts[None, 1:]).sum(1)
    return r, at - starts.long()[r]


def _bits(mask):
    """int64 [.., words] -> truth values [.., 64 words]."""
    return (mask[..., None] >> torch.arange(64, device=DEV) & 1).flatten(-2) > 0


def _places(s, tokens):
    """Position of every row."""
    r, i = _rows(s["starts"], tokens)
    old = s["lens"].long() - (s["starts"][1:] - s["starts"][:-1]).long()
    if s["tree"] is not None:  # (bit i is the row's own)
        bits = _bits(s["tree"])
        i = bits.sum(1) - torch.gather(bits, 1, i[:, None])[:, 0].long()
    return old[r] + i


def _rotate(s):
    c = s["case"]
    n = c["pairs"]
    turn = _places(s, s["q"].shape[0]).double()[:, None] * s["angles"]
    cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]
    out = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        if c["norm"]:
            y = y * ((y * y).mean(2, keepdim=True) + EPS).rsqrt() * weight
        a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if c["interleaved"] else (y[..., :n], y[..., n:2 * n])
        turned = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack(turned, 3).flatten(2) if c["interleaved"] else torch.cat(turned, 2)
        out.append(torch.cat([turned, y[..., 2 * n:]], 2).to(x.dtype))
    return out[0], out[1]


def _attend(s):
    c = s["case"]
    d, h, group = c["dim"], c["heads"], c["group"]
    requests, most, longest = c["requests"], s["max_new"], s["max_len"]
    table, lens, starts = s["table"].long(), s["lens"].long(), s["starts"].long()
    kt = (s["k"][table].float() * s["ks"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(requests, h, -1, d)[:, :, :longest]
    vt = (s["v"][table].float() * s["vs"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(requests, h, -1, d)[:, :, :longest]
    kt = kt.transpose(2, 3).contiguous()
    old = lens - (starts[1:] - starts[:-1])
    i = torch.arange(most, device=DEV)
    at = (starts[:-1, None] + i[None, :]).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[at].reshape(requests, most, h, group, d).permute(0, 2, 1, 3, 4).reshape(requests, h, most * group, d)
    score = torch.matmul(q, kt).mul_(d ** -0.5).view(requests, h, most, group, longest)
    pos = _places(s, s["q"].shape[0])[at][:, :, None]
    j = torch.arange(longest, device=DEV)[None, None, :]
    sees = (j <= pos).logical_and_(j < lens[:, None, None])
    if c["window"]:
        sees &= (j > pos - c["window"]) | (j < c["sinks"])
    if c["kind"] == "tree":
        b = j - old[:, None, None]
        word = (b >> 6).clamp(0, s["tree"].shape[1] - 1).expand(-1, most, -1)
        drafted = torch.gather(s["tree"][at], 2, word).bitwise_right_shift_(b & 63).bitwise_and_(1) > 0
        sees = torch.where(b >= 0, drafted & (j < lens[:, None, None]), sees)
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
    """The definitions in 64 bits, request by request and in parts of rows."""
    s = prepare(case, seed)
    c = case
    if c["kind"] == "logp":
        parts = []
        for x, ids in zip(s["x"].split(256), s["ids"].split(256)):
            # (-0 and 0 are the same value: no order between them)
            order = torch.sort((x.float() + 0.0), dim=1, descending=True, stable=True).indices[:, :c["top"]]
            z = x.double() * c["scale"]
            z = z - torch.logsumexp(z, 1, keepdim=True)
            h = -torch.where(z == -math.inf, 0.0, z.exp() * z).sum(1)
            parts.append((z.gather(1, ids.long()), h, order.to(torch.int32), z.gather(1, order)))
        return tuple(torch.cat(p) for p in zip(*parts))
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    sight, place = [], []  # of every row: the drafted tokens it sees, its position
    masks = None if s["tree"] is None else s["tree"].cpu().numpy().view(np.uint8)
    for r, ln in enumerate(lens):
        n = starts[r + 1] - starts[r]
        own_bits = np.tril(np.ones((n, n), dtype=bool))
        if masks is not None:
            own_bits = np.unpackbits(masks[starts[r]:starts[r + 1]], axis=1, bitorder="little")[:, :n].astype(bool)
        sight.append(own_bits)
        place.append(ln - n + own_bits.sum(1) - own_bits.diagonal())
    if c["kind"] == "rotate":
        pos = torch.from_numpy(np.concatenate(place).astype(np.float64)).to(DEV)
        half, out = c["pairs"], []
        first = np.arange(half) * 2 if c["interleaved"] else np.arange(half)
        second = first + 1 if c["interleaved"] else first + half
        # a pair as a complex number times exp(i angle)
        unit = torch.polar(torch.ones_like(pos)[:, None].expand(-1, half).contiguous(), torch.outer(pos, s["angles"]))
        for name in ("q", "k"):
            vals = []
            for x, u in zip(s[name].split(1024), unit.split(1024)):
                y = x.double()
                if c["norm"]:
                    y = y / torch.sqrt(torch.mean(y ** 2, dim=-1, keepdim=True) + EPS) * s[name + "_weight"].double()
                z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * u[:, None]
                y = y.clone()
                y[..., first], y[..., second] = z.real, z.imag
                vals.append(y)
            out.append(torch.cat(vals))
        return out[0], out[1]
    if work(c)["flops"] > 2e12:
        return None
    h, group, d, p = c["heads"], c["group"], c["dim"], c["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for r, ln in enumerate(lens):
        n = starts[r + 1] - starts[r]
        pages = s["table"][r, :-(-ln // p)].long()
        sees = torch.ones(n, ln, dtype=torch.bool, device=DEV)
        if c["window"]:
            j = torch.arange(ln, device=DEV)[None, :]
            sees = (torch.from_numpy(place[r]).to(DEV)[:, None] - j < c["window"]) | (j < c["sinks"])
        draft = torch.from_numpy(sight[r]).to(DEV)
        sees[:, ln - n:] = draft if c["kind"] == "tree" else sees[:, ln - n:] & draft
        for g in range(h):
            k = (s["k"][pages, g].double() * s["ks"][pages, g].double()[:, None, None]).reshape(-1, d)[:ln]
            v = (s["v"][pages, g].double() * s["vs"][pages, g].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:ln]
            q = s["q"][starts[r]:starts[r + 1], g * group:(g + 1) * group].double()
            z = torch.mm(q.reshape(n * group, d), k.t()).reshape(n, group, ln) / math.sqrt(d)
            z = torch.where(sees[:, None], z, torch.full_like(z, -math.inf))
            z = torch.exp(z - z.max(-1, keepdim=True).values.nan_to_num(neginf=0.0))
            z = z / z.sum(-1, keepdim=True).clamp_min(1e-300)
            out[starts[r]:starts[r + 1], g * group:(g + 1) * group] = torch.mm(z.reshape(n * group, ln), v).reshape(n, group, d)
    return out

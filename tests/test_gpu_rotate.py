"""GPU checks of head norms with rotation against the numpy oracle: frequencies of any sign and
size, eps of any size, weights of queries and of keys."""
import numpy as np
import pytest

from oracle import step as S
from tests.test_gpu_serve import cumsum, dev, host, say
from tests.test_gpu_step import batch_of, check_rotated

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,pairs,interleaved", [(64, 32, False), (96, 13, False), (128, 64, True)])
def test_frequencies_of_any_sign_and_size(palq, dtype, dim, pairs, interleaved):
    """Turning backwards, by half a turn a position and by many; the sign of a frequency is that of the sine."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("frequencies", dtype, dim, pairs, interleaved)
    g = np.random.default_rng(pairs)
    lens, new = [7, 100003, 2 ** 31 - 1], [7, 20, 5]
    starts = cumsum(new)
    f = np.concatenate([[-1.0, np.pi, -np.pi, 4.0, -4.0, 100.25, -1e3, 0.0], -10000.0 ** -(np.arange(pairs - 8) / pairs)])
    x = dev(g.standard_normal((starts[-1], 3, dim)), dtype)
    out, back = torch.empty_like(x), torch.empty_like(x)
    b = batch_of(lens, starts)
    palq.norm_rotate(b, x, out, rotation=P.Rotation(palq, f, interleaved))
    palq.norm_rotate(b, x, back, rotation=P.Rotation(palq, -f, interleaved))
    palq.sync()
    for got, freq in ((out, f), (back, -f)):
        check_rotated(host(got), host(x), S.positions(lens, starts), dtype, freq=freq, interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("eps", [1e30, 1e38, 3.3e38])
def test_eps_beside_squares_past_the_range(palq, dtype, dim, eps):
    """A mean of squares and an eps that fp32 holds, or nearly, and their sum does not: neither is lost."""
    import torch
    say("large eps", dtype, dim, eps)
    g = np.random.default_rng(dim)
    x = g.standard_normal((8, 3, dim)).astype(np.float32)
    x[0] *= 1.5e19   # squares sum to more than the range, their mean is in it
    x[1] *= 1e20
    x[2] = 0
    x[2, :, 5] = 1.7e19  # one square near the range's end
    x[3] *= 1e18
    x[4] *= 1e30
    x[5, 1] = 0
    x[6, 0, 3], x[6, 2] = np.inf, 2e19
    q = dev(x, dtype)
    out = torch.empty_like(q)
    palq.norm_rotate(batch_of([8], [0, 8]), q, out, eps=eps)
    palq.sync()
    with np.errstate(invalid="ignore"):
        check_rotated(host(out), host(q), np.arange(8), dtype, eps=eps)


@pytest.mark.parametrize("which", ["k", "q", "both"])
@pytest.mark.parametrize("tokens", [3, 9000])
@pytest.mark.parametrize("dtype,dim,pairs,interleaved,q_heads,k_heads", [
    ("bf16", 64, 32, False, 18, 3), ("f32", 96, 13, False, 9, 9), ("f16", 128, 64, True, 8, 2), ("f32", 128, 60, False, 4, 11), ("bf16", 256, 128, False, 5, 2)])
def test_weights_of_queries_and_keys(palq, dtype, dim, pairs, interleaved, q_heads, k_heads, tokens, which):
    """Each has its own weight or none, also where a wave takes the heads of both (9000 tokens)."""
    import torch
    from paper_2208_01944_amd import palq as P
    say("weights", dtype, dim, pairs, interleaved, q_heads, k_heads, tokens, which)
    g = np.random.default_rng(dim + tokens)
    lens, starts = [tokens + 50, 77], [0, tokens - 2, tokens]
    f = 1e4 ** -(np.arange(pairs) / pairs)
    part = [(dev(g.standard_normal((tokens, n, dim)), dtype), g.standard_normal(dim).astype(np.float32)) for n in (q_heads, k_heads)]
    (q, qw), (k, kw) = part
    qw, kw = qw if which != "k" else None, kw if which != "q" else None
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    palq.norm_rotate(batch_of(lens, starts), q, qo, k, ko, q_weight=None if qw is None else dev(qw), k_weight=None if kw is None else dev(kw), eps=1e-6,
                     rotation=P.Rotation(palq, f, interleaved))
    palq.sync()
    some = np.r_[0:min(tokens, 40), tokens - 3:tokens]  # (the oracle takes long)
    pos = S.positions(lens, starts)[some]
    for x, got, w in ((q, qo, qw), (k, ko, kw)):
        check_rotated(host(got)[some], host(x)[some], pos, dtype, freq=f, interleaved=interleaved, weight=w, eps=1e-6)

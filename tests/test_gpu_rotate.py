"""GPU checks of head norms with rotation against the numpy oracle: frequencies of any sign and
size."""
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

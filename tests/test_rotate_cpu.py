"""Host-only checks of head norms with rotation: what the binding makes of its numbers."""
import numpy as np
import pytest

from tests.test_serve_cpu import P  # noqa: F401


@pytest.mark.parametrize("weight", [False, True])
def test_eps_that_fp32_does_not_hold(P, weight):  # noqa: F811
    """An eps that is 0 or loses bits in fp32 is refused: as 0 it would stand for no norm at all, and the call return its input."""
    import torch
    ctx = P.Context(-1)
    b = P.Batch(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 4, 32)
    q, w = torch.zeros(6, 4, 64), torch.zeros(64) if weight else None
    for eps in (1e-50, 1e-46, 1e-40, 2.0 ** -127, 5e-324, 0.0, -1e-6, float("nan"), float("inf"), 1e39):
        with pytest.raises(P.PalqError, match="eps"):
            ctx.norm_rotate(b, q, q, q_weight=w, eps=eps)
    for eps in (2.0 ** -126, 1e-6, 3e38, np.float32(1e-5)):
        ctx.norm_rotate(b, q, q, q_weight=w, eps=eps)

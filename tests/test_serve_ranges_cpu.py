"""Host-only checks: numbers past 32 bits do not wrap round on their way through the binding."""
import pytest
import torch


@pytest.fixture(scope="module")
def P():
    from paper_2208_01944_amd import palq
    return palq


def z(*s, d=torch.int8):
    return torch.zeros(*s, dtype=d)


def batch(P, max_new, max_len):
    i32 = torch.int32
    return P.Batch(z(2, 3, d=i32), z(2, d=i32), z(3, d=i32), max_new, max_len)


@pytest.mark.parametrize("big", [1 << 31, (1 << 32) + 5, 1 << 63, 10 ** 30])
def test_loose_bounds(P, big):
    """A bound past 2^31 - 1 bounds nothing more than that does."""
    d = batch(P, big, big).desc
    assert d.max_new == d.max_len == (1 << 31) - 1
    assert batch(P, 3, big).desc.max_new == 3 and batch(P, big, 0).desc.max_len == 0


@pytest.mark.parametrize("bad", [-1, -(1 << 32), -(1 << 32) + 7])
def test_negative_bounds(P, bad):
    for args in ((bad, 4), (4, bad)):
        with pytest.raises(P.PalqError):
            batch(P, *args)


def test_windows(P, monkeypatch):
    ctx, b = P.Context(-1), batch(P, 4, 32)
    c = P.Cache(z(2, 1, 16, 64), z(2, 1, 64, 16), z(2, 1, d=torch.float32), z(2, 1, d=torch.float32))
    x, seen = z(4, 1, 64, d=torch.bfloat16), []
    real = P._attention
    monkeypatch.setattr(P, "_attention", lambda *a: seen.append(a[-1]) or real(*a))
    for window in (0, 5, (1 << 31) - 1, 1 << 31, 1 << 32, (1 << 32) + 5):
        ctx.attention(c, x, x.clone(), b, 1.0, window=window)
    assert seen == [0, 5] + [(1 << 31) - 1] * 4
    for window in (-1, -(1 << 32)):
        with pytest.raises(P.PalqError):
            ctx.attention(c, x, x.clone(), b, 1.0, window=window)


def test_rows_of_2_to_the_32_and_more(P):
    """(Tensors without memory of their own.)"""
    cols = (1 << 32) + 16
    with pytest.raises(P.PalqError) as e:
        P.Context(-1).quantize_rows(torch.empty(1, cols, device="meta"), torch.empty(1, cols, dtype=torch.int8, device="meta"),
                                    torch.empty(1, device="meta"))
    assert e.value.status == P.ERR_UNSUPPORTED

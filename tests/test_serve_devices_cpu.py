"""Host-only checks: the binding refuses tensors that are not on the context's device
before their addresses reach a kernel."""
import pytest
import torch


@pytest.fixture(scope="module")
def P():
    from paper_2208_01944_amd import palq
    return palq


@pytest.fixture()
def ctx(P):
    """A context that runs nothing, to the binding as if it were device 0's."""
    c = P.Context(-1)
    c.device = 0
    return c


def z(*s, d=torch.float32):
    return torch.zeros(*s, dtype=d)


def test_host_tensors_are_refused(P, ctx):
    i8, i32, bf = torch.int8, torch.int32, torch.bfloat16
    cache = P.Cache(z(2, 1, 16, 64, d=i8), z(2, 1, 64, 16, d=i8), z(2, 1), z(2, 1))
    b = P.Batch(z(2, 3, d=i32), z(2, d=i32), z(3, d=i32), 4, 32)
    x = z(4, 1, 64, d=bf)
    quiet = P.Context(-1)
    lin = P.Linear(quiet, z(8, 16, d=i8), z(8), max_rows=4)
    for call in (lambda c: c.cache_append(cache, x, x, b), lambda c: c.cache_read(cache, x, x.clone(), b),
                 lambda c: c.attention(cache, x, x.clone(), b, 1.0), lambda c: c.quantize_rows(z(4, 16), z(4, 16, d=i8), z(4)),
                 lambda c: P.Linear(c, z(8, 16, d=i8), z(8), z(8), max_rows=4)):
        call(quiet)
        with pytest.raises(P.PalqError, match="device|cuda:0"):
            call(ctx)
    lin.run(z(4, 16), z(4, 8))
    lin.ctx = ctx
    with pytest.raises(P.PalqError, match="cuda:0"):
        lin.run(z(4, 16), z(4, 8))


class Elsewhere(torch.Tensor):
    """A host tensor that says it is on device 1."""

    def get_device(self):
        return 1


def test_parts_of_a_cache_or_batch_on_two_devices(P):
    i8, i32 = torch.int8, torch.int32
    for make, ok in ((P.Cache, (z(2, 1, 16, 64, d=i8), z(2, 1, 64, 16, d=i8), z(2, 1), z(2, 1))),
                     (lambda *t: P.Batch(*t, 4, 32), (z(2, 3, d=i32), z(2, d=i32), z(3, d=i32)))):
        assert make(*ok).device == -1
        for i in range(len(ok)):
            with pytest.raises(P.PalqError, match="devices"):
                make(*(t.as_subclass(Elsewhere) if j == i else t for j, t in enumerate(ok)))

"""runtime.Exchange hands the library buffers of the sizes that its kernels read and write (without a GPU: a handle that
only notes what it is given)."""
import numpy as np
import pytest
import torch

from paper_2111_08274_b200 import binding, runtime, workloads


class Handle:
    """Takes the calls of an exchange; fills the products with numbers that tell their places."""

    def __init__(self):
        self.calls = []

    def pack(self, ids, messages, **kw):
        self.calls.append(("pack", list(ids), messages, kw))

    def aggregate_packed(self, ids, messages, **kw):
        self.calls.append(("aggregate", list(ids), messages, kw))

    def integrate(self, *args):
        self.calls.append(("integrate", *args))

    def packed_dots(self, ids, messages, out):
        self.calls.append(("dots", list(ids), messages, out))


class Stream:
    def synchronize(self):
        pass


class Arena:
    def __init__(self, n, p, k, **kw):
        self.wl = workloads.Workload("exchange", n, p, k, 5, "uniform", steps_lo=0, steps_hi=3, **kw)
        self.device, self.stream, self.h = torch.device("cpu"), Stream(), Handle()
        self.stride, self.ids = -(-p // 32) * 32, np.arange(n, dtype=np.int32)
        self.w = torch.arange(n * self.stride, dtype=torch.float32).view(n, self.stride)


@pytest.fixture(autouse=True)
def _no_streams(monkeypatch):
    from paper_2111_08274_b200 import build
    build.build()
    monkeypatch.setattr(runtime.torch.cuda, "stream", lambda s: torch.no_grad())
    before = torch.get_default_dtype()
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("default", [torch.float32, torch.float64, torch.float16, torch.bfloat16])
def test_buffers_do_not_follow_the_default_dtype(default):
    torch.set_default_dtype(default)
    arena = Arena(4, 1003, 2)
    x = runtime.Exchange(arena)
    assert x.residual.dtype == torch.float32 and x.residual.shape == (4, arena.stride) and x.residual.is_contiguous()
    assert x.messages.dtype == torch.uint8 and x.messages.shape == (4, binding.hadfl_packed_bytes(1003))
    assert x.base.dtype == arena.w.dtype and x.base.shape == (1003,)
    assert x.products.dtype == torch.float32
    assert x.read_products().dtype == np.float32

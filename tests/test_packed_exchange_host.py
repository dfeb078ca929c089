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


@pytest.mark.parametrize("n,k,selected", [(5, 2, [4, 0, 1, 3, 2]), (5, 2, [3, 1, 0]), (4, 3, [2]), (4, 3, [1, 2]), (3, 3, [0, 2, 1]),
                                          (6, 1, np.array([5, 2, 0], np.int32))])
def test_products_of_any_number_of_selected_devices(n, k, selected):
    """hadfl_packed_dots writes m x m floats in rows of m for m ids: they are inside the exchange's buffer, and
    `products` and read_products() are those m x m, whatever the number of devices that the workload selects."""
    arena = Arena(n, 100, k)
    x = runtime.Exchange(arena)
    assert x.products.shape == (k, k)
    m = len(selected)
    for r in range(2):
        x.synchronise(selected, r)
        name, ids, messages, out = arena.h.calls[-1]
        assert name == "dots" and ids == list(selected) and messages == x.messages.data_ptr()
        assert x.products.data_ptr() == out and x.products.shape == (m, m) and x.products.is_contiguous()
        room = x.products.untyped_storage()
        assert room.data_ptr() <= out and out + 4 * m * m <= room.data_ptr() + room.nbytes()
        got = x.read_products()
        assert got.shape == (m, m) and got.dtype == np.float32


def test_what_the_library_refuses_leaves_the_products():
    arena = Arena(3, 100, 2)
    x = runtime.Exchange(arena)

    def refuse(ids, messages, **kw):
        raise binding.HadflError("hadfl_pack", binding.ERR_INVALID)
    arena.h.pack = refuse
    for selected in ([0, 1, 2, 0], [], [0, 1, 2, 3, 4]):
        with pytest.raises(binding.HadflError):
            x.synchronise(selected, 0)
    assert arena.h.calls == [] and x.products.shape == (2, 2)

"""Calls of the messages one after the other with nothing in between: their kernels may start under the one before, whose
writes they read.  The same calls with the GPU waited for after each have to give the same."""
import numpy as np
import pytest
import torch

from paper_2111_08274_b200 import binding
from test_gpu_packed import Side, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def rounds_of_calls(n, p, storage, rounding, wait):
    """Rounds of pack, unpack (by a receiver in the same stream), aggregate and products: each call reads what the one
    before it wrote, and all but the residuals are overwritten every time."""
    stream = torch.cuda.Stream()
    s, receiver = (Side(n, p, storage, seed=12, stream=stream) for _ in range(2))
    rng = np.random.default_rng([n, p])
    s.rows((1e-2 * rng.standard_normal((n, p))).astype(np.float32))
    base, _ = s.base((1e-2 * rng.standard_normal(p)).astype(np.float32))
    k = n - 1
    out = torch.zeros((120, k, k), device="cuda")
    torch.cuda.synchronize()

    def done():
        if wait:
            stream.synchronize()
    for r in range(out.shape[0]):
        sel = rng.permutation(n)[:k]
        if r % 10 == 9:
            s.h.local_step(range(n), np.full(n, 2), 1e-2)
            done()
        s.h.pack(sel, s.messages.data_ptr(), base_ptr=base.data_ptr(), residual_ptr=s.residual.data_ptr(), rounding=rounding,
                 round_=r)
        done()
        receiver.h.unpack(sel, s.messages.data_ptr(), base_ptr=base.data_ptr())
        done()
        s.h.packed_dots(sel, s.messages.data_ptr(), out[r].data_ptr())
        done()
        s.h.aggregate_packed(sel, s.messages.data_ptr(), base_ptr=base.data_ptr(), dst_ids=sel[:2], move_base=r % 3 == 0)
        done()
    s.check_guards() if wait else s.h.synchronize()
    return [s.w, receiver.w, s.messages.clone(), s.residual, base, out]


@pytest.mark.parametrize("n,p", [(3, 33), (4, 2003), (8, 20_001), (5, 400_003)])
@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("rounding", [binding.ROUND_NEAREST, binding.ROUND_STOCHASTIC])
def test_calls_one_after_the_other(n, p, storage, rounding):
    want = rounds_of_calls(n, p, storage, rounding, True)
    # rows that no message was read into are as the receiver's initial model left them: the same seed, the same values
    for _ in range(3):
        for x, y in zip(rounds_of_calls(n, p, storage, rounding, False), want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # (an update may be 0 throughout: the base moves to what two devices have, and local steps come every tenth round)
    assert bool(torch.all(torch.isfinite(want[0].float()))) and bool(torch.all(torch.diagonal(want[5], dim1=1, dim2=2) >= 0))


@pytest.mark.parametrize("selected", [[2, 0, 1, 4, 3], [4, 1, 3], [0]])
def test_products_of_an_exchange_with_more_or_fewer_devices_than_the_workload_selects(selected):
    import packed_reference as ref
    from paper_2111_08274_b200 import runtime, workloads
    wl = workloads.Workload("products", 5, 1003, 2, 3, "uniform", steps_lo=1, steps_hi=3, grad_std=1e-2, seed=19)
    arena = runtime.Arena(wl)
    exchange = runtime.Exchange(arena, binding.ROUND_NEAREST)
    arena.h.local_step(arena.ids, wl.steps_for_round(0), wl.lr)
    exchange.synchronise(selected, 0)
    got = exchange.read_products()
    d = np.stack([ref.values(*ref.from_bytes(exchange.messages[i].cpu().numpy(), 1003), 1003) for i in selected])
    # one sum of 1003 products in fp32: 16 steps of 64 products, 2^-23 each at most, and as much within a step's 64 products
    assert got.shape == (len(selected),) * 2 and np.all(np.diag(got) > 0)
    assert np.all(np.abs(got - d @ d.T) <= (16 + 64) * 2.0**-23 * (np.abs(d) @ np.abs(d).T))
    arena.h.debug_check()
    arena.close()

"""Messages of vectors long enough that a block walks over several devices, against the definition on whole rows
(packed_reference_rows.py): every code, scale, residual and read value."""
import numpy as np
import pytest
import torch

import packed_reference_rows as rows
from gpu_common import require_gpu
from test_gpu_packed import Side

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def length(storage, blocks_per_sm):
    """An odd length with that many blocks of columns (256 threads with 32 bytes of a row each) per SM, and 3."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return (int(blocks_per_sm * sms) + 3) * 256 * (16 if storage == "bf16" else 8) - 61


def same(got, want, what):
    got, want = got.contiguous(), want.contiguous()
    off = ((got.view(torch.int32) != want.view(torch.int32)) & ~(got.isnan() & want.isnan())).nonzero()
    assert off.numel() == 0, (what, off.numel(), off[:4].tolist())


# From two blocks of columns per SM on, a block takes all devices of its columns; with 1.6 the devices are in parts of 3, 3 and 2
# (four blocks per SM are wanted, hence three parts of eight); with 0.9 in parts of 2, 2, 2 and 1 of seven.
SHAPES = [(2, 5, 7), (1.6, 8, 9), (0.9, 7, 7), (4.5, 2, 3)]


@pytest.mark.parametrize("blocks_per_sm,k,n", SHAPES)
@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("with_base", [False, True])
@pytest.mark.parametrize("with_residual", [False, True])
def test_pack_several_rows_per_block(blocks_per_sm, k, n, storage, rounding, with_base, with_residual):
    p = length(storage, blocks_per_sm)
    seed = 1000 + 2**40 * k
    s = Side(n, p, storage, seed=seed, pad=64)
    g = torch.Generator(device="cuda").manual_seed(p)

    def values(*shape):
        return torch.randn(shape, generator=g, device="cuda") * torch.exp(2 * torch.randn(shape, generator=g, device="cuda"))
    s.w[:, :p] = 1e-2 * values(n, p)
    places = torch.randint(p, (n, 300), generator=g, device="cuda")
    odd = torch.tensor([0.0, float("inf"), -float("inf"), float("nan"), 3e38, -2.5e38, 1e-40, -0.0], device="cuda").to(s.dtype)
    for i in range(n):
        s.w[i, places[i]] = odd[torch.arange(300, device="cuda") % 8]
    base = (1e-2 * values(p)).to(s.dtype) if with_base else None
    residual = None
    if with_residual:
        s.residual.fill_(123.0)
        s.residual[:, :p] = 1e-3 * values(n, p)
        residual = s.residual.clone()
    kept = s.w.clone()
    ids = [int(i) for i in np.random.default_rng(k).permutation(n)[:k]]
    round_ = (3 << 34) + 2
    s.h.pack(ids, s.messages.data_ptr(), base_ptr=None if base is None else base.data_ptr(),
             residual_ptr=s.residual.data_ptr() if with_residual else None, rounding=rounding, round_=round_)
    s.check_guards()
    assert torch.equal(s.w.view(torch.uint8), kept.view(torch.uint8))
    scales_at = -(-(-(-p // 32) * 16) // 128) * 128
    sent = {}
    for i in range(n):
        if i not in ids:
            assert bool((s.messages[i] == 0xA5).all())
            if with_residual:
                assert torch.equal(s.residual[i], residual[i])
            continue
        u = rows.to_send(s.w[i, :p], base, None if residual is None else residual[i, :p])
        bits = rows.random_bits(seed, i, round_, p, "cuda") if rounding else None
        codes, scales, sent[i] = rows.message(u, bits)
        want = rows.to_bytes(codes, scales, scales_at, s.bytes)
        off = (s.messages[i] != want).nonzero()
        assert off.numel() == 0, (i, off.numel(), off[:4].tolist())
        if with_residual:
            same(s.residual[i, :p], rows.residual_after(u, sent[i]), i)
            assert bool((s.residual[i, p:] == 123.0).all())
    # read by a receiver with rows of its own
    t = Side(n, p, storage, pad=32)
    t.w.fill_(9.0)
    t.h.unpack(ids, s.messages.data_ptr(), base_ptr=None if base is None else base.data_ptr())
    t.check_guards()
    for i in range(n):
        assert bool((t.w[i, p:] == 9.0).all())
        if i in ids:
            x = sent[i] if base is None else base.float() + sent[i]
            same(t.w[i, :p].float(), x.to(t.dtype).float(), i)
        else:
            assert bool((t.w[i] == 9.0).all())

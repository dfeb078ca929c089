"""The whole-row form of the messages' definition against the one that goes through single elements."""
import numpy as np
import pytest
import torch

import packed_reference as ref
import packed_reference_rows as rows


def special(rng, p):
    u = (np.exp(rng.normal(0, 6, p)) * rng.standard_normal(p)).astype(np.float32)
    at = rng.permutation(p)[:p // 20]
    u[at] = rng.choice(np.array([0.0, -0.0, 6.0, 5.0, -0.75, 2.5, 1e-45, -1e-40, 1.5 * 2.0**-125, np.nextafter(np.float32(6), np.float32(7)),
                                 1.5 * 2.0**127, 3e38, -3e38, np.inf, np.nan, 0.25, 3.5], np.float32), len(at))
    return u


@pytest.mark.parametrize("p", [1, 31, 32, 33, 1003, 9001])
@pytest.mark.parametrize("stochastic", [False, True])
def test_same_messages(p, stochastic):
    rng = np.random.default_rng([p, stochastic])
    for turn, u in enumerate((special(rng, p), (1e-3 * rng.standard_normal(p)).astype(np.float32),
                              (0.25 * rng.integers(-24, 25, p)).astype(np.float32))):
        bits = ref.random_bits(5 + (turn << 40), 3, (9 << 32) + turn, p) if stochastic else None
        codes, scales = ref.message(u, bits)
        got = rows.message(torch.from_numpy(u), None if bits is None else torch.from_numpy(bits))
        assert np.array_equal(got[0].numpy(), codes) and np.array_equal(got[1].numpy(), scales)
        used, at, blocks, size = ref.sizes(p)
        assert np.array_equal(rows.to_bytes(got[0], got[1], at, size).numpy(), ref.to_bytes(codes, scales, p))
        want = ref.values(codes, scales, p).astype(np.float32)
        assert np.array_equal(got[2].numpy(), want, equal_nan=True)
        left = rows.residual_after(torch.from_numpy(u), got[2]).numpy()
        assert np.array_equal(left, ref.residual_after(u, codes, scales))


def test_same_random_bits():
    for seed, device, round_, p in ((1, 0, 0, 1), (2**63 - 3, 31, 2**56 - 1, 1000), (77, 4, (1 << 33) + 5, 801)):
        assert np.array_equal(rows.random_bits(seed, device, round_, p).numpy(), ref.random_bits(seed, device, round_, p))


def test_same_differences():
    rng = np.random.default_rng(1)
    w, b, e = ((rng.standard_normal(500) * 10.0**k).astype(np.float32) for k in (0, 0, -3))
    t = torch.from_numpy
    assert np.array_equal(rows.to_send(t(w), t(b), t(e)).numpy(), ref.to_send(w, b, e))
    assert np.array_equal(rows.to_send(t(w), None, t(e)).numpy(), ref.to_send(w, None, e))
    assert np.array_equal(rows.to_send(t(w)).numpy(), ref.to_send(w))

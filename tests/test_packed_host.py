"""Messages of 4 bits per parameter: the layout, the reference that the GPU tests use, and refusals, without a GPU."""
import ctypes as C

import numpy as np
import pytest

import packed_reference as ref
from paper_2111_08274_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2111_08274_b200 import build
    build.build()
    return binding.lib()


@pytest.mark.parametrize("p", [1, 2, 31, 32, 33, 255, 256, 257, 4095, 4096, 4097, 100_000, 11_173_962, 2**34 - 4])
def test_layout(lib, p):
    used, at, blocks, size = ref.sizes(p)
    assert binding.hadfl_packed_scales_at(p) == at and binding.hadfl_packed_bytes(p) == size
    assert at % 128 == 0 and size % 128 == 0 and used <= at and at + blocks <= size


def test_layout_of_no_vector(lib):
    for p in (0, -1, 2**34 - 3):
        assert binding.hadfl_packed_bytes(p) == 0 and binding.hadfl_packed_scales_at(p) == 0


def test_reference_scales_are_the_smallest_that_cut_nothing_off():
    for most in (6.0, np.nextafter(np.float32(6), np.float32(7)), 5.999, 0.75, 0.7500001, 3e-38, 2.5e38, 1e-45):
        s = ref.scale_exponent(np.float32(most))
        assert float(np.float32(most)) <= 6.0 * 2.0**s
        assert s == -127 or float(np.float32(most)) > 6.0 * 2.0**(s - 1)
        assert s <= 125


def test_reference_rounds_to_nearest_ties_to_even():
    y = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], np.float32)
    codes, scales = ref.message(y)
    assert list(codes[:8]) == [0, 2, 2, 4, 4, 6, 6, 7] and scales[0] == 127
    codes, _ = ref.message(-y)
    assert list(codes[:8]) == [8, 10, 10, 12, 12, 14, 14, 15]


def test_reference_stochastic_rounding_is_right_on_average():
    """Over all 2^16 random words the mean of a rounded value is the value, to the 2^-16 of a spacing that they resolve."""
    for y, low, high in ((0.3, 0.0, 0.5), (1.2, 1.0, 1.5), (2.75, 2.0, 3.0), (4.1, 4.0, 6.0)):
        ups = sum(int(np.floor((np.float32(y) - low) / (high - low) * 65536) + r >= 65536) for r in range(65536))
        assert abs(low + (high - low) * ups / 65536 - y) <= (high - low) / 65536 + 1e-6


def test_reference_random_bits_are_the_oracles_generator(oracle):
    want = oracle.philox4x32_10([5, 7, 3, 0x51000000], [11, 0])
    assert ref.philox((5, 7, 3, 0x51000000), (11, 0)) == [int(w) for w in want]


def test_reference_bytes_round_trip():
    rng = np.random.default_rng(3)
    for p in (1, 31, 64, 1000):
        raw = ref.random_message(rng, p)
        assert np.array_equal(ref.to_bytes(*ref.from_bytes(raw, p), p), raw)


def _calls(lib, h, ids, n, msg, base=None, dst=None, n_dst=0):
    i32 = C.POINTER(C.c_int32)
    p = None if ids is None else np.asarray(ids, np.int32).ctypes.data_as(i32)
    d = None if dst is None else np.asarray(dst, np.int32).ctypes.data_as(i32)
    return [lib.hadfl_pack(h, p, n, base, None, 0, 0, msg), lib.hadfl_unpack(h, p, n, base, msg),
            lib.hadfl_aggregate_packed(h, p, n, None, base, 0, d, n_dst, msg),
            lib.hadfl_packed_dots(h, p, n, msg, None, 0, None, msg)]


def test_no_handle_is_refused(lib):
    assert _calls(lib, None, [0], 1, None) == [binding.ERR_INVALID] * 4


def test_refusals_that_need_no_gpu(lib):
    """On a machine without a driver hadfl_init still hands out a handle; what the calls check of their arguments they
    check before any CUDA call, and a pointer that is not device memory is refused too."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the GPU tests make these refusals with a working handle")
    cfg = binding.hadfl_config(4, 1000, 0, 0.9, 0.0, 1e-3, 0.05, 1, 1.0, 0, None, None, 0, None, 0, 0)
    h = C.c_void_p()
    assert lib.hadfl_init(C.byref(cfg), C.byref(h)) == binding.ERR_CUDA
    buffer = np.zeros(1 << 16, np.uint8)
    at = buffer.ctypes.data + -buffer.ctypes.data % 16
    for ids, n in (([0, 1], 2), (None, 1), ([0], 0), ([0], -1), ([4], 1), ([-1], 1), ([0] * 5, 5)):
        assert _calls(lib, h, ids, n, at) == [binding.ERR_INVALID] * 4, (ids, n)
    lib.hadfl_destroy(h)

"""Products of messages on dense data long enough for every part of their kernel: stages of the ring used again, both
accumulators, many sums in 64 bits, one set and two; and at the ends of the range of scales."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_common import require_gpu
from paper_2111_08274_b200 import binding
from test_gpu_packed import Side

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def sm_count():
    return torch.cuda.get_device_properties(0).multi_processor_count


def tile_parameters(rows):
    """Parameters that a tile of the products holds of each message: four times as many pieces of 256 as `rows` fit into 32."""
    return 4 * (32 // rows) * 256


class Long:
    """N messages and a handle for them (the smallest arenas that it takes: bf16)."""

    def __init__(self, n, p):
        self.n, self.p, self.size, self.at = n, p, binding.hadfl_packed_bytes(p), binding.hadfl_packed_scales_at(p)
        self.blocks = -(-p // 32)
        stride = -(-p // 32) * 32
        self.w, self.m = (torch.zeros((n, stride), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.h = binding.Hadfl(n, p, dtype=1, m_dtype=1, w_ptr=self.w.data_ptr(), m_ptr=self.m.data_ptr(),
                               row_stride_elems=stride, init_std=0.0, stream=torch.cuda.current_stream().cuda_stream)

    def messages(self, seed, signs, magnitudes):
        """Dense random messages: `magnitudes` are the codes to draw from, scales 1 or 2."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        out = torch.zeros((self.n, self.size), dtype=torch.uint8, device="cuda")
        pool = torch.tensor(magnitudes, dtype=torch.uint8, device="cuda")
        for i in range(self.n):
            def codes():
                c = pool[torch.randint(len(magnitudes), (16 * self.blocks,), generator=g, device="cuda")]
                return c + 8 * torch.randint(2, c.shape, generator=g, device="cuda", dtype=torch.uint8) if signs else c
            low, high = codes(), codes()
            low[(self.p + 1) // 2:] = 0
            high[self.p // 2:] = 0
            out[i, :16 * self.blocks] = low | (high << 4)
            out[i, self.at:self.at + self.blocks] = 127 + torch.randint(2, (self.blocks,), generator=g, device="cuda",
                                                                        dtype=torch.uint8)
        return out

    def values(self, messages, ids, first, end):
        """Blocks first .. end of the listed messages, fp64."""
        table = torch.tensor(np.concatenate([ref.GRID, -ref.GRID]), device="cuda")
        raw = messages[:, 16 * first:16 * end][ids].int()
        v = torch.stack((table[raw & 15], table[raw >> 4]), dim=-1).reshape(len(ids), -1, 32)
        scale = torch.exp2(messages[:, self.at + first:self.at + end][ids].double() - 127)
        return (v * scale[..., None]).reshape(len(ids), -1)

    def reference(self, a, ia, b, ib):
        """Products in 64 bits: all terms and sums are multiples of 1/4 below 2^50, so that they are exact in any order."""
        want = torch.zeros((len(ia), len(ib)), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 25) // (32 * max(len(ia), len(ib))))
        for first in range(0, self.blocks, step):
            end = min(first + step, self.blocks)
            x = self.values(a, ia, first, end)
            want += x @ (x if b is a and list(ia) == list(ib) else self.values(b, ib, first, end)).T
        return want


def check(s, a, ia, b=None, ib=None):
    """Equality: codes up to 3 and scales of 1 and 2 make terms of up to 36, all multiples of 1/4, so that a sum over the 2^14
    parameters after which it goes to 64 bits is below 2^22 quarters and exact in fp32; so is the 64-bit sum.  What is left
    is one rounding to fp32, in the kernel and here."""
    m, n = len(ia), len(ia if ib is None else ib)
    out = torch.full((m * n + 2,), -7.0, device="cuda")
    s.h.packed_dots(ia, a.data_ptr(), out[1:].data_ptr(), b_ids=ib, b_messages_ptr=None if b is None else b.data_ptr())
    s.h.synchronize()
    s.h.debug_check()
    want = s.reference(a, ia, a if b is None else b, ia if ib is None else ib).float()
    assert out[0] == -7 and out[-1] == -7
    got = out[1:-1].view(m, n)
    off = (got != want).nonzero()
    assert len(off) == 0, (len(off), [(i, j, float(got[i, j]), float(want[i, j])) for i, j in off[:4].tolist()])


SMALL = [0, 1, 2, 3, 4, 5]     # values up to 3


def length(rows, tiles, some):
    """A vector of which `some` blocks of the grid get `tiles` tiles and the others one less; its last tile is not full."""
    return ((tiles - 1) * sm_count() + some) * tile_parameters(rows) - 77


@pytest.mark.parametrize("tiles", [2, 7, 8, 9, 10, 17, 127, 128, 129, 130, 257])
@pytest.mark.parametrize("rows", [32, 17, 8, 5])
def test_one_set_of_dense_messages(rows, tiles):
    s = Long(rows, length(rows, tiles, 1 + tiles % 100))
    a = s.messages(tiles, tiles % 2 == 0, SMALL)
    check(s, a, np.random.default_rng(tiles).permutation(rows))


@pytest.mark.parametrize("tiles", [2, 3, 4, 5, 6, 9, 127, 128, 129, 130, 257])
@pytest.mark.parametrize("m,n", [(32, 32), (17, 32), (8, 3), (2, 5)])
def test_two_sets_of_dense_messages(m, n, tiles):
    rows = max(m, n)
    s = Long(rows, length(rows, tiles, 1 + tiles % 100))
    a, b = (s.messages(2 * tiles + i, tiles % 2 == 0, SMALL) for i in range(2))
    rng = np.random.default_rng(tiles)
    check(s, a, rng.permutation(rows)[:m], b, rng.integers(0, rows, n))


@pytest.mark.parametrize("m,n,shift", [(6, 6, 0), (6, 6, 3), (4, 6, 1), (6, 2, 5)])
def test_two_sets_that_share_messages(m, n, shift):
    """The same messages in another order, and two windows of one buffer: each set has its own ids."""
    s = Long(6, 50_021)
    both = torch.cat([s.messages(m, True, SMALL), s.messages(n, True, SMALL)])
    check(s, both[:6], list(range(m)), both[shift:shift + 6], list(range(n))[::-1])


@pytest.mark.parametrize("two", [False, True])
def test_sums_that_fp32_could_not_hold(two):
    """Nearly all values 3 or 6, of one sign: after some 460 tiles of an accumulator a sum that stayed in fp32 would be beyond
    2^24 quarters and lose its last bits."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    s = Long(32, length(32, 1100, 9))
    codes = [5] * 15 + [1]
    a = s.messages(1, False, codes)
    check(s, a, np.arange(32), *((s.messages(2, False, codes), np.arange(32)) if two else ()))


# ---- the ends of the range -------------------------------------------------------------------------------------------
def products(a, b, n):
    out = torch.zeros((n, n), device="cuda")
    a.h.packed_dots(range(n), a.messages.data_ptr(), out.data_ptr(), b_ids=range(n), b_messages_ptr=b.messages.data_ptr())
    a.check_guards()
    return out.cpu().numpy()


def fill(s, rng, low, high):
    raws = [ref.random_message(rng, s.p, low, high) for _ in range(s.n)]
    for i, raw in enumerate(raws):
        s.set_message(i, raw)
    return np.stack([ref.values(*ref.from_bytes(raw, s.p), s.p) for raw in raws])


@pytest.mark.parametrize("p", [32, 1000, 9001])
def test_products_of_the_smallest_scales_with_the_largest(p):
    """Scale bytes 0 to 2 (2^-127 to 2^-125) times 250 to 252, the largest that hadfl_pack writes: ordinary products.  The
    tolerance is the one that is derived for all sums: 320 steps that lose 2^-23 of the magnitudes each."""
    rng = np.random.default_rng(p)
    a, b = Side(3, p), Side(3, p)
    x, y = fill(a, rng, 0, 3), fill(b, rng, 250, 253)
    assert np.all(np.abs(products(a, b, 3) - x @ y.T) <= 320 * 2.0**-23 * (np.abs(x) @ np.abs(y).T))


@pytest.mark.parametrize("high", [3, 25])
def test_products_below_all_numbers_are_zero(high):
    """All terms are below 36 * 2^-206 and their sums below 2^-150, half the smallest number of fp32."""
    rng = np.random.default_rng(high)
    a, b = Side(4, 5000), Side(4, 5000)
    fill(a, rng, 0, high)
    fill(b, rng, 0, high)
    assert np.all(products(a, b, 4) == 0)


@pytest.mark.parametrize("low", [55, 60, 64])
def test_products_among_the_subnormal_numbers(low):
    """Terms around 2^(2 low - 254), some below and some above 2^-126.  Each of p terms and sums may lose all that is below that
    (2^-126 at most, flushed to zero) on top of what all sums may lose."""
    rng = np.random.default_rng(low)
    a, b = Side(4, 3000), Side(4, 3000)
    x, y = fill(a, rng, low, low + 2), fill(b, rng, low, low + 2)
    err = np.abs(products(a, b, 4) - x @ y.T)
    assert np.all(err <= 320 * 2.0**-23 * (np.abs(x) @ np.abs(y).T) + 3000 * 2.0**-126)


def one_value(s, device, at, code, byte):
    """Adds a parameter to a message."""
    codes, scales = ref.from_bytes(s.message(device), s.p)
    codes[at], scales[at // 32] = code, byte
    s.set_message(device, ref.to_bytes(codes, scales, s.p))


def test_products_that_overflow():
    """A term, or a sum of terms, above the largest number of fp32 is an infinity of its sign; infinities of both signs are no
    number; and other messages' products are as they would be without."""
    p = 70_001
    s = Side(8, p)
    s.messages.zero_()
    far = [5, 20_000, 40_000, 69_990]
    one_value(s, 0, far[0], 7, 252)            # 6 * 2^125
    one_value(s, 1, far[0], 15, 252)           # -6 * 2^125
    one_value(s, 1, far[1], 7, 252)
    one_value(s, 2, far[0], 2, 190)            # 2^63: with itself 2^126, eight of them 2^129
    for k in range(1, 8):
        one_value(s, 2, 9000 * k + 1, 2, 190)
    one_value(s, 3, far[2], 2, 190)            # alone: 2^126
    one_value(s, 4, far[0], 7, 252)            # with device 0 at far[0] above all numbers, at far[1] below
    one_value(s, 4, far[1], 15, 252)
    one_value(s, 5, far[0], 2, 127)            # 1
    one_value(s, 6, far[3], 3, 127)            # 1.5
    one_value(s, 7, far[0], 7, 252)
    one_value(s, 7, far[1], 7, 252)
    out = torch.zeros((8, 8), device="cuda")
    s.h.packed_dots(range(8), s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    got = out.cpu().numpy()
    inf, most, near = np.inf, 6 * 2.0**125, 2.0**63
    want = np.array([
        [inf, -inf, inf, 0, inf, most, 0, inf],
        [-inf, inf, -inf, 0, -inf, -most, 0, np.nan],
        [inf, -inf, inf, 0, inf, near, 0, inf],
        [0, 0, 0, 2.0**126, 0, 0, 0, 0],
        [inf, -inf, inf, 0, inf, most, 0, np.nan],
        [most, -most, near, 0, most, 1, 0, most],
        [0, 0, 0, 0, 0, 0, 2.25, 0],
        [inf, np.nan, inf, 0, np.nan, most, 0, inf]])
    assert np.array_equal(got, want.astype(np.float32), equal_nan=True), got


def test_a_sum_above_all_numbers_whose_parts_are_not():
    """Two terms of 2^127 in pieces whose sums meet in 64 bits only."""
    p = 200_000
    s = Side(1, p)
    s.messages.zero_()
    for at in (3, 150_000):
        one_value(s, 0, at, 2, 190)
        one_value(s, 0, at + 40, 2, 190)       # another block: 2 * 2^126 = 2^127 in the piece
    out = torch.zeros((1, 1), device="cuda")
    s.h.packed_dots([0], s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    assert float(out) == np.inf

"""Messages of 4 bits per parameter on the GPU against their definition (packed_reference.py): quantisation, reading,
aggregation and scalar products, at the sizes, values and arguments where they can go wrong."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_common import require_gpu
from paper_2111_08274_b200 import binding

pytestmark = pytest.mark.gpu

GUARD = 512            # bytes on either side of the messages that no call may touch
STORAGE = {"fp32": binding.DTYPE_FP32, "bf16": binding.DTYPE_BF16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Side:
    """A handle over tensors of its own, with messages, a base and residuals."""

    def __init__(self, n, p, storage="fp32", seed=77, stream=None, pad=0, weight_mode=0, shift=0):
        """shift: elements by which arena, residuals and messages begin behind a multiple of 512 bytes."""
        self.n, self.p, self.seed = n, p, seed
        self.stride = -(-p // 32) * 32 + pad
        self.dtype = torch.bfloat16 if storage == "bf16" else torch.float32
        self.stream = stream or torch.cuda.current_stream()
        with torch.cuda.stream(self.stream):
            self.w = torch.zeros(n * self.stride + shift, dtype=self.dtype, device="cuda")[shift:].view(n, self.stride)
            self.m = torch.zeros((n, self.stride), dtype=torch.float32, device="cuda")
            self.h = binding.Hadfl(n, p, dtype=STORAGE[storage], seed=seed, w_ptr=self.w.data_ptr(),
                                   m_ptr=self.m.data_ptr(), row_stride_elems=self.stride, weight_mode=weight_mode,
                                   stream=self.stream.cuda_stream)
            self.bytes = binding.hadfl_packed_bytes(p)
            self.raw = torch.full((n * self.bytes + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
            at = GUARD - 16 * (shift > 0)
            self.messages = self.raw[at:at + n * self.bytes].view(n, self.bytes)
            self.residual = torch.zeros(n * self.stride + 4 * (shift > 0), device="cuda")[4 * (shift > 0):].view(n, self.stride)
        self.stream.synchronize()

    def rows(self, values):
        """Sets the parameters; returns them as stored, fp32."""
        self.w[:, :self.p] = torch.from_numpy(values).to("cuda").to(self.dtype)
        return self.w[:, :self.p].float().cpu().numpy()

    def base(self, values):
        t = torch.from_numpy(values).to("cuda").to(self.dtype)
        return t, t.float().cpu().numpy()

    def check_guards(self):
        self.h.synchronize()
        self.h.debug_check()
        at = self.messages.data_ptr() - self.raw.data_ptr()
        assert torch.all(self.raw[:at] == 0xA5) and torch.all(self.raw[at + self.n * self.bytes:] == 0xA5)

    def message(self, i):
        return self.messages[i].cpu().numpy()

    def set_message(self, i, raw):
        self.messages[i] = torch.from_numpy(raw)


def bits(x):
    return np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)


def assert_same(got, want, what=""):
    """Equal bit for bit, NaNs whatever their payload."""
    got, want = np.asarray(got, np.float32), np.asarray(want, np.float32)
    off = np.flatnonzero((bits(got) != bits(want)) & ~(np.isnan(got) & np.isnan(want)))
    assert off.size == 0, (what, off.size, [(int(i), got[i], want[i]) for i in off[:4]])


def to_storage(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(dtype).float().numpy()


def check_pack(s, w, ids, base, residual, rounding, round_):
    before = None if residual is None else residual.copy()
    for i in range(s.n):
        if i not in ids:
            assert np.all(s.message(i) == 0xA5)
            if before is not None:
                assert np.array_equal(s.residual[i, :s.p].cpu().numpy(), before[i])
            continue
        u = ref.to_send(w[i], base, None if before is None else before[i])
        r = ref.random_bits(s.seed, i, round_, s.p) if rounding else None
        codes, scales = ref.message(u, r)
        raw = s.message(i)
        want = ref.to_bytes(codes, scales, s.p)
        assert np.array_equal(raw, want), (i, np.flatnonzero(raw != want)[:8])
        if before is not None:
            assert_same(s.residual[i, :s.p].cpu().numpy(), ref.residual_after(u, codes, scales), i)


SIZES = [1, 7, 31, 32, 33, 255, 257, 2049, 4096, 4101]


@pytest.mark.parametrize("p", SIZES)
@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("with_base,with_residual,rounding", [(False, False, 0), (True, True, 1), (True, False, 0), (False, True, 1),
                                                              (False, True, 0), (True, False, 1), (True, True, 0), (False, False, 1)])
def test_pack(p, storage, with_base, with_residual, rounding):
    rng = np.random.default_rng([p, with_base, with_residual, rounding])
    s = Side(4, p, storage, seed=rng.integers(1, 2**63).item(), pad=8 * (p % 3))
    size = np.exp(rng.normal(0, 3, (4, p)))
    w = s.rows((1e-2 * size * rng.standard_normal((4, p))).astype(np.float32))
    base_t, base = s.base((1e-2 * rng.standard_normal(p)).astype(np.float32)) if with_base else (None, None)
    residual = None
    if with_residual:
        residual = (1e-3 * rng.standard_normal((4, p))).astype(np.float32)
        s.residual.fill_(123.0)
        s.residual[:, :p] = torch.from_numpy(residual)
    kept = s.w.clone()
    round_ = (1 << 33) + 5
    ids = [2, 0, 3]
    s.h.pack(ids, s.messages.data_ptr(), base_ptr=base_t.data_ptr() if with_base else None,
             residual_ptr=s.residual.data_ptr() if with_residual else None, rounding=rounding, round_=round_)
    s.check_guards()
    assert torch.equal(s.w, kept)
    if with_residual:
        assert torch.all(s.residual[:, p:] == 123.0)
    check_pack(s, w, ids, base, residual, rounding, round_)


SPECIAL = [0.0, -0.0, 6.0, -6.0, 0.25, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, np.float32(5.9999995), 1e-45, -1e-40, 1.1754944e-38,
           3.0e-38, 3.4028235e38, -3.4e38, np.inf, -np.inf, np.nan, np.nextafter(np.float32(6), np.float32(7)), 2.0**-126,
           1.5 * 2.0**-125, 2.0**-127, 1.5 * 2.0**127, np.nextafter(np.float32(1.5 * 2.0**127), np.float32(np.inf)), 2.9e38]


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("residual", [False, True])
def test_pack_special_values(rounding, residual):
    """One special value per block among ordinary ones, alone in a block, and blocks full of one of them."""
    rng = np.random.default_rng(8)
    blocks = []
    for v in SPECIAL:
        a = rng.standard_normal(32).astype(np.float32)
        a[5] = v
        b = np.zeros(32, np.float32)
        b[31] = v
        blocks += [a, b, np.full(32, v, np.float32)]
    w0 = np.concatenate(blocks)[None]
    p = w0.shape[1] - 3
    s = Side(1, p)
    w = s.rows(np.ascontiguousarray(w0[:, :p]))
    s.h.pack([0], s.messages.data_ptr(), residual_ptr=s.residual.data_ptr() if residual else None, rounding=rounding, round_=3)
    s.check_guards()
    check_pack(s, w, [0], None, np.zeros((1, p), np.float32) if residual else None, rounding, 3)


def test_pack_difference_that_overflows_or_is_not_a_number():
    s = Side(1, 96)
    w0 = np.ones((1, 96), np.float32)
    w0[0, 3], w0[0, 40] = 3e38, np.inf
    b0 = np.zeros(96, np.float32)
    b0[3], b0[40] = -3e38, np.inf
    w = s.rows(w0)
    base_t, base = s.base(b0)
    s.residual.fill_(0.5)
    residual = s.residual[:, :96].cpu().numpy()
    s.h.pack([0], s.messages.data_ptr(), base_ptr=base_t.data_ptr(), residual_ptr=s.residual.data_ptr())
    s.check_guards()
    check_pack(s, w, [0], base, residual, 0, 0)
    assert torch.all(s.residual[0, :64] == 0)


def test_pack_with_a_row_of_the_arena_as_base():
    rng = np.random.default_rng(4)
    s = Side(3, 1003)
    w = s.rows(rng.standard_normal((3, 1003)).astype(np.float32))
    s.h.pack([0, 1, 2], s.messages.data_ptr(), base_ptr=s.w[1].data_ptr())
    s.check_guards()
    check_pack(s, w, [0, 1, 2], w[1], None, 0, 0)
    assert np.all(s.message(1) == 0)


def test_stochastic_messages_differ_by_round_and_device_and_average_to_the_value():
    p = 32 * 2048
    s = Side(2, p)
    w0 = np.tile(np.linspace(-6, 6, 32, dtype=np.float32), (2, p // 32))
    s.rows(w0)
    got = []
    for r in (0, 1):
        s.h.pack([0, 1], s.messages.data_ptr(), rounding=1, round_=r)
        got.append([s.message(i).copy() for i in (0, 1)])
    assert not np.array_equal(got[0][0], got[0][1]) and not np.array_equal(got[0][0], got[1][0])
    mean = ref.values(*ref.from_bytes(got[0][0], p), p).reshape(-1, 32).mean(0)
    # a value moves by at most one spacing (2): the standard deviation of the mean of 2048 is below 1 / sqrt(2048) = 0.022
    assert np.abs(mean - w0[0, :32]).max() < 5 * 0.0221


def arbitrary_messages(s, rng, special=True):
    raws = []
    for i in range(s.n):
        raw = ref.random_message(rng, s.p)
        if special:
            _, at, blocks, _ = ref.sizes(s.p)
            for j, b in enumerate((255, 0, 1, 253)):
                if blocks > 4:
                    raw[at + (3 * i + j) % blocks] = b
        s.set_message(i, raw)
        raws.append(raw)
    return raws, [ref.values(*ref.from_bytes(r, s.p), s.p) for r in raws]


@pytest.mark.parametrize("p", SIZES)
@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("base_is", ["none", "own", "row"])
def test_unpack(p, storage, base_is):
    rng = np.random.default_rng([p, 5])
    s = Side(4, p, storage, pad=16)
    raws, d = arbitrary_messages(s, rng)
    s.w.fill_(9.0)
    w = s.rows(rng.standard_normal((4, p)).astype(np.float32))
    base_t, base = (None, None) if base_is == "none" else s.base(rng.standard_normal(p).astype(np.float32))
    if base_is == "row":
        base_t, base = s.w[3], w[3]
    s.h.unpack([3, 1], s.messages.data_ptr(), base_ptr=None if base_t is None else base_t.data_ptr())
    s.check_guards()
    for i in range(4):
        want = w[i]
        if i in (1, 3):
            with np.errstate(over="ignore", invalid="ignore"):
                x = d[i].astype(np.float32)
                want = to_storage(x if base is None else (base + x).astype(np.float32), s.dtype)
        assert_same(s.w[i, :p].float().cpu().numpy(), want, i)
        assert torch.all(s.w[i, p:] == 9.0)
        assert np.array_equal(s.message(i), raws[i])


@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("n,p,which", [(32, 100_003, 0), (32, 20_000, 31), (9, 300_001, 4), (32, 1_000_003, 16)])
def test_unpack_with_a_base_that_is_written_too(n, p, which, storage):
    """All rows are base + message with the base as it was before the call, the base's own row among them."""
    rng = np.random.default_rng([n, p])
    s = Side(n, p, storage)
    raws = [ref.random_message(rng, p) for _ in range(n)]
    d = [ref.values(*ref.from_bytes(raw, p), p).astype(np.float32) for raw in raws]
    for i in range(n):
        s.set_message(i, raws[i])
    for turn in range(4):
        w = s.rows(rng.standard_normal((n, p), dtype=np.float32))
        s.h.unpack(rng.permutation(n), s.messages.data_ptr(), base_ptr=s.w[which].data_ptr())
        s.check_guards()
        got = s.w[:, :p].float().cpu().numpy()
        for i in range(n):
            assert_same(got[i], to_storage(w[which] + d[i], s.dtype), (turn, i))


def fused_multiply_add(a, d, c):
    """fl(a * d + c), rounded to fp32 once.  The product is exact in the 64 bits of a long double; where the sum is not,
    it is moved by one of its own last places towards what it left out, so that no tie of fp32 is made of it."""
    x, y = np.longdouble(a) * d.astype(np.longdouble), c.astype(np.longdouble)
    s = x + y
    t = s - x
    left = (x - (s - t)) + (y - t)
    away = np.nextafter(s, np.where(left > 0, np.longdouble(np.inf), np.longdouble(-np.inf)))
    return np.where(np.isfinite(left) & (left != 0), away, s).astype(np.float32)


def aggregate_reference(a, d, base):
    with np.errstate(over="ignore", invalid="ignore"):
        acc = (np.longdouble(a[0]) * d[0].astype(np.longdouble)).astype(np.float32)
        for j in range(1, len(d)):
            acc = fused_multiply_add(a[j], d[j], acc)
        return acc if base is None else (base + acc).astype(np.float32)


@pytest.mark.parametrize("p", SIZES)
@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("k", [1, 2, 3, 5, 8])
def test_aggregate_packed(p, storage, k):
    rng = np.random.default_rng([p, k])
    s = Side(8, p, storage, pad=8, weight_mode=k % 2)
    raws, d = arbitrary_messages(s, rng)
    s.w.fill_(9.0)
    w = s.rows(rng.standard_normal((8, p)).astype(np.float32))
    s.h.set_versions(versions=[3, 1, 4, 1, 5, 2, 6, 5])
    sel = [int(i) for i in rng.permutation(8)[:k]]
    a = s.h.aggregation_weights(sel)
    with_base, move, to_all = k != 3, k in (2, 8), k in (2, 5)
    base_t, base = s.base(rng.standard_normal(p).astype(np.float32)) if with_base else (None, None)
    s.h.aggregate_packed(sel, s.messages.data_ptr(), base_ptr=base_t.data_ptr() if with_base else None,
                         dst_ids=range(8) if to_all else None, move_base=move)
    s.check_guards()
    x = aggregate_reference(a, [d[i] for i in sel], base)
    want = to_storage(x, s.dtype)
    receivers = range(8) if to_all else sel
    for i in range(8):
        assert_same(s.w[i, :p].float().cpu().numpy(), want if i in receivers else w[i], i)
        assert torch.all(s.w[i, p:] == 9.0)
        assert np.array_equal(s.message(i), raws[i])
    if with_base:
        assert_same(base_t.float().cpu().numpy(), want if move else base)
    top = max([3, 1, 4, 1, 5, 2, 6, 5][i] for i in sel)
    assert [int(v) for v in s.h.get_versions()[0]] == [top if i in receivers else [3, 1, 4, 1, 5, 2, 6, 5][i] for i in range(8)]


def test_aggregate_packed_with_a_receivers_row_as_base():
    rng = np.random.default_rng(6)
    s = Side(4, 3001)
    _, d = arbitrary_messages(s, rng)
    w = s.rows(rng.standard_normal((4, 3001)).astype(np.float32))
    s.h.aggregate_packed([1, 3], s.messages.data_ptr(), base_ptr=s.w[3].data_ptr(), move_base=True)
    want = aggregate_reference([np.float32(0.5)] * 2, [d[1], d[3]], w[3])
    s.check_guards()
    for i, x in enumerate((w[0], want, w[2], want)):
        assert_same(s.w[i, :3001].cpu().numpy(), x, i)


@pytest.mark.parametrize("storage", ["fp32", "bf16"])
@pytest.mark.parametrize("p", [1, 40, 4099])
def test_buffers_at_odd_multiples_of_16_bytes(p, storage):
    """Arena, base, residuals and messages that begin 16 bytes behind a multiple of 32: whole calls, as above."""
    rng = np.random.default_rng([p, 9])
    shift = 8 if storage == "bf16" else 4
    s = Side(3, p, storage, pad=8, shift=shift)
    assert s.w.data_ptr() % 32 == 16 and s.residual.data_ptr() % 32 == 16 and s.messages.data_ptr() % 32 == 16
    w = s.rows((1e-2 * rng.standard_normal((3, p))).astype(np.float32))
    room = torch.zeros(p + shift, dtype=s.dtype, device="cuda")
    room[shift:] = s.base((1e-2 * rng.standard_normal(p)).astype(np.float32))[0]
    base_t = room[shift:]
    base = base_t.float().cpu().numpy()
    residual = (1e-3 * rng.standard_normal((3, p))).astype(np.float32)
    s.residual[:, :p] = torch.from_numpy(residual)
    s.h.pack([2, 0], s.messages.data_ptr(), base_ptr=base_t.data_ptr(), residual_ptr=s.residual.data_ptr(), rounding=1, round_=1)
    s.check_guards()
    check_pack(s, w, [2, 0], base, residual, 1, 1)
    d = [ref.values(*ref.from_bytes(s.message(i), p), p) for i in (0, 2)]
    s.h.unpack([0], s.messages.data_ptr(), base_ptr=base_t.data_ptr())
    s.check_guards()
    assert_same(s.w[0, :p].float().cpu().numpy(), to_storage(base + d[0].astype(np.float32), s.dtype))
    s.h.aggregate_packed([0, 2], s.messages.data_ptr(), base_ptr=base_t.data_ptr(), dst_ids=[1, 2], move_base=True)
    s.check_guards()
    want = to_storage(aggregate_reference([np.float32(0.5)] * 2, d, base), s.dtype)
    for got in (s.w[1, :p], s.w[2, :p], base_t):
        assert_same(got.float().cpu().numpy(), want)
    out = torch.zeros(5, device="cuda")[1:].view(2, 2)
    s.h.packed_dots([0, 2], s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    want, size = dots_reference(np.stack(d), np.stack(d))
    assert np.all(np.abs(out.cpu().numpy() - want) <= DOTS_TOL * size + 1e-30)


# ---- products --------------------------------------------------------------------------------------------------------
# Sums are formed in fp32 over at most 2^14 parameters at a time, then in 64 bits, and rounded to fp32 once.  A step of
# such a sum loses at most 2^-23 of the magnitudes in it (2^-24 by rounding, twice that where it drops bits instead), and
# at most 2^14 / 64 steps follow one another (64 products are added in one), after the 64 products' own additions:
# |error| <= (256 + 64) * 2^-23 * sum |a b| < 4e-5 * sum |a b|.  Errors of steps differ in sign and their sizes follow the
# sum as it grows, so the tests ask for a tenth of that.
DOTS_TOL = 4e-6


def dots_reference(x, y):
    with np.errstate(over="ignore", invalid="ignore"):
        return x @ y.T, np.abs(x) @ np.abs(y).T


@pytest.mark.parametrize("p", SIZES + [70_001])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 6, 7, 8, 9, 10, 11, 16, 17, 31, 32])
def test_products_of_one_set(p, n):
    rng = np.random.default_rng([p, n])
    s = Side(n, p)
    _, d = arbitrary_messages(s, rng, special=False)
    ids = rng.permutation(n)
    out = torch.full((n * n + 2,), -7.0, device="cuda")
    s.h.packed_dots(ids, s.messages.data_ptr(), out[1:].data_ptr())
    s.check_guards()
    x = np.stack([d[i] for i in ids])
    want, size = dots_reference(x, x)
    got = out.cpu().numpy()
    assert got[0] == -7 and got[-1] == -7
    got = got[1:-1].reshape(n, n)
    assert np.all(np.abs(got - want) <= DOTS_TOL * size + 1e-30)
    assert np.array_equal(got, got.T)


@pytest.mark.parametrize("m,n", [(1, 32), (32, 1), (3, 7), (2, 2), (16, 5), (5, 17), (10, 3), (6, 6)])
@pytest.mark.parametrize("p", [1, 95, 4096, 66_007])
def test_products_of_two_sets(p, m, n):
    rng = np.random.default_rng([p, m, n])
    a, b = Side(32, p), Side(32, p)
    _, da = arbitrary_messages(a, rng, special=False)
    _, db = arbitrary_messages(b, rng, special=False)
    ia, ib = rng.integers(0, 32, m), rng.integers(0, 32, n)       # repeated ids are fine
    out = torch.full((m, n), -7.0, device="cuda")
    a.h.packed_dots(ia, a.messages.data_ptr(), out.data_ptr(), b_ids=ib, b_messages_ptr=b.messages.data_ptr())
    a.check_guards()
    want, size = dots_reference(np.stack([da[i] for i in ia]), np.stack([db[i] for i in ib]))
    assert np.all(np.abs(out.cpu().numpy() - want) <= DOTS_TOL * size + 1e-30)


@pytest.mark.parametrize("n", [2, 4, 11, 32])
@pytest.mark.parametrize("p", [64, 1000, 300_001])
def test_products_are_exact_where_sums_fit(p, n):
    """Scale 1 throughout and one non-zero code in eight: the terms are multiples of 1/4 and the sums below 2^22."""
    rng = np.random.default_rng([p, n, 1])
    s = Side(n, p)
    _, at, blocks, _ = ref.sizes(p)
    d = []
    for i in range(n):
        codes = rng.integers(0, 16, blocks * 32).astype(np.uint8)
        codes[rng.random(blocks * 32) > 0.125] = 0
        codes[p:] = 0
        s.set_message(i, ref.to_bytes(codes, np.full(blocks, 127, np.uint8), p))
        d.append(ref.values(codes, np.full(blocks, 127), p))
    out = torch.zeros((n, n), device="cuda")
    s.h.packed_dots(range(n), s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    d = np.stack(d)
    assert np.array_equal(out.cpu().numpy(), (d @ d.T).astype(np.float32))


def test_products_of_single_parameters_and_blocks():
    """One non-zero parameter per message, at every place of two tiles' worth: a wrong place of a code or scale shows."""
    p, n = 1024, 32
    s = Side(n, p)
    _, at, blocks, _ = ref.sizes(p)
    out = torch.zeros((n, n), device="cuda")
    for first in range(0, p, n):
        d = np.zeros((n, p))
        for i in range(n):
            codes, scales = np.zeros(blocks * 32, np.uint8), np.full(blocks, 100, np.uint8)
            codes[first + i] = 1 + i % 7
            scales[(first + i) // 32] = 120 + i % 13
            s.set_message(i, ref.to_bytes(codes, scales, p))
            d[i] = ref.values(codes, scales, p)
        s.h.packed_dots(range(n), s.messages.data_ptr(), out.data_ptr())
        s.h.synchronize()
        assert np.array_equal(out.cpu().numpy(), (d @ d.T).astype(np.float32)), first


@pytest.mark.parametrize("block", [0, 3, 7, 100, 311])
def test_products_with_a_message_that_has_a_lost_block(block):
    rng = np.random.default_rng(block)
    s = Side(5, 9999)
    raws, d = arbitrary_messages(s, rng, special=False)
    raws[2][ref.sizes(9999)[1] + block] = 255
    s.set_message(2, raws[2])
    out = torch.zeros((5, 5), device="cuda")
    s.h.packed_dots(range(5), s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    got = out.cpu().numpy()
    assert np.all(np.isnan(got[2])) and np.all(np.isnan(got[:, 2]))
    rest = [0, 1, 3, 4]
    x = np.stack([d[i] for i in rest])
    want, size = dots_reference(x, x)
    assert np.all(np.abs(got[np.ix_(rest, rest)] - want) <= DOTS_TOL * size)


@pytest.mark.parametrize("low_a,low_b", [(225, 5), (3, 230), (127, 127), (200, 60), (90, 90)])
def test_products_of_far_scales(low_a, low_b):
    """Scales far from 1 whose products are not: 2^(a - 127) 2^(b - 127) with a + b near 254, or small throughout."""
    rng = np.random.default_rng([low_a, low_b])
    a, b = Side(3, 8200), Side(3, 8200)
    d = []
    for s, low in ((a, low_a), (b, low_b)):
        raws = [ref.random_message(rng, 8200, low, low + 20) for _ in range(3)]
        for i, raw in enumerate(raws):
            s.set_message(i, raw)
        d.append(np.stack([ref.values(*ref.from_bytes(raw, 8200), 8200) for raw in raws]))
    out = torch.zeros((3, 3), device="cuda")
    a.h.packed_dots(range(3), a.messages.data_ptr(), out.data_ptr(), b_ids=range(3), b_messages_ptr=b.messages.data_ptr())
    a.check_guards()
    want, size = dots_reference(*d)
    assert np.all(np.abs(out.cpu().numpy() - want) <= DOTS_TOL * size)


def test_products_do_not_read_other_devices_messages():
    """Messages of devices that are not asked for may hold anything (here: NaN blocks throughout)."""
    rng = np.random.default_rng(21)
    s = Side(8, 5000)
    _, d = arbitrary_messages(s, rng, special=False)
    for i in (0, 1, 4, 5, 6, 7):
        s.messages[i].fill_(255)
    out = torch.zeros((2, 2), device="cuda")
    s.h.packed_dots([3, 2], s.messages.data_ptr(), out.data_ptr())
    s.check_guards()
    x = np.stack([d[3], d[2]])
    want, size = dots_reference(x, x)
    assert np.all(np.abs(out.cpu().numpy() - want) <= DOTS_TOL * size)


def test_products_are_reproducible():
    rng = np.random.default_rng(22)
    s = Side(8, 1_000_003)
    for i in range(8):
        s.set_message(i, ref.random_message(rng, s.p))
    got = []
    for _ in range(3):
        out = torch.zeros((8, 8), device="cuda")
        s.h.packed_dots(range(8), s.messages.data_ptr(), out.data_ptr())
        s.h.synchronize()
        got.append(out.cpu().numpy())
    assert np.array_equal(got[0], got[1]) and np.array_equal(got[0], got[2])


# ---- refusals, graphs, streams, runs ---------------------------------------------------------------------------------
def test_refusals():
    s = Side(4, 1000)
    before, launches = s.w.clone(), s.h.launch_count()
    ok = s.messages.data_ptr()
    host = torch.zeros(1 << 16, dtype=torch.uint8)
    base = torch.zeros(1000, device="cuda")
    out = torch.zeros((4, 4), device="cuda")
    e = s.residual.data_ptr()
    bad = [lambda: s.h.pack([0, 0], ok), lambda: s.h.pack([4], ok), lambda: s.h.pack([-1], ok), lambda: s.h.pack([], ok),
           lambda: s.h.pack([0], None), lambda: s.h.pack([0], ok + 8), lambda: s.h.pack([0], host.data_ptr()),
           lambda: s.h.pack([0], ok, rounding=2), lambda: s.h.pack([0], ok, rounding=-1), lambda: s.h.pack([0], ok, round_=-1),
           lambda: s.h.pack([0], ok, round_=1 << 56), lambda: s.h.pack([0], ok, base_ptr=base.data_ptr() + 4),
           lambda: s.h.pack([0], ok, base_ptr=host.data_ptr()), lambda: s.h.pack([0], ok, residual_ptr=e + 4),
           lambda: s.h.pack([0], ok, residual_ptr=host.data_ptr()), lambda: s.h.pack([0], s.w.data_ptr()),
           lambda: s.h.pack([0], s.m.data_ptr()), lambda: s.h.pack([0], ok, residual_ptr=s.m.data_ptr()),
           lambda: s.h.pack([0], ok, residual_ptr=s.w.data_ptr()), lambda: s.h.pack([0], ok, base_ptr=s.w.data_ptr() + 16),
           lambda: s.h.pack([0], ok, base_ptr=ok), lambda: s.h.pack([0], ok, base_ptr=e, residual_ptr=e),
           lambda: s.h.pack([0], ok, residual_ptr=ok), lambda: s.h.pack([0], ok, base_ptr=s.m.data_ptr()),
           lambda: s.h.unpack([1, 1], ok), lambda: s.h.unpack([], ok), lambda: s.h.unpack([9], ok),
           lambda: s.h.unpack([0], s.w.data_ptr()), lambda: s.h.unpack([0], 0), lambda: s.h.unpack([0], ok, base_ptr=ok),
           lambda: s.h.aggregate_packed([0, 0], ok), lambda: s.h.aggregate_packed([], ok), lambda: s.h.aggregate_packed([4], ok),
           lambda: s.h.aggregate_packed([0], ok, dst_ids=[1, 1]), lambda: s.h.aggregate_packed([0], ok, dst_ids=[4]),
           lambda: s.h.aggregate_packed([0], ok, dst_ids=[]), lambda: s.h.aggregate_packed([0], ok, move_base=True),
           lambda: s.h.aggregate_packed([0], ok + 4), lambda: s.h.aggregate_packed([0], ok, base_ptr=s.w.data_ptr() + 32),
           lambda: s.h.aggregate_packed([0], ok, base_ptr=s.w[2].data_ptr(), move_base=True),
           lambda: s.h.packed_dots([], ok, out.data_ptr()), lambda: s.h.packed_dots([4], ok, out.data_ptr()),
           lambda: s.h.packed_dots([0] * 5, ok, out.data_ptr()), lambda: s.h.packed_dots([0], ok, None),
           lambda: s.h.packed_dots([0], ok, host.data_ptr()), lambda: s.h.packed_dots([0], ok, out.data_ptr() + 2),
           lambda: s.h.packed_dots([0], ok, ok), lambda: s.h.packed_dots([0], ok, s.w.data_ptr()),
           lambda: s.h.packed_dots([0], ok, out.data_ptr(), b_ids=[0]),
           lambda: s.h.packed_dots([0], ok, out.data_ptr(), b_messages_ptr=ok),
           lambda: s.h.packed_dots([0], ok, out.data_ptr(), b_ids=[7], b_messages_ptr=ok),
           lambda: s.h.packed_dots([0], ok, out.data_ptr(), b_ids=[], b_messages_ptr=ok)]
    for i, call in enumerate(bad):
        with pytest.raises(binding.HadflError) as err:
            call()
        assert err.value.code == binding.ERR_INVALID, i
    s.check_guards()
    assert s.h.launch_count() == launches and torch.equal(s.w, before) and torch.all(s.messages == 0xA5)
    s.h.pack([0], ok)                                             # the handle still works
    s.check_guards()


@pytest.mark.parametrize("n,p", [(4, 3001), (32, 70_001)])
def test_captured_and_replayed(n, p):
    """Pack, aggregate and products in a graph: replays do what the calls do, on new parameters each time."""
    rng = np.random.default_rng(30)
    stream = torch.cuda.Stream()
    s, t = Side(n, p, stream=stream), Side(n, p, stream=stream)
    sel = [int(i) for i in rng.permutation(n)[:max(2, n // 2)]]
    outs = [torch.zeros((len(sel), len(sel)), device="cuda") for _ in range(2)]
    bases = [torch.zeros(p, device="cuda") for _ in range(2)]

    def calls(x, base, out):
        x.h.pack(sel, x.messages.data_ptr(), base_ptr=base.data_ptr(), residual_ptr=x.residual.data_ptr(), rounding=1, round_=4)
        x.h.aggregate_packed(sel, x.messages.data_ptr(), base_ptr=base.data_ptr(), dst_ids=range(n), move_base=True)
        x.h.packed_dots(sel, x.messages.data_ptr(), out.data_ptr())
    calls(s, bases[0], outs[0])         # once before the capture
    calls(t, bases[1], outs[1])
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls(s, bases[0], outs[0])
    for r in range(3):
        w = rng.standard_normal((n, p)).astype(np.float32)
        s.rows(w)
        t.rows(w)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        calls(t, bases[1], outs[1])
        torch.cuda.synchronize()
        for x, y in ((s.w, t.w), (s.messages, t.messages), (s.residual, t.residual), (outs[0], outs[1]), (bases[0], bases[1])):
            assert torch.equal(x, y), r
    s.check_guards()


def test_two_handles_on_two_streams_at_once():
    rng = np.random.default_rng(31)
    sides = [Side(8, 200_003, stream=torch.cuda.Stream(), seed=5) for _ in range(2)]
    w = rng.standard_normal((8, 200_003)).astype(np.float32)
    outs = [torch.zeros((8, 8), device="cuda") for _ in range(2)]
    for s in sides:
        s.rows(w)
    torch.cuda.synchronize()
    for _ in range(20):
        for s, out in zip(sides, outs):
            s.h.pack(range(8), s.messages.data_ptr(), residual_ptr=s.residual.data_ptr())
            s.h.packed_dots(range(8), s.messages.data_ptr(), out.data_ptr())
    for s in sides:
        s.check_guards()
    assert torch.equal(sides[0].messages, sides[1].messages) and torch.equal(outs[0], outs[1])
    assert torch.equal(sides[0].residual, sides[1].residual)


def test_calls_wait_for_other_streams_and_copies_before_them():
    """The kernels may start under the one before them in their stream: what else the stream waits for - an event of
    another stream, a copy, a kernel of another kind - has to be done before they read all the same."""
    rng = np.random.default_rng(33)
    p = 3_000_017
    other, stream = torch.cuda.Stream(), torch.cuda.Stream()
    s = Side(2, p, stream=stream)
    sets = [[torch.from_numpy(ref.random_message(rng, p)).cuda() for _ in range(2)] for _ in range(2)]
    want = [[ref.values(*ref.from_bytes(m.cpu().numpy(), p), p).astype(np.float32) for m in two] for two in sets]
    busy = torch.randn(4096, 4096, device="cuda")
    for i in range(2):
        s.messages[i].copy_(sets[0][i])
    s.h.unpack([0, 1], s.messages.data_ptr())
    torch.cuda.synchronize()
    for r in range(12):
        now = sets[r % 2]
        with torch.cuda.stream(stream):
            s.h.unpack([0, 1], s.messages.data_ptr())            # the kernel before, with the messages of the last turn
            if r % 3 == 0:                                       # the new ones from another stream, late
                event = torch.cuda.Event()
                event.record(stream)
                with torch.cuda.stream(other):
                    other.wait_event(event)
                    for _ in range(4):
                        busy = torch.tanh(busy @ busy)
                    for i in range(2):
                        s.messages[i].copy_(now[i])
                    event = torch.cuda.Event()
                    event.record(other)
                stream.wait_event(event)
            elif r % 3 == 1:                                     # by copies in the stream
                for i in range(2):
                    s.messages[i].copy_(now[i], non_blocking=True)
            else:                                                # by kernels that are not the library's
                busy = torch.tanh(busy @ busy)
                for i in range(2):
                    torch.bitwise_or(now[i], now[i], out=s.messages[i])
            s.h.unpack([1, 0], s.messages.data_ptr())
            got = s.w[:, :p].clone()
        stream.synchronize()
        for i in range(2):
            assert np.array_equal(got[i].cpu().numpy(), want[r % 2][i]), (r, i)
    s.check_guards()


def test_residuals_carry_what_messages_leave_out():
    """A constant update sent many times: the sum of the messages stays within one scale of the sum of the updates."""
    rng = np.random.default_rng(32)
    p, rounds = 2048, 50
    s = Side(1, p)
    w = s.rows((1e-2 * rng.standard_normal((1, p))).astype(np.float32))[0].astype(np.float64)
    total = np.zeros(p)
    for r in range(rounds):
        s.h.pack([0], s.messages.data_ptr(), residual_ptr=s.residual.data_ptr())
        total += ref.values(*ref.from_bytes(s.message(0), p), p)
    scales = np.exp2(ref.from_bytes(s.message(0), p)[1].astype(np.float64) - 127)
    assert np.all(np.abs(total - rounds * w) <= np.repeat(scales, 32) + rounds * 1e-8)


def test_long_rows():
    """Rows beyond 2^31 elements apart: a base, a message and products whose offsets need 64 bits."""
    p = (1 << 31) + 4133
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    stride = -(-p // 32) * 32
    w = torch.zeros((2, stride), dtype=torch.bfloat16, device="cuda")
    m = torch.zeros((2, stride), dtype=torch.bfloat16, device="cuda")
    h = binding.Hadfl(2, p, dtype=1, m_dtype=1, w_ptr=w.data_ptr(), m_ptr=m.data_ptr(), row_stride_elems=stride,
                      init_std=0.0, stream=torch.cuda.current_stream().cuda_stream)
    w.zero_()                              # the initial model has zeros of both signs
    size = binding.hadfl_packed_bytes(p)
    at = binding.hadfl_packed_scales_at(p)
    messages = torch.full((2, size), 0xA5, dtype=torch.uint8, device="cuda")
    places = [0, 5, (1 << 30) + 7, (1 << 31) - 1, 1 << 31, (1 << 31) + 4097, p - 1]
    for i, q in enumerate(places):
        w[1, q] = 1.0 + i
    h.pack([1], messages.data_ptr())
    raw = messages[1]
    reads = [1, 2, 3, 4, 4, 6, 8]          # 5 of 6 and 3.5 of 6 are ties
    for q, want in zip(places, reads):
        code = int(raw[q // 2]) >> (4 * (q & 1)) & 15
        assert ref.GRID[code & 7] * 2.0 ** (int(raw[at + q // 32]) - 127) == want
    assert int(raw[:at].ne(0).sum()) == len(places) and int(raw[p // 32 + at + 1:].ne(0).sum()) == 0
    out = torch.zeros((1, 1), device="cuda")
    h.packed_dots([1], messages.data_ptr(), out.data_ptr())
    w[0].fill_(3.0)
    h.unpack([1], messages.data_ptr(), base_ptr=w[0].data_ptr())
    h.synchronize()
    h.debug_check()
    assert [float(w[1, q]) - 3.0 for q in places] == reads
    w[1].zero_()
    h.aggregate_packed([1], messages.data_ptr(), base_ptr=w[0].data_ptr(), dst_ids=[1])
    h.synchronize()
    assert [float(w[1, q]) - 3.0 for q in places] == reads
    assert float(out) == sum(v * v for v in reads)
    assert float(w[1, places[-1] - 1]) == 3.0 and int(w[1, :p].ne(3.0).sum()) == len(places)
    h.destroy()

"""The definition of packed_reference.py on whole rows at once (torch, 64 bits, the fp32 roundings that the definition has
made as such), for vectors too long to go through one element at a time."""
import torch

BLOCK = 32
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MOST = 6 * 2.0**125


def _high_low(a, m):
    """High and low 32 bits of the products of 32-bit words and a constant, in int64: by halves of the constant."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    middle = (low >> 16) + (high & 0xFFFF)
    return (high >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (low & 0xFFFF)


def random_bits(seed, device, round_, p, at="cpu"):
    """16 bits per parameter of a device (Philox4x32-10)."""
    c0 = torch.arange(-(-p // 8), dtype=torch.int64, device=at)
    c1, c2, c3 = (torch.full_like(c0, v) for v in (round_ % 2**32, device, 0x51000000 + round_ // 2**32))
    k0, k1 = seed % 2**32, seed // 2**32
    for _ in range(10):
        (ah, al), (bh, bl) = _high_low(c0, 0xD2511F53), _high_low(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = bh ^ c1 ^ k0, bl, ah ^ c3 ^ k1, al
        k0, k1 = (k0 + 0x9E3779B9) % 2**32, (k1 + 0xBB67AE85) % 2**32
    words = torch.stack((c0, c1, c2, c3), 1)
    return torch.stack((words % 65536, words // 65536), 2).reshape(-1)[:p]


def to_send(w, base=None, residual=None):
    u = w.float()
    if base is not None:
        u = u - base.float()
    return u if residual is None else u + residual


def message(u, bits=None):
    """(codes [whole blocks * 32], scale bytes, the values that they stand for) of fp32 values."""
    p = u.numel()
    x = torch.zeros(-(-p // BLOCK) * BLOCK, dtype=torch.float64, device=u.device)
    x[:p] = u.double()
    blocks = x.view(-1, BLOCK)
    lost = ~(blocks.abs() <= MOST).all(1)
    most = torch.where(lost, torch.zeros_like(blocks[:, 0]), blocks.abs().amax(1))
    mantissa, exponent = torch.frexp(most)                 # most = mantissa * 2^exponent, 1/2 <= mantissa < 1
    s = torch.where(mantissa <= 0.75, exponent - 3, exponent - 2).clamp(min=-127)
    s = torch.where(most == 0, torch.full_like(s, -127), s)
    size = torch.exp2(s.double())[:, None]
    y = torch.where(lost[:, None], torch.zeros_like(blocks), blocks.abs() / size).reshape(-1)
    grid = torch.tensor(GRID, dtype=torch.float64, device=u.device)
    if bits is None:
        middle = (grid[1:] + grid[:-1]) / 2
        code = torch.bucketize(y, middle)                  # how many are below y
        tie = (code < 7) & (y == middle[code.clamp(max=6)])
        code = code + (tie & (code % 2 == 1)).long()
    else:
        t = torch.where(y < 1, (y.float() + 1).double() - 1, y)
        code = torch.bucketize(t, grid, right=True) - 1
        gap = (grid[1:] - grid[:-1])[code.clamp(max=6)]
        r = torch.zeros_like(code)
        r[:p] = bits
        code = code + ((code < 7) & (torch.floor((t - grid[code]) / gap * 65536).long() + r >= 65536)).long()
    negative = torch.signbit(x) & ~lost.repeat_interleave(BLOCK)
    value = torch.copysign(grid[code], x).view(-1, BLOCK) * size
    value = torch.where(lost[:, None], torch.full_like(value, float("nan")), value).reshape(-1)[:p]
    scale = torch.where(lost, torch.full_like(s, 255), s + 127)
    return (code + 8 * negative.long()).to(torch.uint8), scale.to(torch.uint8), value.float()


def to_bytes(codes, scales, scales_at, size):
    out = torch.zeros(size, dtype=torch.uint8, device=codes.device)
    out[:codes.numel() // 2] = codes[0::2] | (codes[1::2] << 4)
    out[scales_at:scales_at + scales.numel()] = scales
    return out


def residual_after(u, values):
    return torch.where(torch.isnan(values), torch.zeros_like(u), u - values)

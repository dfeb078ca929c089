"""Messages of microscaled 4-bit floating point from their definition, in numpy and 64 bits (the fp32 roundings that
the definition has are made as such).  One element or block at a time where that is the clearest."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def sizes(p):
    """(bytes of codes that say something, offset of the scales, number of scales, bytes of the message)."""
    blocks = -(-p // BLOCK)
    at = -(-16 * blocks // 128) * 128
    return 16 * blocks, at, blocks, at + -(-blocks // 128) * 128


def philox(counter, key):
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def random_bits(seed, device, round_, p):
    """16 bits per parameter."""
    out = np.empty(-(-p // 8) * 8, dtype=np.int64)
    for g in range(-(-p // 8)):
        words = philox((g, round_ & 0xFFFFFFFF, device, 0x51000000 | (round_ >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
        for i, w in enumerate(words):
            out[8 * g + 2 * i], out[8 * g + 2 * i + 1] = w & 0xFFFF, w >> 16
    return out[:p]


def to_send(w, base=None, residual=None):
    """The fp32 values u of a row: fl(fl(w - base) + residual)."""
    u = np.asarray(w, dtype=np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        if base is not None:
            u = (u - np.asarray(base, dtype=np.float32)).astype(np.float32)
        if residual is not None:
            u = (u + np.asarray(residual, dtype=np.float32)).astype(np.float32)
    return u


def scale_exponent(most):
    """The smallest s >= -127 with most <= 6 * 2^s, for a finite fp32 value."""
    s = -127                       # at most 125, since larger values make the block read as NaN
    while float(most) > 6.0 * 2.0 ** s:
        s += 1
    return s


def message(u, bits=None):
    """(codes [whole blocks * 32], scale bytes) of fp32 values; `bits`: 16 random bits per value, or None for nearest."""
    p = len(u)
    blocks = -(-p // BLOCK)
    x = np.zeros(blocks * BLOCK)
    with np.errstate(invalid="ignore"):
        x[:p] = u.astype(np.float64)
    codes, scales = np.zeros(blocks * BLOCK, np.uint8), np.zeros(blocks, np.uint8)
    for b in range(blocks):
        v = x[b * BLOCK:(b + 1) * BLOCK]
        if not np.all(np.abs(v) <= 6 * 2.0 ** 125):
            scales[b] = 255
            continue
        s = scale_exponent(np.abs(v).max())
        scales[b] = s + 127
        y = np.abs(v) / 2.0 ** s
        for i in range(BLOCK):
            at = b * BLOCK + i
            if bits is None or at >= p:
                far = np.abs(GRID - y[i])
                near = np.flatnonzero(far == far.min())
                c = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
            else:
                t = y[i]
                if t < 1:  # what fl(t + 1) leaves of t
                    t = float(np.float32(np.float32(t) + np.float32(1))) - 1
                c = int(np.searchsorted(GRID, t, side="right")) - 1
                if c < 7:
                    gap = GRID[c + 1] - GRID[c]
                    c += int(np.floor((t - GRID[c]) / gap * 65536) + bits[at] >= 65536)
            codes[at] = c + (8 if np.signbit(v[i]) else 0)
    return codes, scales


def values(codes, scales, p):
    """What a message reads as: exact, but for what fp32 cannot hold (scales that pack does not write)."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    with np.errstate(over="ignore"):
        return (v.reshape(-1, BLOCK) * s[:, None]).reshape(-1)[:p].astype(np.float32).astype(np.float64)


def to_bytes(codes, scales, p):
    used, at, blocks, size = sizes(p)
    out = np.zeros(size, np.uint8)
    out[:used] = codes[0::2] | (codes[1::2] << 4)
    out[at:at + blocks] = scales
    return out


def from_bytes(raw, p):
    used, at, blocks, _ = sizes(p)
    codes = np.empty(2 * used, np.uint8)
    codes[0::2], codes[1::2] = raw[:used] & 15, raw[:used] >> 4
    return codes, raw[at:at + blocks].copy()


def residual_after(u, codes, scales):
    p = len(u)
    lost = np.repeat(scales == 255, BLOCK)[:p]
    with np.errstate(invalid="ignore"):
        left = (u - values(codes, scales, p).astype(np.float32)).astype(np.float32)
    return np.where(lost, np.float32(0), left)


def random_message(rng, p, low=110, high=130):
    """The bytes of an arbitrary message (any codes, scales 2^(low-127) .. 2^(high-127))."""
    _, _, blocks, _ = sizes(p)
    codes = rng.integers(0, 16, blocks * BLOCK).astype(np.uint8)
    codes[p:] = 0
    return to_bytes(codes, rng.integers(low, high, blocks).astype(np.uint8), p)

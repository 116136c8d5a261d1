"""The float side of the integer format in 64 bits, from its definition in include/niti.h (numpy; no code of the library)."""
import numpy as np


def exponents(top, integer_bits=7):
    """s = max(floor(log2 A) - (integer_bits - 1), -100); 0 for A = 0."""
    top = np.asarray(top, dtype=np.float64)
    e = np.frexp(top)[1] - 1
    return np.where(top > 0, np.maximum(e - (integer_bits - 1), -100), 0)


def round_units(u, mode):
    """Non-negative magnitudes in units of the result to whole numbers (float64)."""
    u = np.asarray(u, dtype=np.float64)
    if mode == 1:
        return np.floor(u + 0.5)
    v = np.floor(u * 65536).astype(np.int64)
    return ((v >> 16) + (((v >> 8) & 255) > (v & 255))).astype(np.float64)


def steady(u, slack, mode):
    """Where a magnitude that is off by less than `slack` units still rounds the same way."""
    u = np.asarray(u, dtype=np.float64)
    if mode == 1:
        return np.abs(u - np.floor(u) - 0.5) > slack
    v = np.floor(u * 65536).astype(np.int64)
    k = np.ceil(slack * 65536) + 1
    top, bot = (v >> 8) & 255, v & 255
    return (bot >= k) & (bot <= 255 - k) & (np.abs(top - bot) > k)


def check_payload(q, s, y, mode, slack):
    """Payload q and exponents s (broadcast) against 64-bit values y whose float32 counterparts are off by `slack` units of
    the result at most: everywhere the nearest whole number (nearest) or one of the two around (pseudo-stochastic), and
    exactly the defined one where `slack` cannot change it."""
    u = np.abs(y) * np.exp2(-s.astype(np.float64))
    want = np.minimum(round_units(u, mode), 127)
    got = np.abs(q.astype(np.float64))
    assert np.all((q == 0) | (np.sign(q) == np.sign(y)))
    sure = steady(u, slack, mode)
    assert np.array_equal(got[sure], want[sure])
    reach = 0.5 if mode == 1 else 1.0
    assert np.all((np.abs(got - u) <= reach + slack) | ((got == 127) & (u > 127 - slack)))
    return sure.mean() if sure.size else 1.0


def decode_e4m3(code, s, block=256):
    """Values of 8-bit state codes (float64)."""
    code = code.astype(np.int64)
    field, frac = (code >> 3) & 15, code & 7
    mag = np.where(field > 0, (8 + frac) * np.exp2(field - 10.0), frac * 2.0 ** -9)
    scale = np.repeat(np.exp2(s.astype(np.float64)), block)[:code.size]
    return np.where(code >= 128, -mag, mag) * scale


def block_exponents(x, block=256):
    """Exponents of the blocks of non-negative values."""
    return exponents(np.concatenate([x, np.zeros(-x.size % block)]).reshape(-1, block).max(1), 8)


def split_e4m3(x, s=None, block=256):
    """Of non-negative values: block exponents (those of the maxima unless given), the codes' whole part, the 16-bit
    fraction behind it (real-valued), and codes' units per value."""
    n = x.size
    s = block_exponents(x, block) if s is None else s
    x = np.concatenate([x, np.zeros(-n % block)]).reshape(-1, block)
    t = x * np.exp2(-s[:, None].astype(np.float64))
    e = np.maximum(np.where(t > 0, np.frexp(t)[1] - 1, -6), -6)
    u = t * np.exp2(3.0 - e)
    whole = np.floor(u)
    return s, ((e + 6) * 8 + whole).reshape(-1)[:n].astype(np.int64), ((u - whole) * 65536).reshape(-1)[:n], \
        np.exp2(3.0 - e - s[:, None]).reshape(-1)[:n]


def random_bits(n, step):
    """The 32 random bits of elements 0 .. n - 1 of a tensor in a step (Python integers' arithmetic mod 2^32)."""
    x = np.arange(n, dtype=np.uint64) ^ np.uint64(step * 0x9E3779B9 % 2 ** 32)
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) % np.uint64(2 ** 32)
    return (x ^ (x >> np.uint64(16))).astype(np.int64)

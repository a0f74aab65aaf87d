"""Codes of a cache in 8 or 4 bits from their definition, in 64 bits: which values they stand for, and which code a value gets."""
import numpy as np

from decode_ref import f64


def values(bits):
    """What the codes that are not negative stand for, in order (NaN aside)."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    return np.array([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127])


def decode(codes, scales, bits):
    """codes uint8 [.., 128 or 64], scales uint8 [.., 4] -> float64 [.., 128]"""
    c = codes.astype(np.int64)
    if bits == 4:
        c = np.stack([c & 15, c >> 4], -1).reshape(c.shape[:-1] + (128,))
    top = 1 << (bits - 1)
    table = values(bits)
    v = np.where(c % top < table.size, table[np.minimum(c % top, table.size - 1)], np.nan)
    v = np.where(c >= top, -v, v)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def encode(rows, bits):
    """bf16 patterns [.., 128] -> (codes uint8 [.., 128 or 64], scales uint8 [.., 4]); of a group that is not finite the codes are 0."""
    x = f64(rows).reshape(rows.shape[:-1] + (4, 32))
    size = np.abs(x).max(-1)
    finite = np.isfinite(size)
    largest = 448.0 if bits == 8 else 6.0
    e = np.full(size.shape, -100)
    for power in range(-99, 120 if bits == 8 else 126):  # beyond that the largest code would be no finite bf16
        e = np.where(finite & (size > largest * 2.0 ** (power - 1)), power, e)
    y = np.where(finite[..., None], x, 0.0) / (2.0 ** e)[..., None]
    sign = np.signbit(np.where(finite[..., None], x, 0.0))
    y = np.minimum(np.abs(y), largest)
    table = values(bits)
    below = np.searchsorted(table, y, side="right") - 1
    above = np.minimum(below + 1, table.size - 1)
    down, up = y - table[below], table[above] - y
    code = np.where((up < down) | ((up == down) & (below % 2 == 1)), above, below)
    code = (code + (sign << (bits - 1))).reshape(rows.shape).astype(np.uint8)
    if bits == 4:
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code, np.where(finite, e + 127, 255).astype(np.uint8)


def bf16_bits(x):
    """Patterns of values that bf16 holds."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    assert not (u & 0xFFFF).any()
    return (u >> 16).astype(np.uint16)


def random_codes(rng, bits, *size):
    """Codes and scales of rows whose values are about as large as a normal distribution's."""
    n = 128 * bits // 8
    codes = rng.integers(0, 256, size + (n,), dtype=np.uint8)
    if bits == 8:  # exponents of 4 bits spread far: half of them near the largest
        codes = np.where((codes & 0x7F) < 0x48, codes | 0x48, codes).astype(np.uint8)
        codes = np.where((codes & 0x7F) == 0x7F, codes & 0xF7, codes).astype(np.uint8)
    scales = rng.integers(-8 if bits == 8 else -3, -6 if bits == 8 else -1, size + (4,)) + 127
    return codes, scales.astype(np.uint8)


def by_head(x):
    """[layers, rows, heads, ..] -> [layers, heads, rows, ..]"""
    return np.ascontiguousarray(np.swapaxes(x, 1, 2))


def pages_by_head(x):
    """[layers, pages, rows, heads, ..] -> [layers, pages, heads, rows, ..]"""
    return np.ascontiguousarray(np.swapaxes(x, 2, 3))

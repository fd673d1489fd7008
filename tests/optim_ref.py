"""AdamW and its 8-bit moments written from the definitions in include/tc.h:
the step in 64 bits, the codes bit by bit in numpy."""
import numpy as np

BLOCK = 256


def adamw64(p, g, m, v, c, lr, b1, b2, eps, wd, t):
    """(p, m, v) after one step, all in binary64"""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = g * c
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = p - lr * wd * p - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p, m, v


def moments32(g, m, v, c, b1, b2):
    """the moments in binary32, each operation rounded: what is then encoded"""
    f = np.float32
    g = (g.astype(f) * f(c)).astype(f)
    m = (m * f(b1)).astype(f) + (g * f(1 - b1)).astype(f)
    v = (v * f(b2)).astype(f) + ((g * g).astype(f) * f(1 - b2)).astype(f)
    return m.astype(f), v.astype(f)


def block_exponents(x):
    top = np.abs(x).reshape(-1, BLOCK).max(1).astype(np.float32)
    return np.minimum(((top.view(np.uint32).astype(np.int64) + 0xFFFFF) >> 23) - 127, 127)


def _bits(x, e, bias):
    """x 2^(-bias - e), rounded once to binary32, as its pattern"""
    y = np.ldexp(np.abs(x).astype(np.float64).reshape(-1, BLOCK), (-bias - e)[:, None])
    return y.astype(np.float32).reshape(-1).view(np.uint32).astype(np.int64)


def noise(pos, seed, swap=False):
    h = ((pos.astype(np.uint64) >> np.uint64(1)) ^ np.uint64(seed)) & np.uint64(0xFFFFFFFF)
    h = (h * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0xB7E15163)) & np.uint64(0xFFFFFFFF)
    h = h ^ (h >> np.uint64(16))
    r = np.where((pos & 1) ^ swap, h >> np.uint64(16), h & np.uint64(0xFFFF)).astype(np.int64)
    return (r << 4) | 8


def encode_m(x, seed):
    e = block_exponents(x)
    u = np.minimum((_bits(x, e, 112) + noise(np.arange(x.size, dtype=np.int64), seed, True)) >> 20, 127)
    return (u | np.where(np.signbit(x), 128, 0)).astype(np.uint8), e.astype(np.int8)


def encode_v(x, seed):
    e = block_exponents(x)
    u = np.minimum((_bits(x, e, 96) + noise(np.arange(x.size, dtype=np.int64), seed)) >> 20, 255)
    return np.where(x > 0, np.maximum(u, 1), u).astype(np.uint8), e.astype(np.int8)


def decode(code, e, bits, bias):
    u = (code & ((1 << bits) - 1)).astype(np.uint32) << np.uint32(20)
    x = np.ldexp(u.view(np.float32).astype(np.float64).reshape(-1, BLOCK), (bias + e.astype(np.int64))[:, None])
    x = x.astype(np.float32).reshape(-1)
    return np.where(code >= 128, -x, x).astype(np.float32) if bits == 7 else x

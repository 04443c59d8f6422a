"""AdamW with moments in 8 bits, in numpy: fp32 arithmetic in the documented order with one rounding per operation, the
codes by their definition, so that codes are compared bit for bit; and the same update in 64 bits."""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & M32
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x6A09E667)) & M32
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0xBB67AE85)) & M32
    return x ^ (x >> np.uint64(16))


def random16(first, n, seed, step, k):
    """The 16 random bits of m and of v, for the values first .. first + n of tensor k."""
    with np.errstate(over="ignore"):
        key = mix(np.uint64(seed) + np.uint64(0x9E3779B1) * np.uint64(k) + np.uint64(0x6A09E667) * mix(step))
        i = np.arange(first, first + n, dtype=np.uint64)
        low, high = i & M32, i >> np.uint64(32)
        x = mix(low * np.uint64(0x9E3779B1) + high * np.uint64(0xBB67AE85) + key)
    return (x & np.uint64(0xFFFF)).astype(np.int64), (x >> np.uint64(16)).astype(np.int64)


def decode(codes, exps, signed):
    c = codes.astype(np.int64)
    e = np.repeat(exps.astype(np.int64), 256)[:len(c)]
    mag = c & 127 if signed else c
    below = 15 if signed else 31
    value = np.where(mag == 0, 0.0, (1 + (mag % 8) / 8) * np.exp2((e - below - 127 + mag // 8).astype(float)))
    value = np.where(signed & (c > 127), -value, value)
    return np.where(e == 255, np.nan, value)


def encode(x, random, signed):
    """x: fp32.  A value between two codes goes up where the fraction of the way and random / 65536 reach 1."""
    below, top = (15, 127) if signed else (31, 255)
    x = np.asarray(x, dtype=np.float64)
    n = len(x)
    a = np.abs(x)
    codes = np.zeros(n, dtype=np.uint8)
    exps = np.zeros((n + 255) // 256, dtype=np.uint8)
    for b in range(len(exps)):
        part = a[b * 256:(b + 1) * 256]
        if not np.isfinite(part).all():
            exps[b] = 255
            continue
        frac, e = np.frexp(part.max())       # frac in [0.5, 1)
        e = int(e) - 1 + (1 if 2 * frac > 1.875 else 0) if frac else -127   # (zeros: the least exponent)
        exps[b] = e = min(max(e + 127, below + 1), 254)
        frac, own = np.frexp(part)
        # place on the scale of all codes: 8 steps an octave
        place = (own - 1 + 127 - (int(e) - below)) * 8.0 + (2 * frac - 1) * 8
        c = np.floor(place + random[b * 256:(b + 1) * 256] / 65536)
        least = 0 if signed else 1
        c = np.where(part == 0, 0, np.clip(c, least, top))
        codes[b * 256:(b + 1) * 256] = c
    if signed:
        codes |= np.where(x < 0, 128, 0).astype(np.uint8)
    return codes, exps


def step32(p, g, m, v, t, scale, lr, b1, b2, eps, wd):
    """One step with every operation rounded to fp32 as the kernels round it (m and v; p to a few units)."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = g.astype(f) * f(scale)
        m = m.astype(f) * f(b1) + g * f(1.0 - b1)
        v = v.astype(f) * f(b2) + (g * g) * f(1.0 - b2)
        p = p.astype(np.float64) * (1 - lr * wd) - lr / (1 - b1 ** t) * m.astype(np.float64) / (
            np.sqrt(v.astype(np.float64)) / np.sqrt(1 - b2 ** t) + eps)
    return p, m, v

"""The group norm with its activation in 64 bits, from its formulas, and how far fp32 arithmetic may be off.

u = 2^-24 is fp32's rounding.  A group has m values, x = xn / rstd + mean.
Statistics: a sum of m values in a tree of partial sums (64 values a lane, lanes, waves) is off by at most 100 u times the
sum of magnitudes (64 + 6 + 16 additions and what follows them), so mean by MEAN = 100 u mean|x|.  The squares are taken about that
mean or about a lane's first value, whose distance is one of the data's: with d the largest |x - mean| of the group,
the variance is off by at most 100 u (var + 4 d^2 k / m) + 2 d MEAN u + MEAN^2, where k is the number of lanes with such a
value (all where each has one: k / m <= 1).  `STAT` below takes 100 u (var + 4 d^2) + MEAN^2 for all.
"""
import numpy as np

U = 2.0 ** -24
STORE = {"fp32": U, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -25}  # (half a step of fp16's subnormal values)


def act(kind, a):
    if kind == "linear":
        return a
    q = 1.0 / (1.0 + np.exp(-a))
    return q if kind == "sigmoid" else a * q


def slope(kind, a):
    if kind == "linear":
        return np.ones_like(a)
    q = 1.0 / (1.0 + np.exp(-a))
    return q * (1 - q) if kind == "sigmoid" else q * (1 + a * (1 - q))


def columns(v, shape):
    return 0.0 * np.zeros(shape) if v is None else v.reshape(1, 1, *shape)


def stats(x, groups, eps):
    """mean, rstd [images, groups] of x [images, positions, width], and how far off they may be."""
    g = x.reshape(x.shape[0], x.shape[1], groups, -1)
    mean = g.mean((1, 3))
    off = g - mean[:, None, :, None]
    var, d = (off ** 2).mean((1, 3)), np.abs(off).max((1, 3))
    emean = 100 * U * np.abs(g).mean((1, 3)) + U * np.abs(mean)
    evar = 100 * U * (var + 4 * d ** 2) + emean ** 2
    rstd = 1.0 / np.sqrt(var + eps)
    # d(rstd) / rstd = -d(var) / 2 (var + eps), a second-order term, and sum, root and quotient
    rel = evar / (var + eps)
    return mean, rstd, emean, rstd * (rel / 2 + rel ** 2 + 8 * U)


def spread(s, width):
    """Statistics of groups as [images, 1, width]."""
    return np.repeat(s, width // s.shape[1], axis=1)[:, None, :]


def forward(x, groups, weight, bias, kind, eps, dtype):
    """y, mean, rstd and the bounds of their errors."""
    width = x.shape[2]
    mean, rstd, emean, erstd = stats(x, groups, eps)
    w = np.ones(width) if weight is None else weight
    b = np.zeros(width) if bias is None else bias
    off, r = x - spread(mean, width), spread(rstd, width)
    a = off * r * w + b
    # (x - mean): its rounding and mean's error; times scale (weight rstd): two roundings; plus bias: one
    ea = (np.abs(off) * U + spread(emean, width)) * r * np.abs(w)
    ea = ea + np.abs(off * w) * spread(erstd, width) + 3 * U * np.abs(off * r * w) + U * np.abs(a)
    y = act(kind, a)
    # slopes are below 1.1; an exponential of -a is off by (|a| + 2) u relative, which reaches q as at most that times q
    ey = ea if kind == "linear" else 1.2 * ea + (4 + np.abs(a)) * 2 * U * np.maximum(np.abs(y), 1e-30)
    ey = ey + STORE[dtype] * (np.abs(y) + ey) + TINY[dtype]
    return y, mean, rstd, ey, emean, erstd


def backward(x, groups, mean, rstd, dy, weight, bias, kind, dtype):
    """dx, dweight, dbias from given statistics, and the bounds of their errors."""
    n, p, width = x.shape
    w = np.ones(width) if weight is None else weight
    b = np.zeros(width) if bias is None else bias
    r = spread(rstd, width)
    xn = (x - spread(mean, width)) * r
    a = xn * w + b
    s = slope(kind, a)
    da = dy * s
    # xn: two roundings; a: two more; the slope's derivative is below 0.6, the slope's own arithmetic 8 roundings of terms below 1 + |a| q
    exn = 2 * U * np.abs(xn)
    ea = exn * np.abs(w) + 2 * U * (np.abs(a) + np.abs(b))
    es = 0.0 if kind == "linear" else 0.6 * ea + (8 + np.abs(a)) * 2 * U * np.minimum(1.0, 2 * (1 + np.abs(a)) * np.exp(-np.abs(a) * 0.999))
    eda = np.abs(dy) * es + U * np.abs(da)

    def grouped(t):
        return t.reshape(n, p, groups, -1).mean((1, 3))

    def back(t):
        return spread(t, width)

    t1, t2 = da * w * xn, da * w
    m1, m2 = back(grouped(t1)), back(grouped(t2))
    # a sum in a tree: 100 u of the magnitudes, as for the mean; over positions, then over columns with the weight
    e1 = back(grouped(eda * np.abs(w * xn) + np.abs(da * w) * exn + 200 * U * np.abs(t1)))
    e2 = back(grouped(eda * np.abs(w) + 200 * U * np.abs(t2)))
    dx = r * (t2 - m2 - xn * m1)
    size = np.abs(t2) + np.abs(m2) + np.abs(xn * m1)
    edx = r * (eda * np.abs(w) + e2 + np.abs(xn) * e1 + np.abs(m1) * exn + 5 * U * size)
    edx = edx + STORE[dtype] * (np.abs(dx) + edx) + TINY[dtype]
    dw, db = (da * xn).sum((0, 1)), da.sum((0, 1))
    # sums over positions and images: up to 200 additions in a row of partial sums' rows
    edw = (eda * np.abs(xn) + np.abs(da) * exn + 400 * U * np.abs(da * xn)).sum((0, 1)) + 1e-37
    edb = (eda + 400 * U * np.abs(da)).sum((0, 1)) + 1e-37
    return dx, dw, db, edx, edw, edb

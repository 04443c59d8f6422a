"""The block norm in 64 bits (numpy), from its formulas, with bounds on what fp32 arithmetic may be off by."""
import numpy as np

U = 2.0 ** -24  # half a unit in the last place of fp32, relative


def act(kind, g):
    if kind == "linear":
        return g, np.ones_like(g)
    with np.errstate(over="ignore"):
        q = 1.0 / (1.0 + np.exp(-g))
    if kind == "sigmoid":
        return q, q * (1.0 - q)
    return g * q, q * (1.0 + g * (1.0 - q))


def forward(x, b, wpre, wpost, gate, kind, post, rs, bs, eps):
    """x, b, gate (or None): float64 [rows, width] (a shared gate: [width]).  Returns y, h, rpre, rpost."""
    rpost = None
    if b is None:
        y = x
    else:
        u = b
        if post:
            rpost = 1.0 / np.sqrt((b * b).mean(1) + eps)
            u = b * rpost[:, None] * (1.0 if wpost is None else wpost)
        if gate is not None:
            u = u * act(kind, gate)[0]
        y = rs * x + bs * u
    rpre = 1.0 / np.sqrt((y * y).mean(1) + eps)
    return y, y * rpre[:, None] * (1.0 if wpre is None else wpre), rpre, rpost


def backward(y, b, rpre, rpost, dh, dy, wpre, wpost, gate, kind, post, rs, bs):
    """Gradients with the statistics given, and for each a bound on the error of fp32 arithmetic (absolute, element
    by element).  Bounds: a sum of n terms that no partial sum takes more than n_serial of is off by at most
    (n_serial + 16) U times the sum of magnitudes; rows are summed by at most width / 256 + 48 terms in a chain, columns by at
    most rows / 32 + 48.  A product of k factors is off by k U; exp(-g) by (|g| + 4) U."""
    rows, width = y.shape
    T = U * (64 + width / 256)
    TR = U * (64 + rows / 32)
    one = np.ones(width)
    wpre = one if wpre is None else wpre
    wpost = one if wpost is None or not post else wpost
    dh = np.zeros_like(y) if dh is None else dh
    dy = np.zeros_like(y) if dy is None else dy
    yn, n = y * rpre[:, None], dh * wpre
    s1 = (n * yn).mean(1, keepdims=True)
    d = dy + rpre[:, None] * (n - yn * s1)
    e_s1 = T * np.abs(n * yn).mean(1, keepdims=True)
    e_d = 8 * U * (np.abs(dy) + rpre[:, None] * (np.abs(n) + np.abs(yn * s1))) + rpre[:, None] * np.abs(yn) * e_s1
    out = {"dpre": ((dh * yn).sum(0), TR * np.abs(dh * yn).sum(0))}
    if b is None:
        out["dx"] = (d, e_d)
        return out
    out["dx"] = (rs * d, abs(rs) * e_d + 2 * U * np.abs(rs * d))
    t, e_t = bs * d, abs(bs) * e_d + 2 * U * np.abs(bs * d)
    r = rpost[:, None] if post else np.ones((rows, 1))
    bn = b * r
    a, slope, e_g = np.ones_like(b), None, 0.0
    if gate is not None:
        a, slope = (np.broadcast_to(v, b.shape) for v in act(kind, gate))
        e_g = 0.0 if kind == "linear" else U * (np.abs(gate) + 12)
        # (the slopes' differences 1 - q and 1 + g (1 - q) are of magnitude up to 1 + |g|)
        e_slope = 0.0 if kind == "linear" else U * (np.abs(gate) + 12) * (1 + np.abs(gate))
        dg = t * bn * wpost * slope
        e_dg = (e_t + 8 * U * np.abs(t)) * np.abs(bn * wpost * slope) + np.abs(t * bn * wpost) * e_slope
        if gate.ndim == 1:
            out["dgate"] = (dg.sum(0), e_dg.sum(0) + TR * np.abs(dg).sum(0))
        else:
            out["dgate"] = (dg, e_dg)
    e_a = np.abs(t * a) * (4 * U + e_g) + e_t * np.abs(a)  # of t * act(gate)
    if kind == "silu" and gate is not None:
        e_a = e_a + np.abs(t) * U * (np.abs(gate) + 12) * np.abs(gate)
    if post:
        out["dpost"] = ((t * a * bn).sum(0), (e_a * np.abs(bn)).sum(0) + TR * np.abs(t * a * bn).sum(0))
    e, e_e = t * a * wpost, e_a * np.abs(wpost) + 2 * U * np.abs(t * a * wpost)
    if post:
        s2 = (e * bn).mean(1, keepdims=True)
        e_s2 = (e_e * np.abs(bn)).mean(1, keepdims=True) + T * np.abs(e * bn).mean(1, keepdims=True)
        out["db"] = (r * (e - bn * s2),
                     r * (e_e + np.abs(bn) * e_s2) + 6 * U * r * (np.abs(e) + np.abs(bn * s2)))
    else:
        out["db"] = (e, e_e)
    return out


def forward_bounds(x, b, y, h, rpre, wpost, gate, kind, post, rs, bs, rpost):
    """Bounds for y, h, rpre, rpost (relative for the statistics); see backward."""
    width = x.shape[1]
    T = U * (64 + width / 256)
    if b is None:
        e_y = np.zeros_like(y)
    else:
        u = b * (rpost[:, None] * (1.0 if wpost is None else wpost) if post else 1.0)
        e_act = 0.0
        if gate is not None:
            a = act(kind, gate)[0]
            e_act = 0.0 if kind == "linear" else U * (np.abs(gate) + 12) * (1 + (np.abs(gate) if kind == "silu" else 0))
            e_act = e_act * np.abs(bs * u)
            u = u * a
        e_y = 3 * U * np.abs(rs * x) + (T + 8 * U) * np.abs(bs * u) + e_act
    rel = T + rpre * np.sqrt((e_y * e_y).mean(1)) * 1.01
    e_h = np.abs(h) * (rel[:, None] + 4 * U) + e_y * np.divide(np.abs(h), np.abs(y), out=np.zeros_like(h), where=y != 0)
    return {"y": e_y, "h": e_h, "rpre": rel * rpre, "rpost": None if rpost is None else T * rpost}


def stored(err, value, dtype):
    """The bound of a value rounded to its type at the store."""
    import torch
    half = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    tiny = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}[dtype]
    return err * 1.01 + half * 1.01 * (np.abs(value) + err) + tiny

"""Gradients against differences of a loss, in directions where a wrong gradient shows."""


def along_gradients(loss, tensors, grads, step=2.0 ** -6, tolerance=1e-3):
    """Moves each tensor along its own gradient, where the derivative is the gradient's norm: a gradient that is a
    hundredth too large or too small, or that has a part of more than a twentieth of its size too much, misses by more than `tolerance`
    of it.  (A gradient g' gives the derivative g g' / |g'|, against |g'|.)  Central differences are off by step^2 / 6
    times a third derivative, (step / size of a row)^2 of the norm."""
    for name, t in tensors.items():
        norm = float(grads[name].double().norm())
        way = (grads[name].double() / norm).to(t.dtype)
        keep = t.clone()
        t.copy_(keep + step * way)
        up = loss()
        t.copy_(keep - step * way)
        down = loss()
        t.copy_(keep)
        slope = (up - down) / (2 * step)
        assert abs(slope - norm) <= tolerance * norm, (name, slope, norm)


def along_rows(loss, t, grad, size, step=2.0 ** -8, tolerance=1e-2):
    """Stretches each row of `t` [rows, width] by itself: what is divided by its root mean square does not change, so neither
    loss nor gradient has anything in that direction.  `size`: of what the means over a row take out of it."""
    for r in range(t.shape[0]):
        assert abs(float((grad[r].double() * t[r].double()).sum())) <= tolerance * size[r], r
        keep = t[r].clone()
        t[r] = keep * (1 + step)
        up = loss()
        t[r] = keep * (1 - step)
        down = loss()
        t[r] = keep
        assert abs((up - down) / (2 * step)) <= tolerance * size[r], r

"""The 64-bit formulas that the GPU kernels are held to, against differences of the forward formula (CPU)."""
import numpy as np
import pytest

from tests import block_norm_ref as ref


@pytest.mark.parametrize("gate", [None, "shared", "full"])
@pytest.mark.parametrize("kind", ["linear", "sigmoid", "silu"])
@pytest.mark.parametrize("post", [True, False])
def test_backward_formulas_match_differences(gate, kind, post):
    rng = np.random.default_rng(11)
    rows, width, eps, rs, bs = 3, 10, 1e-3, 0.9, 0.7
    v = {"x": rng.standard_normal((rows, width)), "b": rng.standard_normal((rows, width)),
         "wpre": 1 + 0.1 * rng.standard_normal(width), "wpost": 1 + 0.1 * rng.standard_normal(width)}
    if gate:
        v["gate"] = rng.standard_normal(width if gate == "shared" else (rows, width))
    dh, dy = rng.standard_normal((2, rows, width))

    def run(v):
        return ref.forward(v["x"], v["b"], v["wpre"], v["wpost"], v.get("gate"), kind, post, rs, bs, eps)

    def loss(v):
        y, h, _, _ = run(v)
        return (y * dy).sum() + (h * dh).sum()

    y, _, rpre, rpost = run(v)
    got = ref.backward(y, v["b"], rpre, rpost, dh, dy, v["wpre"], v["wpost"], v.get("gate"), kind, post, rs, bs)
    names = {"x": "dx", "b": "db", "wpre": "dpre", "gate": "dgate"}
    if post:
        names["wpost"] = "dpost"
    for name, out in names.items():
        if name not in v:
            continue
        step, diff = 1e-5, np.zeros_like(v[name])
        for i in np.ndindex(diff.shape):
            sides = []
            for s in (step, -step):
                w = dict(v, **{name: v[name].copy()})
                w[name][i] += s
                sides.append(loss(w))
            diff[i] = (sides[0] - sides[1]) / (2 * step)
        # central differences: off by step^2 times a third derivative (of order 1..100 here), and by 1e-16 * |loss| / step
        assert np.abs(got[out][0] - diff).max() <= 1e-7 * max(1.0, np.abs(diff).max()), (name, out)


def test_entry_norm_matches_differences():
    rng = np.random.default_rng(12)
    x, dh = rng.standard_normal((2, 4, 7))
    w = 1 + 0.1 * rng.standard_normal(7)
    eps = 1e-3
    y, h, rpre, _ = ref.forward(x, None, w, None, None, "linear", False, 1, 1, eps)
    got = ref.backward(y, None, rpre, None, dh, None, w, None, None, "linear", False, 1, 1)
    diff = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        p, m = x.copy(), x.copy()
        p[i] += 1e-5
        m[i] -= 1e-5
        f = [(ref.forward(q, None, w, None, None, "linear", False, 1, 1, eps)[1] * dh).sum() for q in (p, m)]
        diff[i] = (f[0] - f[1]) / 2e-5
    assert np.abs(got["dx"][0] - diff).max() <= 1e-7 * np.abs(diff).max()

"""The block norm's gradients against differences: the 64-bit formulas on the CPU, and that each mistake planted in them is
found; then the GPU kernels by the same checks, on inputs of the same values."""
import pytest
import torch

from tests import block_norm_ref as ref
from tests.gradient_checks import along_gradients, along_rows

ROWS, WIDTH, EPS, RS, BS = 16, 320, 1e-6, 0.9, 0.7


def inputs(gate, dtype=torch.float64):
    rng = torch.Generator().manual_seed(77)
    scale = torch.exp(0.5 * torch.randn((ROWS, 1), generator=rng))
    t = {k: torch.randn((ROWS, WIDTH), generator=rng) * scale for k in ("x", "b", "gate")}
    t["wpre"], t["wpost"] = (1 + 0.2 * torch.randn(WIDTH, generator=rng) for _ in range(2))
    dh, dy = (0.1 * torch.randn((ROWS, WIDTH), generator=rng) for _ in range(2))
    if gate == "shared":
        t["gate"] = 0.5 + 0.5 * torch.randn(WIDTH, generator=rng)
    elif gate is None:
        del t["gate"]
    return {k: v.to(dtype) for k, v in t.items()}, dh.to(dtype), dy.to(dtype)


NAMES = {"x": "dx", "b": "db", "wpre": "dpre", "wpost": "dpost", "gate": "dgate"}


class Formula:
    """The forward and backward formulas in 64 bits; `mistake` changes the gradients that it returns."""

    def __init__(self, gate, kind, mistake=None):
        self.t, self.dh, self.dy = inputs(gate)
        self.kind, self.mistake = kind, mistake

    def forward(self):
        t = {k: v.numpy() for k, v in self.t.items()}
        return ref.forward(t["x"], t["b"], t["wpre"], t["wpost"], t.get("gate"), self.kind, True, RS, BS, EPS)

    def loss(self, dy=True):
        y, h, _, _ = self.forward()
        return float((y * self.dy.numpy()).sum() * dy + (h * self.dh.numpy()).sum())

    def gradients(self, dy=True):
        t = {k: v.numpy() for k, v in self.t.items()}
        y, _, rpre, rpost = self.forward()
        got = ref.backward(y, t["b"], rpre, rpost, self.dh.numpy(), self.dy.numpy() * dy, t["wpre"], t["wpost"], t.get("gate"),
                           self.kind, True, RS, BS)
        got = {k: torch.from_numpy(got[NAMES[k]][0].copy()) for k in t}
        if self.mistake is not None:
            self.mistake(self, got, y, rpre, rpost)
        return got


def check(f):
    along_gradients(f.loss, f.t, f.gradients())


def check_rows(f):
    """Rows of the branch stretched, which its norm takes back."""
    t = f.t
    g = f.gradients()
    size = [float((g["b"][r].double().norm() * t["b"][r].double().norm())) for r in range(ROWS)]
    along_rows(f.loss, t["b"], g["b"], size)


CASES = [("full", "silu"), ("shared", "sigmoid"), (None, "linear")]


@pytest.mark.parametrize("gate,kind", CASES)
def test_formulas(gate, kind):
    f = Formula(gate, kind)
    check(f)
    check_rows(f)


def scaled(name, by):
    def change(f, got, y, rpre, rpost):
        got[name] *= by
    return change


def without_post_mean(f, got, y, rpre, rpost):
    r = torch.from_numpy(rpost)[:, None]
    bn = f.t["b"] * r
    # db = r (e - bn mean(e bn)): e from the loss's other gradients, t = bs * d
    d = got["x"] / RS
    a = torch.from_numpy(ref.act(f.kind, f.t["gate"].numpy())[0])
    e = BS * d * a * f.t["wpost"]
    got["b"] += r * bn * (e * bn).mean(1, keepdim=True)


def without_last_row(name):
    def change(f, got, y, rpre, rpost):
        keep = f.t, f.dh, f.dy
        cut = {k: v if v.dim() == 1 else v[:-1] for k, v in f.t.items()}
        f.t, f.dh, f.dy = cut, f.dh[:-1], f.dy[:-1]
        mistake, f.mistake = f.mistake, None
        got[name] = f.gradients()[name]
        f.mistake = mistake
        f.t, f.dh, f.dy = keep
    return change


@pytest.mark.parametrize("mistake", [scaled("x", 0.8), scaled("b", 1.01), scaled("wpre", 0.99), scaled("wpost", -1.0),
                                     scaled("gate", 0.5), without_last_row("wpre"), without_last_row("wpost")])
def test_planted_mistakes_are_found_along_the_gradients(mistake):
    with pytest.raises(AssertionError):
        check(Formula("full", "silu", mistake))


def test_a_planted_loss_of_the_branch_mean_is_found_along_its_rows():
    with pytest.raises(AssertionError):
        check_rows(Formula("full", "silu", without_post_mean))


def test_a_planted_loss_of_the_streams_mean_is_found():
    """Where h alone is wanted and there is no branch, stretching a row of x changes nothing."""
    def both(mistake):
        t, dh, _ = inputs(None)

        def loss():
            return float((ref.forward(t["x"].numpy(), None, t["wpre"].numpy(), None, None, "linear", False, 1, 1, EPS)[1]
                          * dh.numpy()).sum())
        y, _, rpre, _ = ref.forward(t["x"].numpy(), None, t["wpre"].numpy(), None, None, "linear", False, 1, 1, EPS)
        g = torch.from_numpy(ref.backward(y, None, rpre, None, dh.numpy(), None, t["wpre"].numpy(), None, None, "linear", False,
                                          1, 1)["dx"][0])
        if mistake:
            yn = t["x"] * torch.from_numpy(rpre)[:, None]
            g = g + torch.from_numpy(rpre)[:, None] * yn * (dh * t["wpre"] * yn).mean(1, keepdim=True)
        along_rows(loss, t["x"], g, [float(g[r].norm() * t["x"][r].norm()) for r in range(ROWS)])
    both(False)
    with pytest.raises(AssertionError):
        both(True)


class Kernels:
    """The GPU's forward and backward pass in fp32 on the same inputs."""

    def __init__(self, gate, kind):
        t, dh, dy = inputs(gate, torch.float32)
        self.t, self.dh, self.dy, self.kind = {k: v.cuda() for k, v in t.items()}, dh.cuda(), dy.cuda(), kind

    def same(self):
        return dict(pre_weight=self.t["wpre"], post_weight=self.t["wpost"], gate=self.t.get("gate"), gate_act=self.kind,
                    residual_scale=RS, branch_scale=BS)

    def loss(self):
        from paper_2104_02621_amd import capscaps as cc
        r = cc.block_norm_fwd(self.t["x"], self.t["b"], eps=EPS, **self.same())
        return float((r.y.double() * self.dy.double()).sum() + (r.h.double() * self.dh.double()).sum())

    def gradients(self):
        from paper_2104_02621_amd import capscaps as cc
        r = cc.block_norm_fwd(self.t["x"], self.t["b"], eps=EPS, save=True, **self.same())
        g = cc.block_norm_bwd(r.y, self.t["b"], r.rstd_pre, r.rstd_post, self.dh, self.dy, **self.same())
        got = {"x": g.dx, "b": g.dbranch, "wpre": g.dpre_weight, "wpost": g.dpost_weight, "gate": g.dgate}
        return {k: got[k] for k in self.t}


@pytest.mark.gpu
@pytest.mark.parametrize("gate,kind", CASES)
def test_kernels(gate, kind):
    """fp32: a loss of 2 * 5120 products of about 0.1, off by about sqrt(10240) * 0.1 * 2^-23 = 1e-6, over 2^-5 and 2^-7: 4e-5 and
    1.5e-4 of slopes, which are above 1."""
    f = Kernels(gate, kind)
    check(f)
    check_rows(f)

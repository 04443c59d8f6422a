"""The gradient of the logits in two terms of 16 bits, where a caller asks for it: dx and dweight are sums in fp32, rounded once.
Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests.head_loss_ref import HALF, TINY, U, gamma
from tests.test_gpu_head_loss import BF16, FP16, FP32, NAMES, Case, close

pytestmark = pytest.mark.gpu


def gradients(c, r, terms):
    """dx and dweight in 64 bits from what the forward pass gave, and how far they may be off with the gradient of z in `terms`."""
    h = c.head()
    lse, logq = r.lse.double()[:, None], (-r.loss[:, None] if c.teacher is None else r.logq).double()
    coef = torch.where(h.row, c.dloss.double() * c.tau, 0.0)[:, None]
    n = torch.arange(c.rows, device="cuda")[:, None].expand(h.pick.shape)
    at = n[h.there], h.pick[h.there]
    q = torch.exp(h.z - lse)
    eq = q * (h.ez + (2 * (h.z - lse).abs() + 8) * U + 2 * U * lse.abs())
    q[at] = torch.exp(logq)[h.there]
    eq[at] = ((2 * logq.abs() + 8) * U * torch.exp(logq))[h.there]
    t, et = torch.zeros_like(q), torch.zeros_like(q)
    t.index_put_(at, h.t[h.there], accumulate=True)
    et.index_put_(at, ((8 + 2 * h.logt.abs()) * 4 * U * h.t)[h.there], accumulate=True)
    g = coef * (q - t)
    eg = coef.abs() * (eq + et) + 4 * U * coef.abs() * (q + t)
    # each term is off by half a step of what the ones before leave over; fp16's smallest step, scaled, at the bottom
    low = 2.0 ** -38 * coef.abs().max() if c.dtype == FP16 else 0.0
    eg = eg + HALF[c.dtype] ** terms * (g.abs() + eg) + torch.where(h.row[:, None], low, 0.0)

    def product(a, ea, b):
        v = a @ b
        e = ea @ b.abs() + gamma(terms * a.shape[1], c.dtype) * (a.abs() @ b.abs())
        return v, e + HALF[c.dtype] * (v.abs() + e) + TINY[c.dtype]

    return product(g, eg, h.w), product(g.T, eg.T, h.x)


# tiles of every size; parts; several pieces of the classes; rows left out
SHAPES = [(300, 72, 513), (600, 64, 20011), (1100, 520, 3001), (2500, 256, 9000), (5000, 64, 150001)]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=NAMES.get)
@pytest.mark.parametrize("top", [None, 5])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_two_terms(shape, top, dtype):
    c = Case(*shape, dtype, top=top, tau=1.0 if top is None else 2.0, bias=True, left=0.1)
    r = c.forward()
    (dx, edx), (dw, edw) = gradients(c, r, 2)
    one, two = c.backward(r), c.backward(r, gradient_terms=2)
    close(two.dx, dx, edx, "dx")
    close(two.dweight, dw, edw, "dweight")
    assert torch.equal(two.dbias, one.dbias)  # (which is taken before the rounding)
    # one term, the rule here, adds an error of its own (which in fp16 is within the worst case of fp32 sums over 20011 classes)
    for got, fine, want in ((one.dx, two.dx, dx), (one.dweight, two.dweight, dw)):
        assert float((fine.double() - want).square().sum()) < float((got.double() - want).square().sum())


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=NAMES.get)
def test_terms_of_the_rule(dtype):
    for shape, terms in (((300, 64, 513), 1), ((256, 64, 513), 2), ((300, 64, 256), 2)):
        c = Case(*shape, dtype, bias=True)
        r = c.forward()
        want, other = c.backward(r, gradient_terms=terms), c.backward(r, gradient_terms=3 - terms)
        for a, b in zip(c.backward(r), want):
            assert torch.equal(a, b)
        assert torch.equal(want.dx, other.dx) == (dtype == FP32)


@pytest.mark.parametrize("shape", [(64, 64, 300), (100, 864, 1001)])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=NAMES.get)
def test_one_term_of_few_rows(shape, dtype):
    c = Case(*shape, dtype, top=3, bias=True, left=0.1)
    r = c.forward()
    g = c.backward(r, gradient_terms=1)
    (dx, edx), (dw, edw) = gradients(c, r, 1)
    close(g.dx, dx, edx, "dx")
    close(g.dweight, dw, edw, "dweight")


def test_other_numbers_of_terms_are_refused():
    c = Case(3, 64, 130, BF16)
    r = c.forward()
    for terms in (-1, 3):
        with pytest.raises(ValueError, match="gradient_terms"):
            c.backward(r, gradient_terms=terms)
        head = cc.HeadArgs(3, 64, 130, cc.BF16, 64, 1, cc.FP32, 1.0, terms)
        assert cc.capscaps_class_loss_workspace_bytes(head, 1) == 0

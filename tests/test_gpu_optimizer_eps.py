"""AdamW with an eps far below the usual, where the quotient's divisor or the second moment are subnormal numbers, on
both sides of the rule that chooses the quotient.  Needs an MI355X."""
import numpy as np
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import adamw_ref as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LR, B1 = 1e-2, 0.9


@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -133, 2.0 ** -100, 2.0 ** -66, 2.0 ** -45, 2.0 ** -40, 2.0 ** -36, 2.0 ** -34,
                                 2.0 ** -27, 2.0 ** 99, 2.0 ** 101, 2.0 ** 127], ids=lambda e: f"2^{int(np.log2(e))}")
@pytest.mark.parametrize("b2", [0.99, 0.999])
@pytest.mark.parametrize("bits", [32, 8])
def test_small_and_large_eps(eps, b2, bits):
    """Gradients from nothing to 1e4, in blocks of their own size (blocks of 8-bit moments share exponents), and some
    of which v is subnormal.  The bound is that of any other eps: m and v are exact, then two products and sums, a root, a
    quotient and the bias corrections, each to a few units in the last place, of the step; one of p."""
    rng = torch.Generator().manual_seed(31)
    sizes = [0.0, 1e-18, 3e-20, 1e-19, 1e-17, 1e-12, 1e-6, 1.0, 1e4]
    g = torch.cat([torch.randn(256, generator=rng) * s for s in sizes])
    n = len(g)
    before = torch.randn(n, generator=rng) * (torch.arange(n) % 3 > 0)     # zeros, to show the smallest steps
    p = before.cuda()
    opt = cc.AdamW([p], lr=LR, betas=(B1, b2), eps=eps, state_bits=bits, seed=1)
    opt.step([g.cuda()])
    want, m, v = ref.step32(before.numpy(), g.numpy(), np.zeros(n, np.float32), np.zeros(n, np.float32), 1, 1.0, LR, B1, b2,
                            eps, 0.0)
    got = p.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    move = np.abs(want - before.numpy())
    over = np.abs(got - want) - (3 * U * np.abs(before.numpy()) + 16 * U * move + 1e-40)
    assert (over <= 0).all(), (int(over.argmax()), got[over.argmax()], want[over.argmax()])
    if bits == 32:
        assert np.array_equal(opt.m[0].cpu().numpy(), m) and np.array_equal(opt.v[0].cpu().numpy(), v)

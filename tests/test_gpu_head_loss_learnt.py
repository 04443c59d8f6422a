"""Rows that a head has learnt: no class is more likely than certain, so no loss is below zero.  Needs an MI355X."""
import pytest
import torch

from tests.head_loss_ref import U
from tests.test_gpu_head_loss import BF16, FP16, FP32, NAMES, Case, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=NAMES.get)
@pytest.mark.parametrize("top", [None, 1, 3])
@pytest.mark.parametrize("shape", [(30, 136, 257), (70, 136, 20011), (600, 136, 20011)], ids=lambda s: "x".join(map(str, s)))
def test_nothing_is_more_likely_than_certain(shape, top, dtype):
    c = Case(*shape, dtype, top=top, bias=True)
    first = c.index if top is None else c.index[:, 0]
    c.x.copy_(c.w[first.clamp(min=0)] * 8 + c.x / 4)  # (the target's logit is some 30 above the others')
    h, r = c.head(), c.forward()
    loss, lse, logq, eloss, else_, elogq = h.forward()
    close(r.lse, lse, else_, "lse")
    close(r.loss, loss, eloss, "loss")
    kept = -r.loss[:, None] if top is None else r.logq
    close(kept, logq, elogq, "logq")
    assert bool((kept <= 0).all()) and float(kept.max()) > -1e-3
    g = c.backward(r)
    dx, dw, db, edx, edw, edb = h.backward(r.lse, kept, c.dloss)
    close(g.dx, dx, edx, "dx")
    close(g.dweight, dw, edw, "dweight")
    # The bias's sums take an entry's q from the products' logits, as any other class's, where the reference takes it from logq: off by
    # the logit's error as well, and by what lse and logq, which are rounded each by itself, differ from it
    arg = h.z - r.lse.double()[:, None]
    eq = torch.exp(arg) * (h.ez + (2 * arg.abs() + 8) * U + 2 * U * r.lse.double().abs()[:, None])
    eq = eq.gather(1, h.pick) + torch.exp(logq) * elogq.expm1()
    eq = torch.where(h.there, eq, 0.0) * (c.dloss.double() * c.tau)[:, None]
    edb = edb.index_add(0, h.pick.flatten(), eq.flatten())
    close(g.dbias, db, edb, "dbias")

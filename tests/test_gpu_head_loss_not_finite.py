"""The bias's gradient of the losses of a head where a row's gradient, or a teacher's logit, is not finite: what the formulas make
of it.  Needs an MI355X."""
import pytest
import torch

from tests.test_gpu_head_loss import BF16, FP16, FP32, NAMES, Case, close

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
TYPES = [FP32, BF16, FP16]
# logits in parts; more classes than are kept in parts, in few rows and in many; few rows of large weights
SHAPES = [(20, 64, 130), (90, 64, 130), (300, 64, 513), (70, 64, 20011), (600, 64, 20011), (20, 800, 15013)]
SHAPE_IDS = ["x".join(map(str, s)) for s in SHAPES]


def formula(h, lse, logq, dloss):
    """g = dloss tau (q - t) in 64 bits, [rows, classes], of rows that count."""
    q = torch.exp(h.z - lse.double()[:, None])
    n = torch.arange(len(q), device="cuda")[:, None].expand(h.pick.shape)
    q[n[h.there], h.pick[h.there]] = torch.exp(logq.double())[h.there]
    t = torch.zeros_like(q).index_put_((n[h.there], h.pick[h.there]), h.t[h.there], accumulate=True)
    return ((dloss.double() * h.tau)[:, None] * (q - t))[h.row]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("top", [None, 3])
@pytest.mark.parametrize("values", [(INF,), (-INF,), (NAN,), (INF, INF), (INF, -INF)], ids=str)
def test_bias_gradient_of_rows_whose_gradient_is_not_finite(values, top, shape, dtype):
    c = Case(*shape, dtype, top=top, bias=True, scale=1.0)
    r = c.forward()
    for k, v in enumerate(values):
        c.dloss[3 + 7 * k] = v
    kept = -r.loss[:, None] if top is None else r.logq
    want = formula(c.head(), r.lse, kept, c.dloss).sum(0)
    assert not bool(torch.isfinite(want).any())
    got = c.backward(r).dbias.double()
    assert torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("value", [INF, NAN])
def test_bias_gradient_of_a_teacher_that_is_not_finite(value, shape, dtype):
    """The shares of such a row are NaN: so are the gradients of its entries' classes, and of no others."""
    c = Case(*shape, dtype, top=4, bias=True)
    c.index[2] = torch.tensor([5, 9, -1, 100], device="cuda")
    r = c.forward()
    h = c.head()
    _, _, db, _, _, edb = h.backward(r.lse, r.logq, c.dloss)
    want = c.backward(r)
    c.teacher[2, 1] = value
    got = c.backward(r)
    hit = torch.zeros(shape[2], dtype=torch.bool, device="cuda")
    hit[[5, 9, 100]] = True
    assert bool(torch.isnan(got.dbias[hit]).all())
    close(got.dbias[~hit], db[~hit], edb[~hit], "dbias")
    others = torch.arange(shape[0], device="cuda") != 2
    assert torch.equal(got.dx[others], want.dx[others]) and bool(torch.isnan(got.dx[2]).all())


@pytest.mark.parametrize("top", [None, 4])
def test_several_pieces_of_the_classes(top):
    c = Case(4096, 64, 70001, FP32, top=top, bias=True, scale=1.0)
    first = torch.arange(0, 70001, 700, device="cuda")  # (classes of every piece)
    if top is None:
        c.index[:len(first)] = first
    else:
        c.index[:len(first), 0] = first
    r = c.forward()
    c.dloss[:len(first)] = INF
    c.dloss[1] = -INF
    want = formula(c.head(), r.lse, -r.loss[:, None] if top is None else r.logq, c.dloss).sum(0)
    got = c.backward(r).dbias.double()
    assert torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
    if top is not None:
        c.teacher[0, 0] = c.teacher[5, 0] = NAN  # (entries that count, of classes 0 and 3500)
        c.dloss.fill_(1.0)
        got = c.backward(r)
        entries = torch.cat([c.index[0], c.index[5]])
        hit = torch.zeros(70001, dtype=torch.bool, device="cuda")
        hit[entries[entries >= 0]] = True
        assert torch.equal(torch.isnan(got.dbias), hit)

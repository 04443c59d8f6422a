"""The losses of a head for up to 64 rows of fp32, which have kernels of their own, element by element: row counts at the ends of
their tiles, widths in parts that no vector divides, classes that no tile divides, rows left out, strides and addresses, gradients
one by one, what is not finite.  Backward they are those of weights of 16 MB and more for each of up to three tiles of 16 rows, forward of
most; the smaller ones here take the products of terms.  Tolerances: tests/head_loss_ref.py.  Needs an MI355X."""
import pytest
import torch

from tests.test_gpu_head_loss import BF16, FP16, FP32, Case

pytestmark = pytest.mark.gpu

ROWS = [2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64]
LARGE = (803, 15013)  # 48.2 MB: both ways for any number of rows
SIZES = pytest.mark.parametrize("width,classes", [(530, 300), LARGE])


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("width,classes", [(803, 1501), (66, 129), (1280, 515), (5, 2000), LARGE, (4100, 3001), (130, 95003),
                                           (801, 20011), (61, 17001)])  # (more classes than the products of terms keep logits of)
def test_class_loss(rows, width, classes):
    Case(rows, width, classes, FP32, bias=rows % 2 == 1, left=0.2).check()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("top,tau", [(1, 1.0), (9, 2.0), (70, 0.5)])
@pytest.mark.parametrize("classes", [1501, LARGE[1]])
def test_distillation(classes, rows, top, tau):
    Case(rows, 803, classes, FP32, top=top, tau=tau, bias=rows % 2 == 0, left=0.2, teacher=BF16 if top == 9 else FP32).check()


@pytest.mark.parametrize("rows", [3, 20, 40, 64])
@pytest.mark.parametrize("gap,shift", [(8, 0), (5, 0), (0, 3), (1, 1), (64, 8)])
def test_strides_and_addresses(gap, shift, rows):
    Case(rows, 530, 300, FP32, gap=gap, shift=shift, left=0.1).check()
    Case(rows, 64, 300, FP32, gap=gap, shift=shift, top=5, bias=True, index=torch.int32, teacher=FP16).check()
    Case(rows, *LARGE, FP32, gap=gap, shift=shift, top=5, bias=True, index=torch.int32, teacher=FP16).check()


@SIZES
@pytest.mark.parametrize("rows", [20, 40, 64])
@pytest.mark.parametrize("top", [None, 4])
def test_rows_left_out(top, rows, width, classes):
    c = Case(rows, width, classes, FP32, top=top, bias=True, left=0.5)
    out = c.index < 0 if top is None else (c.index < 0).all(1)
    want = c.forward()
    grads = c.backward(want)
    c.x[out] = float("nan")
    c.dloss[out] = float("inf")
    r = c.forward()
    for a, b in zip((*r, *c.backward(r)), (*want, *grads)):
        assert torch.equal(a, b)
    assert 0 < int(out.sum()) < rows and (r.loss[out] == 0).all()


@SIZES
@pytest.mark.parametrize("rows", [20, 40, 64])
@pytest.mark.parametrize("top", [None, 4])
def test_no_row_counts(top, rows, width, classes):
    c = Case(rows, width, classes, FP32, top=top, bias=True, left=1.0)
    r = c.forward()
    for t in (*r, *c.backward(r)):
        assert (t == 0).all()


@SIZES
@pytest.mark.parametrize("rows", [20, 40, 64])
def test_nan_stays_in_its_row(rows, width, classes):
    c = Case(rows, width, classes, FP32)
    want = c.forward()
    grads = c.backward(want)
    c.x[17, 3] = float("nan")
    r = c.forward()
    g = c.backward(r)
    others = torch.arange(rows, device="cuda") != 17
    assert torch.isnan(r.loss[17]) and torch.equal(r.loss[others], want.loss[others])
    assert torch.isnan(g.dx[17]).all() and torch.equal(g.dx[others], grads.dx[others])


@SIZES
@pytest.mark.parametrize("rows", [20, 40, 64])
@pytest.mark.parametrize("top", [None, 4])
def test_gradients_one_by_one(top, rows, width, classes):
    c = Case(rows, width, classes, FP32, top=top, bias=True)
    r = c.forward()
    want = c.backward(r)
    a, b, e = c.backward(r, want_dweight=False), c.backward(r, want_dx=False), c.backward(r, want_dx=False, want_dweight=False)
    assert torch.equal(a.dx, want.dx) and a.dweight is None and torch.equal(b.dweight, want.dweight) and b.dx is None
    for t in (a, b, e):
        assert torch.equal(t.dbias, want.dbias)


@SIZES
@pytest.mark.parametrize("rows", [20, 40, 64])
def test_graph_and_repeats(rows, width, classes):
    c = Case(rows, width, classes, FP32, top=5, bias=True, left=0.3)
    first, index = c.x.clone(), c.index.clone()
    r = c.forward()
    g = c.backward(r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cr = c.forward()
        cg = c.backward(cr)
    for k in range(4):
        c.x.copy_(first * (1.0 + 0.25 * k))
        c.index.copy_(index.roll(k, 0))
        graph.replay()
        want = c.forward()
        grads = c.backward(want)
        torch.cuda.synchronize()
        for a, b in zip((*cr, *cg), (*want, *grads)):
            assert torch.equal(a, b), k
    c.x.copy_(first), c.index.copy_(index)
    again = c.forward()
    for a, b in zip((*again, *c.backward(again)), (*r, *g)):
        assert torch.equal(a, b)

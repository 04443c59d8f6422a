"""Gradients of the losses of a head are scaled by the largest dloss that is finite.  Needs an MI355X."""
import pytest
import torch

from tests.test_gpu_head_loss import BF16, FP16, FP32, NAMES, Case, close

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
TYPES = [FP32, BF16, FP16]
# logits in parts; more classes than are kept in parts, in few rows and in many; few rows of large weights
SHAPES = [(20, 64, 130), (90, 64, 130), (300, 64, 513), (70, 64, 20011), (600, 64, 20011), (20, 800, 15013)]
SHAPE_IDS = ["x".join(map(str, s)) for s in SHAPES]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_the_other_rows_gradients_stay_as_they_are(value, shape, dtype):
    """One row's dloss says nothing about how the others' are scaled."""
    c = Case(*shape, dtype, bias=True)
    r = c.forward()
    c.dloss[3] = 0.1  # (the smallest)
    c.dloss /= 8192
    want = c.backward(r)
    c.dloss[3] = value
    got = c.backward(r)
    others = torch.arange(shape[0], device="cuda") != 3
    dx, _, _, edx, _, _ = c.head().backward(r.lse, -r.loss[:, None], c.dloss.nan_to_num(0.0, 0.0, 0.0))
    close(got.dx[others], dx[others], edx[others], "dx")
    assert torch.equal(got.dx[others], want.dx[others])
    assert not bool(torch.isfinite(got.dx[3]).any())

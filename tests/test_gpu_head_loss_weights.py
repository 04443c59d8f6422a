"""The losses of a head with weights whose rows overlap or are one row: the same, bit for bit, as with a dense copy of them.
Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests.test_gpu_head_loss import BF16, FP16, FP32, NAMES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=NAMES.get)
@pytest.mark.parametrize("top", [None, 3])
@pytest.mark.parametrize("rows,classes", [(5, 300), (300, 300), (700, 20011), (5, 70001)])
@pytest.mark.parametrize("stride", [0, 8, 24, 56])
def test_rows_closer_than_their_width(stride, rows, classes, top, dtype):
    c = Case(rows, 64, classes, dtype, top=top, bias=True, left=0.2)
    values = torch.randn((classes - 1) * stride + 64, generator=torch.Generator().manual_seed(stride + 1)) / 4
    c.w = values.to(dtype).cuda().as_strided((classes, 64), (stride, 1))
    r = c.forward()
    g = c.backward(r)
    c.w = c.w.clone(memory_format=torch.contiguous_format)
    assert c.w.stride() == (64, 1)
    want = c.forward()
    for a, b in zip((*r, *g), (*want, *c.backward(want))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=NAMES.get)
@pytest.mark.parametrize("stride", [0, 8, 64])
def test_one_class_at_any_stride(stride, dtype):
    """Through the C ABI: one class has no next one."""
    c = Case(9, 64, 1, dtype)
    want = c.forward()
    loss, lse = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    code = {FP32: cc.FP32, BF16: cc.BF16, FP16: cc.FP16}[dtype]
    head = cc.HeadArgs(9, 64, 1, code, 64, 1, cc.FP32, 1.0)
    need = cc.capscaps_class_loss_workspace_bytes(head, 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    args = cc.HeadFwdArgs(c.x.data_ptr(), c.w.data_ptr(), None, c.index.data_ptr(), None, 64, stride, 1, 0, loss.data_ptr(),
                          lse.data_ptr(), None)
    assert cc.capscaps_class_loss_fwd(head, args, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == cc.OK
    assert torch.equal(loss, want.loss) and torch.equal(lse, want.lse) and bool((lse != 0).any())

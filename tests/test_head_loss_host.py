"""The head losses' checks of arguments (no GPU needed: refused calls do not reach it) and their reference's own pins."""
import ctypes

import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import head_loss_ref as ref

WS = (0x100000, 1 << 40)


def head(**more):
    values = dict(rows=4, width=64, classes=100, dtype=cc.BF16, index_bits=64, top=1, teacher_dtype=cc.FP32, temperature=1.0)
    values.update(more)
    return cc.HeadArgs(**values)


TENSORS = dict(x=0x1000, weight=0x2000, bias=0x3000, index=0x4000, teacher=None, x_stride=64, weight_stride=64, index_stride=1,
               teacher_stride=0)


def fwd(h, distill=False, ws=WS, **more):
    values = dict(TENSORS, loss=0x5000, lse=0x6000, logq=0x7000 if distill else None)
    if distill:
        values.update(teacher=0x8000, teacher_stride=8, index_stride=8)
    values.update(more)
    call = cc.capscaps_distill_loss_fwd if distill else cc.capscaps_class_loss_fwd
    return call(h, cc.HeadFwdArgs(**values), *ws)


def bwd(h, distill=False, ws=WS, **more):
    values = dict(TENSORS, loss=0x5000, lse=0x6000, logq=0x7000 if distill else None, dloss=0x9000, dx=0xa000, dweight=0xb000,
                  dbias=0xc000, dloss_stride=1)
    if distill:
        values.update(teacher=0x8000, teacher_stride=8, index_stride=8)
    values.update(more)
    call = cc.capscaps_distill_loss_bwd if distill else cc.capscaps_class_loss_bwd
    return call(h, cc.HeadBwdArgs(**values), *ws)


@pytest.mark.parametrize("more", [
    dict(rows=-1), dict(rows=(1 << 20) + 1), dict(width=0), dict(width=(1 << 20) + 1), dict(classes=0),
    dict(classes=(1 << 26) + 1), dict(dtype=3), dict(index_bits=16), dict(top=0), dict(top=1025), dict(temperature=0.0),
    dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-7)], ids=str)
def test_heads_that_are_refused(more):
    for distill in (False, True):
        assert fwd(head(**more), distill) == cc.EINVAL
        assert bwd(head(**more), distill) == cc.EINVAL
    for back in (0, 1):
        assert cc.capscaps_class_loss_workspace_bytes(head(**more), back) == 0
        assert cc.capscaps_distill_loss_workspace_bytes(head(**more), back) == 0


BAD_TENSORS = [dict(x=None), dict(weight=None), dict(index=None), dict(x=0x1001), dict(weight=0x2001), dict(bias=0x3002),
               dict(index=0x4004), dict(x_stride=-1), dict(weight_stride=-64), dict(index_stride=-1), dict(x_stride=1 << 41)]


@pytest.mark.parametrize("more", BAD_TENSORS, ids=str)
def test_tensors_that_are_refused(more):
    for distill in (False, True):
        assert fwd(head(), distill, **more) == cc.EINVAL
        assert bwd(head(), distill, **more) == cc.EINVAL


def test_arguments_that_are_refused():
    for more in (dict(loss=None), dict(lse=None), dict(loss=0x5001), dict(lse=0x6002), dict(logq=0x7000), dict(teacher=0x8000)):
        assert fwd(head(), **more) == cc.EINVAL, more
    for more in (dict(logq=None), dict(logq=0x7002), dict(teacher=None), dict(teacher=0x8002), dict(teacher_stride=-1)):
        assert fwd(head(top=8), True, **more) == cc.EINVAL, more
    for more in (dict(loss=None), dict(lse=None), dict(dloss=None), dict(dloss=0x9001), dict(dloss_stride=-1), dict(dx=0xa001),
                 dict(dweight=0xb001), dict(dbias=0xc002), dict(dx=None, dweight=None, dbias=None)):
        assert bwd(head(), **more) == cc.EINVAL, more
    assert bwd(head(top=8), True, logq=None) == cc.EINVAL
    # a class loss has one entry a row and no temperature
    assert fwd(head(top=2)) == cc.EINVAL and fwd(head(temperature=2.0)) == cc.EINVAL
    assert fwd(head(top=8, teacher_dtype=5), True) == cc.EINVAL
    assert cc.capscaps_class_loss_fwd(None, None, *WS) == cc.EINVAL
    assert cc.capscaps_class_loss_fwd(head(), None, *WS) == cc.EINVAL
    assert cc.capscaps_distill_loss_bwd(head(), None, *WS) == cc.EINVAL


@pytest.mark.parametrize("distill", [False, True])
def test_workspaces(distill):
    need = cc.capscaps_distill_loss_workspace_bytes if distill else cc.capscaps_class_loss_workspace_bytes
    for call, back in ((fwd, 0), (bwd, 1)):
        n = need(head(), back)
        assert n > 0
        assert call(head(), distill, (None, n)) == cc.EWORKSPACE
        assert call(head(), distill, (0x100000, n - 1)) == cc.EWORKSPACE
        assert call(head(), distill, (0x100008, n)) == cc.EINVAL


def test_workspaces_hold_a_piece_of_the_logits():
    """... and not all of them."""
    large = head(rows=1 << 16, width=64, classes=1 << 18)
    for back in (0, 1):
        assert cc.capscaps_class_loss_workspace_bytes(large, back) < 4 << 30  # (the logits: 64 GB)


@pytest.mark.parametrize("rows,width,classes", [(1 << 20, 8, 1 << 26), (1 << 20, 1 << 20, 256), (1, 1, 1 << 26), (1, 1 << 20, 1 << 20)])
@pytest.mark.parametrize("dtype", [cc.BF16, cc.FP32])
def test_the_largest_heads_have_workspaces(rows, width, classes, dtype):
    for back in (0, 1):
        need = cc.capscaps_class_loss_workspace_bytes(head(rows=rows, width=width, classes=classes, dtype=dtype), back)
        x = rows * width * (6 if dtype == cc.FP32 else 2)
        assert 0 < need < 3 * x + (1 << 30) * 8 + (8 * classes + 8 * width * rows if back else 0) + 4 * rows * width * back


def test_workspaces_of_heads_that_are_refused():
    """A class loss has one entry and no temperature, a teacher's logits a type."""
    assert cc.capscaps_class_loss_workspace_bytes(head(top=2), 0) == 0
    assert cc.capscaps_class_loss_workspace_bytes(head(temperature=2.0), 1) == 0
    assert cc.capscaps_distill_loss_workspace_bytes(head(top=2, teacher_dtype=9), 0) == 0
    assert cc.capscaps_distill_loss_workspace_bytes(head(top=2, temperature=2.0), 0) > 0


def test_structures_have_the_headers_sizes():
    assert ctypes.sizeof(cc.HeadArgs) == 40
    assert ctypes.sizeof(cc.HeadFwdArgs) == 96
    assert ctypes.sizeof(cc.HeadBwdArgs) == 136


class OnGpu(torch.Tensor):
    """A host tensor that says it is on a GPU."""
    index = 0
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", self.index)

    def get_device(self):
        return self.index


class OnGpu1(OnGpu):
    index = 1


def on(*shape, dtype=torch.float32, kind=OnGpu):
    return torch.zeros(shape, dtype=dtype).as_subclass(kind)


I64 = torch.int64


@pytest.mark.parametrize("call", [
    lambda x, w, t: cc.class_loss_fwd(torch.ones(4, 8), w, t),
    lambda x, w, t: cc.class_loss_fwd(x, on(5, 7), t),
    lambda x, w, t: cc.class_loss_fwd(x, on(0, 8), t),
    lambda x, w, t: cc.class_loss_fwd(x, on(5, 8, dtype=torch.bfloat16), t),
    lambda x, w, t: cc.class_loss_fwd(x.double(), w.double(), t),
    lambda x, w, t: cc.class_loss_fwd(x, on(5, 8, kind=OnGpu1), t),
    lambda x, w, t: cc.class_loss_fwd(x, w, on(4)),
    lambda x, w, t: cc.class_loss_fwd(x, w, on(3, dtype=I64)),
    lambda x, w, t: cc.class_loss_fwd(x, w, on(4, dtype=I64, kind=OnGpu1)),
    lambda x, w, t: cc.class_loss_fwd(x, w, t, bias=on(4)),
    lambda x, w, t: cc.class_loss_fwd(x, w, t, bias=on(5, dtype=torch.float16)),
    lambda x, w, t: cc.class_loss_fwd(x, on(8, 5).T, t),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4, 2)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 0, dtype=I64), on(4, 0)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 1025, dtype=I64), on(4, 1025)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4, 3, dtype=torch.float64)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4, 3, kind=OnGpu1)),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4, 3), temperature=0.0),
    lambda x, w, t: cc.distill_loss_fwd(x, w, on(4, 3, dtype=I64), on(4, 3), temperature=float("nan")),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(3), on(4), on(4)),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(4), on(4), on(3)),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(4), on(4), on(4, dtype=torch.float16)),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(4), on(4), on(4, kind=OnGpu1)),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(4), on(4), on(8)[::2]),
    lambda x, w, t: cc.class_loss_bwd(x, w, t, on(4), on(4), on(4), want_dx=False, want_dweight=False),
    lambda x, w, t: cc.distill_loss_bwd(x, w, on(4, 3, dtype=I64), on(4, 3), on(4), on(4, 2), on(4)),
])
def test_wrapper_refuses(call, monkeypatch):
    made = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: made(*a, **k).as_subclass(OnGpu))
    for name in ("class", "distill"):
        for way in ("fwd", "bwd"):
            monkeypatch.setattr(cc, f"capscaps_{name}_loss_{way}", lambda *a: pytest.fail("not refused"))
    with pytest.raises(ValueError):
        call(on(4, 8), on(5, 8), on(4, dtype=I64))


def test_sizes_that_a_c_int_would_cut(monkeypatch):
    x = on(1, 8).expand((1 << 20) + 1, 8)
    with pytest.raises(ValueError):
        cc.class_loss_fwd(x, on(5, 8), on(1, dtype=I64).expand((1 << 20) + 1))
    with pytest.raises(ValueError):
        cc.class_loss_fwd(on(1, 8), on(1, 8).expand((1 << 26) + 1, 8), on(1, dtype=I64))


@pytest.mark.parametrize("top", [None, 4])
def test_reference_against_torch(top, monkeypatch):
    gen = torch.Generator().manual_seed(0)
    x, w, b = (torch.randn(*s, generator=gen, dtype=torch.float64).requires_grad_() for s in ((6, 5), (9, 5), (9,)))
    d, tau = torch.rand(6, generator=gen, dtype=torch.float64), 1.0 if top is None else 2.0
    z = (x @ w.T + b) / tau
    if top is None:
        index = torch.tensor([3, -1, 8, 0, 0, 5])[:, None]
        teacher = None
        loss = torch.nn.functional.cross_entropy(z, index[:, 0], ignore_index=-1, reduction="none")
    else:
        index = torch.stack([torch.randperm(9, generator=gen)[:4] for _ in range(6)])
        index[1] = -1
        index[2, 1:3] = -1
        teacher = torch.randn(6, 4, generator=gen)
        target = torch.full((6, 9), float("-inf"), dtype=torch.float64)
        for r in range(6):
            for k in range(4):
                if index[r, k] >= 0:
                    target[r, index[r, k]] = teacher[r, k].double() / tau
        target[1] = 0.0
        kl = torch.nn.functional.kl_div(torch.log_softmax(z, 1), torch.softmax(target, 1), reduction="none").sum(1)
        loss = tau ** 2 * kl * (torch.arange(6) != 1)
    grads = torch.autograd.grad(loss, (x, w, b), d)
    xs, ws, bs = x.detach(), w.detach(), b.detach()
    monkeypatch.setitem(ref.HALF, torch.float64, ref.U), monkeypatch.setitem(ref.TINY, torch.float64, 0.0)
    h = ref.Head(xs, ws, bs, index, teacher, tau)
    got = h.forward()
    torch.testing.assert_close(got[0], loss.detach(), rtol=0, atol=1e-12)
    back = h.backward(got[1], got[2], d)
    for a, g in zip(back, grads):
        torch.testing.assert_close(a, g, rtol=0, atol=1e-12)

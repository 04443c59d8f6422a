"""The group norm's checks of arguments (no GPU needed: refused calls do not reach it) and its reference's own pins."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import group_norm_ref as ref


def norm(**more):
    values = dict(images=2, positions=6, width=24, groups=3, x_dtype=cc.BF16, dtype=cc.BF16, act=cc.ACT_SILU, eps=1e-5)
    values.update(more)
    return cc.GroupNormArgs(**values)


def fwd(n, ws=None, nbytes=0, **more):
    values = dict(x=0x1000, weight=0x2000, bias=0x2000, y=0x3000, mean=0x4000, rstd=0x4000, x_stride=24, y_stride=24)
    values.update(more)
    return cc.capscaps_group_norm_fwd(n, cc.GroupFwdArgs(**values), ws, nbytes)


def bwd(n, ws=0x100000, nbytes=1 << 30, **more):
    values = dict(x=0x1000, weight=0x2000, bias=0x2000, mean=0x4000, rstd=0x4000, dy=0x5000, dx=0x6000, dweight=0x7000,
                  dbias=0x7000, x_stride=24, dy_stride=24, dx_stride=24)
    values.update(more)
    return cc.capscaps_group_norm_bwd(n, cc.GroupBwdArgs(**values), ws, nbytes)


BAD_NORMS = [dict(images=0), dict(positions=0), dict(width=0), dict(groups=0), dict(groups=5), dict(groups=25),
             dict(width=(1 << 30) + 24), dict(positions=1 << 31), dict(images=1 << 61), dict(dtype=7), dict(x_dtype=cc.FP16),
             dict(act=3), dict(act=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
             dict(eps=1e-40), dict(dtype=cc.FP32)]


@pytest.mark.parametrize("more", BAD_NORMS, ids=str)
def test_norms_that_are_refused(more):
    assert fwd(norm(**more)) == cc.EINVAL
    assert bwd(norm(**more)) == cc.EINVAL
    assert cc.capscaps_group_norm_fwd_workspace_bytes(norm(**more)) == 0
    assert cc.capscaps_group_norm_bwd_workspace_bytes(norm(**more)) == 0


@pytest.mark.parametrize("more", [dict(x=None), dict(y=None), dict(x=0x1001), dict(y=0x3001), dict(weight=0x2002),
                                  dict(bias=0x2001), dict(mean=0x4002), dict(rstd=0x4001), dict(x_stride=-1),
                                  dict(y_stride=23), dict(y=0x1000, y_stride=32), dict(x_stride=1 << 41)], ids=str)
def test_forward_arguments_that_are_refused(more):
    assert fwd(norm(), **more) == cc.EINVAL


@pytest.mark.parametrize("more", [dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None),
                                  dict(dx=0x1000), dict(dx=0x5000, dx_stride=32), dict(dx_stride=23), dict(dy_stride=-2),
                                  dict(dweight=0x7001), dict(dbias=0x7002), dict(dy=0x5001)], ids=str)
def test_backward_arguments_that_are_refused(more):
    assert bwd(norm(), **more) == cc.EINVAL


def test_null_structures_and_workspaces():
    assert cc.capscaps_group_norm_fwd(None, None, None, 0) == cc.EINVAL
    assert cc.capscaps_group_norm_fwd(norm(), None, None, 0) == cc.EINVAL
    assert cc.capscaps_group_norm_bwd(norm(), None, None, 0) == cc.EINVAL
    large = norm(positions=5000, width=2400)
    need = cc.capscaps_group_norm_fwd_workspace_bytes(large)
    assert need > 0
    strides = dict(x_stride=2400, y_stride=2400)
    assert fwd(large, None, need, **strides) == cc.EWORKSPACE
    assert fwd(large, 0x100000, need - 1, **strides) == cc.EWORKSPACE
    assert fwd(large, 0x100008, need, **strides) == cc.EINVAL
    for n in (large, norm()):
        need = cc.capscaps_group_norm_bwd_workspace_bytes(n)
        strides = dict(x_stride=n.width, dy_stride=n.width, dx_stride=n.width)
        assert need > 0
        assert bwd(n, None, need, **strides) == cc.EWORKSPACE
        assert bwd(n, 0x100000, need - 1, **strides) == cc.EWORKSPACE
        assert bwd(n, 0x100004, need, **strides) == cc.EINVAL


def test_structures_have_the_headers_sizes():
    assert ctypes.sizeof(cc.GroupNormArgs) == 40
    assert ctypes.sizeof(cc.GroupFwdArgs) == 64
    assert ctypes.sizeof(cc.GroupBwdArgs) == 96


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


@pytest.mark.parametrize("call", [
    lambda x: cc.group_norm_fwd(x, 5),
    lambda x: cc.group_norm_fwd(x, 0),
    lambda x: cc.group_norm_fwd(x, 4, act="relu6"),
    lambda x: cc.group_norm_fwd(x, 4, channel_dims=3),
    lambda x: cc.group_norm_fwd(x, 4, channel_dims=0),
    lambda x: cc.group_norm_fwd(x[:0], 4),
    lambda x: cc.group_norm_fwd(x.double(), 4),
    lambda x: cc.group_norm_fwd(x.half(), 4, dtype=torch.bfloat16),
    lambda x: cc.group_norm_fwd(x, 4, weight=on(7)),
    lambda x: cc.group_norm_fwd(x, 4, weight=on(8, dtype=torch.float16)),
    lambda x: cc.group_norm_fwd(x, 4, bias=on(8, kind=OnGpu1)),
    lambda x: cc.group_norm_fwd(x, 4, y=on(2, 3, 8, dtype=torch.bfloat16)),
    lambda x: cc.group_norm_fwd(x, 4, y=on(2, 3, 4)),
    lambda x: cc.group_norm_fwd(x, 4, y=on(2, 3, 8, kind=OnGpu1)),
    lambda x: cc.group_norm_fwd(x.transpose(1, 2), 3),
    lambda x: cc.group_norm_fwd(torch.ones(2, 3, 8), 4),
    lambda x: cc.group_norm_bwd(x, 4, None, on(8), x),
    lambda x: cc.group_norm_bwd(x, 4, on(8), on(7), x),
    lambda x: cc.group_norm_bwd(x, 4, on(8), on(8), on(2, 3, 4)),
    lambda x: cc.group_norm_bwd(x, 4, on(8), on(8), on(2, 3, 8, kind=OnGpu1)),
    lambda x: cc.group_norm_bwd(x.half(), 4, on(8), on(8), on(2, 3, 8, dtype=torch.bfloat16)),
])
def test_wrapper_refuses(call, monkeypatch):
    for name in ("empty", "zeros"):
        made = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, made=made, device=None, **k: made(*a, **k).as_subclass(OnGpu))
    with pytest.raises(ValueError):
        call(on(2, 3, 8))


def test_reference_against_torch():
    rng = np.random.default_rng(0)
    x, dy = rng.standard_normal((2, 5, 12)), rng.standard_normal((2, 5, 12))
    w, b = rng.standard_normal(12), rng.standard_normal(12)
    tx, tw, tb = (torch.tensor(t, requires_grad=True) for t in (x, w, b))
    y = torch.nn.functional.silu(torch.nn.functional.group_norm(tx.transpose(1, 2), 3, tw, tb, 1e-5)).transpose(1, 2)
    grads = torch.autograd.grad(y, (tx, tw, tb), torch.tensor(dy))
    got = ref.forward(x, 3, w, b, "silu", 1e-5, "fp32")
    np.testing.assert_allclose(got[0], y.detach().numpy(), rtol=0, atol=1e-12)
    back = ref.backward(x, 3, got[1], got[2], dy, w, b, "silu", "fp32")
    for a, g in zip(back, grads):
        np.testing.assert_allclose(a, g.numpy(), rtol=0, atol=1e-12)

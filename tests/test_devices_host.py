"""Tensors of several GPUs in one call are refused before the library is called.  No GPU is needed: tensors in host memory
say that they are on one, and no call of the library may be reached."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc


class On(torch.Tensor):
    is_cuda = True
    gpu = 0

    def get_device(self):
        return self.gpu


class OnOther(On):
    gpu = 1


def on(gpu, shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnOther if gpu else On)


@pytest.fixture(autouse=True)
def reached(monkeypatch):
    calls = []
    for name in ("capscaps_block_norm_fwd", "capscaps_block_norm_bwd", "capscaps_grad_norm", "capscaps_adamw_step",
                 "capscaps_adamw_state_values"):
        monkeypatch.setattr(cc, name, lambda *a, name=name, **k: calls.append(name) or cc.OK)
    monkeypatch.setattr(cc, "_stream", lambda device: 0)
    monkeypatch.setattr(cc, "_current_gpu", lambda: None)   # (as a host tensor's index)
    return calls


SHAPE = (4, 8)


@pytest.mark.parametrize("other", [None, "x", "branch", "gate", "y", "h"])
def test_block_norm_forward(reached, other):
    a = {k: on(k == other, SHAPE) for k in ("x", "branch", "gate", "y", "h")}
    if other is None:
        cc.block_norm_fwd(a.pop("x"), a.pop("branch"), **a)
        assert reached == ["capscaps_block_norm_fwd"]
        return
    with pytest.raises(ValueError, match="not on the GPU"):
        cc.block_norm_fwd(a.pop("x"), a.pop("branch"), **a)
    assert not reached


@pytest.mark.parametrize("other", [None, "y", "branch", "gate", "dh", "dy"])
def test_block_norm_backward(reached, other):
    a = {k: on(k == other, SHAPE) for k in ("y", "branch", "gate", "dh", "dy")}
    stats = [torch.ones(4), torch.ones(4)]

    def call():
        return cc.block_norm_bwd(a["y"], a["branch"], *stats, a["dh"], a["dy"], gate=a["gate"])
    if other is None:
        call()
        assert reached == ["capscaps_block_norm_bwd"]
        return
    with pytest.raises(ValueError, match="not on the GPU"):
        call()
    assert not reached


def test_gradient_norm(reached):
    def norm(*gpus, control=0, workspace=0):
        c = on(control, 4)
        return cc.grad_norm([on(g, 9) for g in gpus], control=c, workspace=on(workspace, 65536, torch.uint8))
    norm(0, 0)
    norm(1, 1, control=1, workspace=1)
    assert len(reached) == 2
    for bad in (dict(control=1), dict(workspace=1)):
        with pytest.raises(ValueError, match="GPU"):
            norm(0, 0, **bad)
    with pytest.raises(ValueError, match="GPU"):
        norm(0, 1)
    c = on(0, 4)
    with pytest.raises(ValueError, match="workspace"):    # in host memory
        cc.grad_norm([on(0, 9)], control=c, workspace=torch.zeros(65536, dtype=torch.uint8))
    with pytest.raises(ValueError, match="workspace"):
        cc.grad_norm([on(0, 9)], control=c, workspace=on(0, 2 * 65536, torch.uint8)[::2])
    with pytest.raises(ValueError, match="device tensors"):
        cc.grad_norm([torch.zeros(9)])
    assert len(reached) == 2


def optimizer(bits, **other):
    def of(name, n, dtype):
        return on(name in other, n, dtype)
    kind = torch.float32 if bits == 32 else torch.uint8
    state = [[of(name, 300, kind)] for name in ("m", "v")]
    if bits == 8:
        state += [[of(name, 2, torch.uint8)] for name in ("m_exp", "v_exp")]
    return cc.AdamW([of("param", 300, torch.float32)], state_bits=bits, state=state,
                    copies=[of("copy", 300, torch.bfloat16)])


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(reached, bits):
    opt = optimizer(bits)
    opt.step([on(0, 300)])
    assert len(reached) == 1
    for name in ("param", "m", "v", "copy") + (("m_exp", "v_exp") if bits == 8 else ()):
        with pytest.raises(ValueError, match="one GPU"):
            optimizer(bits, **{name: True})
    with pytest.raises(ValueError, match="GPU"):
        opt.step([on(1, 300)])
    with pytest.raises(ValueError, match="GPU"):
        opt.step([on(0, 300)], control=on(1, 4))
    with pytest.raises(ValueError, match="device tensors"):
        opt.step([torch.zeros(300)])
    opt.m[0] = on(1, 300, torch.float32 if bits == 32 else torch.uint8)
    with pytest.raises(ValueError, match="one GPU"):
        opt.step([on(0, 300)])
    if bits == 8:
        with pytest.raises(ValueError, match="GPU"):
            optimizer(8).state_values(out=[[on(k, 300, torch.bfloat16)] for k in (0, 1)])
    with pytest.raises(ValueError, match="one GPU"):
        cc.AdamW([on(0, 300), on(1, 300)], state=[[on(0, 300), on(1, 300)] for _ in range(2)])
    assert len(reached) == 1

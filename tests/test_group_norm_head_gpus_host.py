"""On which GPU the group norm's and the head losses' calls are made, where torch's current one is another.  No GPU is
needed: torch's own calls are stood in for."""
from contextlib import contextmanager

import pytest
import torch

from paper_2104_02621_amd import capscaps as cc

CALLS = ("group_norm_fwd", "group_norm_bwd", "class_loss_fwd", "class_loss_bwd", "distill_loss_fwd", "distill_loss_bwd")


class On1(torch.Tensor):
    """A host tensor that says it is on the second GPU."""
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", 1)

    def get_device(self):
        return 1


def on1(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(On1)


@pytest.fixture
def calls(monkeypatch):
    """(call, current GPU, stream) of each call; streams are named 100 + their GPU."""
    seen, current = [], [0]

    @contextmanager
    def switched(device):
        before, current[0] = current[0], device.index
        yield
        current[0] = before

    for name in CALLS:
        monkeypatch.setattr(cc, "capscaps_" + name,
                            lambda *a, name=name: seen.append((name, current[0], a[-1])) or cc.OK)
    monkeypatch.setattr(cc, "_stream", lambda device: 100 + device.index)
    monkeypatch.setattr(cc, "_current_gpu", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", switched)
    made = torch.empty  # (there is no second GPU)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: made(*a, **k).as_subclass(On1))
    return seen, current


@pytest.mark.parametrize("now", [0, 1, 3])
def test_calls_are_made_on_the_tensors_gpu(calls, now):
    seen, current = calls
    current[0] = now
    x = on1(2, 6, 8)
    r = cc.group_norm_fwd(x, 4, weight=on1(8), bias=on1(8), save=True)
    cc.group_norm_bwd(x, 4, r.mean, r.rstd, x, weight=on1(8), bias=on1(8))
    rows, weight, targets = on1(5, 8), on1(9, 8), on1(5, dtype=torch.int64)
    r = cc.class_loss_fwd(rows, weight, targets, bias=on1(9))
    cc.class_loss_bwd(rows, weight, targets, r.loss, r.lse, on1(5), bias=on1(9))
    index, logits = on1(5, 3, dtype=torch.int32), on1(5, 3)
    r = cc.distill_loss_fwd(rows, weight, index, logits)
    cc.distill_loss_bwd(rows, weight, index, logits, r.lse, r.logq, on1(1))
    assert [s[0] for s in seen] == list(CALLS)
    assert all(s[1:] == (1, 101) for s in seen), seen
    assert current[0] == now


def test_shapes_and_types_of_what_is_returned(calls):
    x = on1(2, 3, 2, 4, dtype=torch.bfloat16)
    r = cc.group_norm_fwd(x, 2, channel_dims=2, save=True)
    assert r.y.shape == x.shape and r.y.dtype == torch.bfloat16 and r.mean.shape == r.rstd.shape == (2, 2)
    assert cc.group_norm_fwd(x, 2, channel_dims=2).mean is None
    g = cc.group_norm_bwd(x, 2, r.mean, r.rstd, x, weight=on1(2, 4), channel_dims=2)
    assert g.dx.dtype == torch.bfloat16 and g.dweight.shape == (2, 4) and g.dweight.dtype == torch.float32 and g.dbias is None
    rows, weight = on1(2, 5, 8, dtype=torch.float16), on1(9, 8, dtype=torch.float16)
    r = cc.class_loss_fwd(rows, weight, on1(2, 5, dtype=torch.int32))
    assert r.loss.shape == r.lse.shape == (2, 5) and r.loss.dtype == torch.float32
    g = cc.class_loss_bwd(rows, weight, on1(2, 5, dtype=torch.int32), r.loss, r.lse, on1(2, 5), bias=on1(9))
    assert g.dx.shape == rows.shape and g.dx.dtype == g.dweight.dtype == torch.float16 and g.dbias.dtype == torch.float32
    r = cc.distill_loss_fwd(rows, weight, on1(2, 5, 3, dtype=torch.int64), on1(2, 5, 3, dtype=torch.bfloat16))
    assert r.logq.shape == (2, 5, 3) and r.logq.dtype == torch.float32

"""On which GPU the calls of the block norm, the gradient norm and AdamW are made, where torch's current one is another.  No
GPU is needed: torch's own calls are stood in for."""
from contextlib import contextmanager

import pytest
import torch

from paper_2104_02621_amd import capscaps as cc


class On1(torch.Tensor):
    """A host tensor that says it is on the second GPU."""
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", 1)

    def get_device(self):
        return 1


def on1(shape, dtype=torch.float32):
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

    for name in ("block_norm_fwd", "block_norm_bwd", "grad_norm", "adamw_step", "adamw_state_values"):
        monkeypatch.setattr(cc, "capscaps_" + name,
                            lambda *a, name=name: seen.append((name, current[0], a[-1])) or cc.OK)
    monkeypatch.setattr(cc, "_stream", lambda device: 100 + device.index)
    monkeypatch.setattr(cc, "_current_gpu", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", switched)
    for name in ("empty", "zeros"):   # (there is no second GPU)
        made = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, made=made, device=None, **k: made(*a, **k).as_subclass(On1))
    return seen, current


def use():
    x, b, dh = (on1((4, 8)) for _ in range(3))
    stats = [on1(4), on1(4)]
    cc.block_norm_fwd(x, b)
    cc.block_norm_bwd(x, b, *stats, dh, None)
    g = [on1(300), on1(5)]
    cc.grad_norm(g, control=on1(4))
    for bits in (32, 8):
        opt = cc.AdamW([on1(300), on1(5)], state_bits=bits)
        opt.step(g)
        opt.state_values()


@pytest.mark.parametrize("now", [0, 1, 3])
def test_calls_are_made_on_the_tensors_gpu(calls, now):
    seen, current = calls
    current[0] = now
    use()
    assert [s[0] for s in seen] == ["block_norm_fwd", "block_norm_bwd", "grad_norm", "adamw_step", "adamw_step",
                                    "adamw_state_values"]
    assert all(s[1:] == (1, 101) for s in seen), seen
    assert current[0] == now

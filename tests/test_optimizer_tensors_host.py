"""Which memory AdamW hands to the library, without a GPU: tensors that say they are on one, and a library call that
notes its arguments."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc


class OnGpu(torch.Tensor):
    """A host tensor that passes for a device tensor; its memory is never touched."""
    is_cuda = True


def on_gpu(n, dtype=torch.float32):
    return torch.zeros(n, dtype=dtype).as_subclass(OnGpu)


SIZES = [300, 5]


@pytest.fixture
def calls(monkeypatch):
    """What each step gave the library: a list of (param, m, v, m_exp, v_exp, copy, grad, n) for every tensor."""
    seen = []

    def step(items, count, *rest):
        seen.append([(t.param, t.m, t.v, t.m_exp, t.v_exp, t.copy, t.grad, t.n) for t in items])
        return cc.OK

    def values(items, count, m_out, v_out, stream):
        seen.append([(t.m, t.v, t.m_exp, t.v_exp) for t in items])
        return cc.OK

    monkeypatch.setattr(cc, "capscaps_adamw_step", step)
    monkeypatch.setattr(cc, "capscaps_adamw_state_values", values)
    monkeypatch.setattr(cc, "_stream", lambda device: 0)
    monkeypatch.setattr(cc, "_current_gpu", lambda: None)   # (as a host tensor's index)
    return seen


def make(bits, copies=None):
    kind = torch.float32 if bits == 32 else torch.uint8
    state = [[on_gpu(n, kind) for n in SIZES] for _ in range(2)]
    if bits == 8:
        state += [[on_gpu((n + 255) // 256, torch.uint8) for n in SIZES] for _ in range(2)]
    return cc.AdamW([on_gpu(n) for n in SIZES], state_bits=bits, state=state, copies=copies)


def now(opt, grads):
    def ptr(t):
        return None if t is None else t.data_ptr()
    return [(ptr(p), ptr(m), ptr(v), ptr(me), ptr(ve), ptr(c), ptr(g), p.numel()) for p, m, v, me, ve, c, g in
            zip(opt.params, opt.m, opt.v, opt.m_exp, opt.v_exp, opt.copies, grads)]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_goes_to_the_tensors_as_they_are(calls, bits):
    opt = make(bits, [on_gpu(n, torch.bfloat16) for n in SIZES])
    grads = [on_gpu(n) for n in SIZES]
    kind = torch.float32 if bits == 32 else torch.uint8

    def check():
        opt.step(grads)
        assert calls[-1] == now(opt, grads)

    check()
    held = [list(s) for s in (opt.params, opt.m, opt.v, opt.copies)]  # (so that no address is used again)
    opt.params[1].data = on_gpu(5)          # storage replaced
    check()
    opt.params[0] = on_gpu(300)             # tensors replaced
    check()
    opt.m[0] = on_gpu(300, kind)
    check()
    opt.v[1] = on_gpu(5, kind)
    check()
    opt.copies[0], opt.copies[1] = None, on_gpu(5, torch.float16)
    check()
    opt.copies = [on_gpu(300, torch.float16), None]
    check()
    if bits == 8:
        opt.m_exp[0], opt.v_exp[1] = on_gpu(2, torch.uint8), on_gpu(1, torch.uint8)
        check()
        opt.v[0] = on_gpu(300, kind)
        opt.state_values(out=[[on_gpu(n, torch.bfloat16) for n in SIZES] for _ in range(2)])
        assert calls[-1] == [t[1:5] for t in now(opt, grads)]
    del held


@pytest.mark.parametrize("bits", [32, 8])
def test_replaced_tensors_are_checked(calls, bits):
    def refused(change, match):
        opt = make(bits)
        change(opt)
        for _ in range(2):   # and stay refused
            with pytest.raises(ValueError, match=match):
                opt.step([on_gpu(n) for n in SIZES])
        assert not calls

    kind = torch.float32 if bits == 32 else torch.uint8
    refused(lambda opt: opt.m.__setitem__(0, on_gpu(301, kind)), "sizes")
    refused(lambda opt: opt.v.__setitem__(1, on_gpu(5, torch.float16)), "moments")
    refused(lambda opt: opt.params.__setitem__(0, on_gpu(300, torch.float16)), "float32")
    refused(lambda opt: opt.params.__setitem__(0, torch.zeros(300)), "device")
    refused(lambda opt: opt.copies.__setitem__(0, on_gpu(300)), "16-bit")
    refused(lambda opt: opt.m.pop(), "as many")

    def strided(opt):
        opt.params[0] = on_gpu(300).view(15, 20)
        opt.step([on_gpu(n) for n in SIZES])
        calls.clear()
        opt.params[0].data = opt.params[0].data.t()    # same address, values in another order
    refused(strided, "contiguous")


def test_a_capture_does_not_count_the_steps_before_it(calls, monkeypatch):
    """Steps that were counted on the host are added to the optimizer's control once, not by each replay of a graph."""
    opt = make(32)
    opt.step([on_gpu(n) for n in SIZES])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="before the capture"):
        opt.control
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    assert opt.control.view(torch.int32)[3] == 1
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert opt.control.view(torch.int32)[3] == 1

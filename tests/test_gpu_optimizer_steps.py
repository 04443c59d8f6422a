"""How AdamW counts its steps: on the host, in its own control, in a caller's, and by controls for one step alone; saved
and gone on from; captured.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc

pytestmark = pytest.mark.gpu

SIZES = [3000, 41]


def inputs(steps=5, bad=2):
    """Parameters, and gradients of each step; those of step `bad` hold an infinity."""
    rng = torch.Generator().manual_seed(21)
    params = [torch.randn(n, generator=rng).cuda() for n in SIZES]
    grads = [[torch.randn(n, generator=rng).cuda() for n in SIZES] for _ in range(steps)]
    if bad is not None:
        grads[bad][0][7] = float("inf")
    return params, grads


def everything(opt):
    return [t for s in (opt.params, opt.m, opt.v) + ((opt.m_exp, opt.v_exp) if opt.state_bits == 8 else ()) for t in s]


def counted(c):
    return int(c.cpu().view(torch.int32)[3])


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(everything(a), everything(b)))


@pytest.mark.parametrize("bits", [32, 8])
def test_what_grad_norm_returned_counts_as_a_kept_control_does(bits):
    opts = []
    for way in ("kept", "own", "returned"):
        params, grads = inputs()
        opt, kept = cc.AdamW(params, state_bits=bits, seed=3), torch.zeros(4, device="cuda")
        for k, g in enumerate(grads):
            if way == "returned":
                c = cc.grad_norm(g, max_norm=1.0)
                assert counted(c) == (0 if k == 2 else 1)   # of this step alone
            else:
                c = cc.grad_norm(g, max_norm=1.0, control=kept if way == "kept" else opt.control)
            opt.step(g, control=c)
        assert opt.steps == 4
        if way != "kept":
            assert counted(opt.control) == 4
        opts.append(opt)
    assert same(opts[0], opts[1]) and same(opts[0], opts[2])
    # one of them for two optimizers
    a, b = (cc.AdamW(inputs()[0], state_bits=bits, seed=3) for _ in range(2))
    for g in inputs()[1]:
        c = cc.grad_norm(g, max_norm=1.0)
        a.step(g, control=c)
        b.step(g, control=c)
    assert same(a, opts[0]) and same(b, opts[0])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("way", ["own", "returned"])
def test_a_saved_state_goes_on_with_steps_counted_on_the_device(bits, way):
    def run(stop):
        params, grads = inputs()
        opt = cc.AdamW(params, state_bits=bits, seed=4)
        for k, g in enumerate(grads):
            if k == stop:
                state = [[t.clone() for t in s] for s in (opt.m, opt.v, opt.m_exp, opt.v_exp)[:4 if bits == 8 else 2]]
                opt = cc.AdamW(params, state_bits=bits, seed=4, state=state, steps=opt.steps)
            opt.step(g, control=cc.grad_norm(g, max_norm=1.0, control=opt.control if way == "own" else None))
        return opt
    whole = run(None)
    assert whole.steps == 4
    for stop in (1, 3, 4):
        again = run(stop)
        assert again.steps == 4 and same(whole, again)


@pytest.mark.parametrize("bits", [32, 8])
def test_ways_of_counting_follow_each_other(bits):
    params, grads = inputs(bad=None)
    opt = cc.AdamW(params, state_bits=bits, steps=10)
    g = grads[0]
    want = 10
    for way in ("host", "host", "own", "returned", "own", "host", "returned", "host", "host", "own", "host"):
        if way == "host":
            opt.step(g)
        else:
            opt.step(g, control=cc.grad_norm(g, control=opt.control if way == "own" else None))
        want += 1
        if way != "host":
            assert counted(opt.control) == want
    assert opt.steps == want and counted(opt.control) == want
    # a caller's control, then the others
    opt, mine = cc.AdamW(params, state_bits=bits), torch.zeros(4, device="cuda")
    for k in range(3):
        opt.step(g, control=cc.grad_norm(g, control=mine))
    assert opt.steps == 3 and counted(mine) == 3
    opt.step(g)
    assert opt.steps == 4 and counted(opt.control) == 4
    opt = cc.AdamW(params, state_bits=bits)
    mine.zero_()
    for k in range(3):
        opt.step(g, control=cc.grad_norm(g, control=mine))
    opt.step(g, control=cc.grad_norm(g, control=opt.control))
    assert opt.steps == 4
    opt.steps = 7
    assert opt.steps == 7 and counted(opt.control) == 7


def test_a_control_that_does_not_know_the_steps_is_refused():
    params, grads = inputs(bad=None)
    g, fresh = grads[0], torch.zeros(4, device="cuda")
    resumed = cc.AdamW(params, steps=1000)
    begun = cc.AdamW(params)
    begun.step(g)
    on_device = cc.AdamW(params)
    on_device.step(g, control=cc.grad_norm(g))
    held = [t.clone() for t in params]
    for opt in (resumed, begun, on_device):
        with pytest.raises(ValueError, match="counted steps without"):
            opt.step(g, control=cc.grad_norm(g, control=fresh))
    assert all(torch.equal(a, b) for a, b in zip(held, params))


@pytest.mark.parametrize("way", ["own", "returned"])
def test_captured_steps_count(way):
    def program():
        params, grads = inputs(bad=None)
        opt, g = cc.AdamW(params, state_bits=8, steps=5), grads[0]
        return opt, lambda: opt.step(g, control=cc.grad_norm(g, 1.0, control=opt.control if way == "own" else None))
    eager, run = program()
    captured, step = program()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        run()
        graph.replay()
        torch.cuda.synchronize()
        assert eager.steps == captured.steps == 6 + k and same(eager, captured), k

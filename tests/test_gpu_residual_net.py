"""The example that runs norms, convolutions, gradient norm and AdamW together: its gradients against differences of its
own loss, training in every combination of types, served results, and a captured step against an eager one."""
import pytest
import torch

from paper_2104_02621_amd.residual_net import ResidualCapsNet, main, synthetic_batch

pytestmark = pytest.mark.gpu


def small(dtype, **more):
    net = ResidualCapsNet(channels=4, caps=4, blocks=2, size=6, classes=3, dtype=dtype, **more)
    return net, *synthetic_batch(5, 6, 4, 3, dtype)


def test_gradients_against_differences_of_the_loss():
    """In fp32, along a random direction for each parameter, steps of 2^-6: differences of a loss near 1 whose fp32 error is
    about 2^-20 are off by 2^-15; third derivatives add about 2^-12 of the first's size times a few tens."""
    net, images, targets = small(torch.float32, state_bits=32)
    _, grads = net.loss_and_gradients(images, targets)
    loss = lambda: float((net.forward(images).double() - targets.double()).square().mean())  # noqa: E731
    for k, (p, g) in enumerate(zip(net.params, grads)):
        assert g.shape == p.shape and g.dtype == torch.float32, k
        way = g / g.norm()
        keep, step = p.clone(), 2.0 ** -6
        p.copy_(keep + step * way)
        up = loss()
        p.copy_(keep - step * way)
        down = loss()
        p.copy_(keep)
        want = float((g.double() * way.double()).sum())
        assert abs((up - down) / (2 * step) - want) <= 0.02 * abs(want) + 2.0 ** -14, k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("bits", [8, 32])
def test_training_lowers_the_loss(dtype, bits):
    net, images, targets = small(dtype, state_bits=bits, lr=1e-2)
    first = float(net.step(images, targets))
    for _ in range(60):
        last = net.step(images, targets)
    assert float(last) < 0.25 * first
    assert int(net.control.cpu().view(torch.int32)[3]) == 61
    if dtype != torch.float32:   # the layers read the rounded parameters
        for k, low in zip(net.kernels, net.layers):
            assert torch.equal(low, k.to(dtype))
    one, all_of = net.forward(images[:1]), net.forward(images)
    # (one image may take other kernels than five: sums in another order, 16-bit activations)
    assert float((one - all_of[:1]).abs().max()) <= 0.05 * float(all_of.abs().max())


def test_a_captured_step_is_the_eager_one():
    eager, images, targets = small(torch.bfloat16)
    captured, _, _ = small(torch.bfloat16)
    for net in (eager, captured):
        net.step(images, targets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step(images, targets)
    for k in range(4):
        eager.step(images, targets)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.control, captured.control), k
        for a, b in zip(eager.params + eager.opt.m + eager.opt.v, captured.params + captured.opt.m + captured.opt.v):
            assert torch.equal(a, b), k


def test_command(capsys):
    main(["--steps", "11", "--batch", "4", "--blocks", "1", "--graph"])
    said = capsys.readouterr().out
    assert "step 11" in said and "one image served" in said

"""The group norm's statistics where an image's first positions are far from the others (a border, a class token): the squares are taken
about values near the mean, not about these.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests.group_norm_ref import U
from tests.test_gpu_group_norm import BF16, FP32, NAMES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [FP32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("far", [10.0, 1000.0, -30000.0])
@pytest.mark.parametrize("shape", [(2048, 4096, 64, 1), (64, 2048, 1024, 1), (600, 1000, 60, 3), (3, 5000, 270, 10)])
def test_first_positions_far_from_the_others(shape, far, dtype):
    """100 roundings of the variance, whatever its size: a lane's values up to the first new centre, 8 of them, lie around the first one,
    whose distance from the mean is one of those that the variance is made of; the sums past it are of values around a mean."""
    images, positions, width, groups = shape
    gen = torch.Generator(device="cuda").manual_seed(positions)
    x = torch.randn((images, positions, width), generator=gen, device="cuda")
    x[:, 0] += far
    x = x.to(dtype)
    got = cc.group_norm_fwd(x, groups, save=True).rstd.double()
    for n in range(0, images, 64):
        g = x[n:n + 64].double().view(-1, positions, groups, width // groups)
        want = (g - g.mean((1, 3), keepdim=True)).square().mean((1, 3)).add(1e-5).rsqrt()
        off = float((got[n:n + 64] / want - 1).abs().max())
        assert off <= (100 / 2 + 8) * U, (off, n)

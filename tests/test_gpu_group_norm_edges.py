"""The group norm at the edges of its range: more images than a launch has workgroups, groups whose values are far larger than they
differ.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import group_norm_ref as ref
from tests.test_gpu_group_norm import BF16, FP16, FP32, NAMES, Case, close, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images", [1 << 22, (1 << 22) + 3])
def test_more_images_than_one_launch_has_workgroups_for(images):
    """513 values, an odd number, are a workgroup of 1024 threads: 2^32 of them and more, of which a launch takes fewer.  One
    image, broadcast, so that each of the result is the first."""
    row = torch.randn((1, 1, 513), generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    r = cc.group_norm_fwd(row.expand(images, 1, 513), 1, act="silu", save=True)
    want = cc.group_norm_fwd(row, 1, act="silu", save=True)
    for part in r.y.split(1 << 20):
        assert bool((part == want.y).all())
    assert bool((r.mean == want.mean).all()) and bool((r.rstd == want.rstd).all())


@pytest.mark.parametrize("layer", [FP32, BF16, FP16], ids=NAMES.get)
@pytest.mark.parametrize("value", [2e36, -2e36])
@pytest.mark.parametrize("shape", [(2, 5, 24, 3), (1, 3, 27, 1), (2, 7, 64, 4), (1, 1, 32, 1)])
def test_gradients_of_large_equal_values(shape, value, layer):
    """mean * rstd passes fp32's range, x - mean is 0: gradients are those of a group without variance."""
    c = Case(*shape, (FP32, layer))
    c.x.fill_(value)
    r = c.forward()
    assert bool(((r.mean - value).abs() <= 1e-6 * abs(value)).all())
    mean = torch.full_like(r.mean, value)  # (the sum's rounding, 1e29 of 2e36, is no small distance)
    rstd = torch.full_like(r.rstd, 1e-5 ** -0.5)
    g = c.backward(cc.GroupNorm(r.y, mean, rstd))
    dx, dw, db, edx, edw, edb = ref.backward(f64(c.x), c.groups, f64(mean), f64(rstd), f64(c.dy), f64(c.w), f64(c.b), "silu",
                                             NAMES[layer])
    close(g.dx, dx, edx, "dx")
    close(g.dweight, dw, edw, "dweight")
    close(g.dbias, db, edb, "dbias")

"""The group norm at the edges of its range: more images than a launch has workgroups.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests.test_gpu_group_norm import BF16

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

"""The block norm on the GPU where a call is at the edge of what it takes: launches of the most workgroups, outputs
that are not wanted, rows far apart, values that are not finite.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc

pytestmark = pytest.mark.gpu

FP32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16


def test_more_rows_than_one_launch_has_workgroups_for():
    """2^23 + 3 rows of 2048 values in fours, a workgroup of 512 each: 2^32 threads and more, of which a launch takes
    fewer.  One row, broadcast, so that each row of the result is the first."""
    rows = (1 << 23) + 3
    row = torch.randn((1, 2048), generator=torch.Generator().manual_seed(3)).cuda()
    h = cc.block_norm_fwd(row.expand(rows, 2048), dtype=BF16).h
    want = cc.block_norm_fwd(row, dtype=BF16).h
    for part in h.split(1 << 20):
        assert bool((part == want).all())

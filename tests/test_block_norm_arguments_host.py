"""What the Python calls of the block norm make of their arguments, without a GPU."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc


@pytest.mark.parametrize("width", [(1 << 30) + 1, 1 << 32, (1 << 32) + 8])
@pytest.mark.parametrize("dims", [1, 2])
def test_rows_wider_than_the_library_takes_are_refused(width, dims):
    """(The structure's width is a C int: 2^32 + 8 would be 8.)"""
    x = torch.zeros(1).expand((1, width) if dims == 1 else (1, 2, (width + 1) // 2))
    with pytest.raises(ValueError, match="up to 2\\^30"):
        cc.block_norm_fwd(x, norm_dims=dims)
    with pytest.raises(ValueError, match="up to 2\\^30"):
        cc.block_norm_bwd(x, None, None, None, x, None, norm_dims=dims)

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


def launch(block, branch, forward, apart):
    import ctypes
    out = (ctypes.c_longlong * 2)()
    fn = cc._load().capscaps_testing_block_norm_launch
    fn.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 3 + [ctypes.c_void_p]
    assert fn(ctypes.addressof(block), branch, forward, apart, ctypes.addressof(out)) == 1
    return tuple(out)


@pytest.mark.parametrize("types", [(cc.FP32, cc.FP32, cc.FP32), (cc.BF16, cc.BF16, cc.BF16), (cc.BF16, cc.FP32, cc.BF16),
                                   (cc.FP16, cc.FP16, cc.FP32), (cc.FP16, cc.FP32, cc.FP32)])
def test_no_launch_passes_the_limit_of_threads(types):
    """Workgroups times threads stay below 2^32 for every width in registers, however many rows there are."""
    for width in range(1, 16385):
        for rows in (1, 1 << 23, 1 << 33, (1 << 40) + 1):
            b = cc.BlockArgs(rows, width, *types, 1, cc.GATE_NONE, cc.ACT_LINEAR, 1.0, 1.0, 1e-6)
            for way in ((1, 1, 0), (1, 0, 0), (0, 1, 0), (0, 0, 0), (1, 1, 1), (1, 0, 1)):
                blocks, threads = launch(b, *way)
                assert 1 <= blocks and 64 <= threads <= 1024 and blocks * threads < 1 << 32, (rows, width, way)
                assert blocks <= rows

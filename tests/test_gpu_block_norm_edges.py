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


def rows_of(rows, width, dtype, seed):
    return torch.randn((rows, width), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


# (layers, stream, branch): vectors of eight and of four, one and several a lane, remainders, rows of no group
KERNELS = [(27, (FP32, FP32, FP32)), (64, (BF16, BF16, BF16)), (600, (FP16, FP16, FP32)), (1027, (BF16, FP32, BF16)),
           (5000, (FP32, FP32, FP32)), (9000, (BF16, BF16, BF16)), (9001, (FP16, FP16, FP32)), (12000, (FP16, FP32, FP16)),
           (20001, (BF16, FP32, FP32))]


@pytest.mark.parametrize("gate", [None, "shared", "full"])
@pytest.mark.parametrize("width,types", KERNELS, ids=lambda v: v if isinstance(v, int) else None)
def test_without_a_norm_the_branch_gradient_does_not_depend_on_the_branch(width, types, gate):
    layer, stream, branch = types
    rows = 37
    y, dh, dy = (rows_of(rows, width, t, k) for k, t in enumerate((stream, layer, stream)))
    rpre = torch.rsqrt(y.double().square().mean(1) + 1e-6).float()
    b = rows_of(rows, width, branch, 7)
    g = None if gate is None else rows_of(rows, width, layer, 8) if gate == "full" else torch.randn(width, device="cuda")
    same = dict(post_norm=False, gate=g, gate_act="sigmoid" if gate else "linear", branch_scale=0.5, dtype=layer)
    bad = b.clone()
    bad[3, width // 2], bad[4, width - 1], bad[5, 0] = float("inf"), float("nan"), float("-inf")
    for grads in ((None, dy), (dh, dy), (dh, None)):
        want = cc.block_norm_bwd(y, b, rpre, None, *grads, **same)
        got = cc.block_norm_bwd(y, bad, rpre, None, *grads, **same)
        assert torch.isfinite(got.dbranch).all()
        assert torch.equal(got.dbranch, want.dbranch) and torch.equal(got.dx, want.dx)


@pytest.mark.parametrize("layer", [BF16, FP16])
@pytest.mark.parametrize("shape,dims", [((1, 200), 1), ((200,), 1), ((1, 1, 1, 8, 1, 5, 5), 4), ((8, 1, 5, 5), 4)])
def test_one_row_takes_the_gates_that_many_rows_take(shape, dims, layer):
    """A learned scale of shape [1, ..., width] for all rows, and a gate for every value: for one row of a tensor what they
    are for many.  (In float32 layers both have one type and mean the same for one row.)"""
    many = (3,) + shape if shape[0] != 1 else (3,) + shape[1:]
    x, b, per_value, dy = (rows_of(3, 200, t, k).reshape(many) for k, t in enumerate((FP32, layer, layer, FP32)))
    vector = torch.randn(200, generator=torch.Generator().manual_seed(9)).cuda()
    weight = torch.rand(200, device="cuda")

    def one(t):
        return t[1].reshape(shape)

    for gate_of_all, gate in ((vector.view((1,) + many[1:]), vector.view(shape)), (per_value, one(per_value))):
        same = dict(post_weight=weight, gate_act="silu", norm_dims=dims, dtype=layer)
        want = cc.block_norm_fwd(x, b, gate=gate_of_all, save=True, **same)
        got = cc.block_norm_fwd(one(x), one(b), gate=gate, save=True, **same)
        assert torch.equal(got.y, one(want.y)) and torch.equal(got.h, one(want.h))
        back = cc.block_norm_bwd(got.y, one(b), None, got.rstd_post.reshape(1), None, one(dy), gate=gate, **same)
        assert back.dgate.shape == gate.shape and back.dgate.dtype == gate.dtype
        few = cc.block_norm_bwd(want.y, b, None, want.rstd_post.reshape(3), None, dy, gate=gate_of_all, **same)
        assert torch.equal(back.dbranch, one(few.dbranch))
        if gate_of_all is per_value:
            assert torch.equal(back.dgate, one(few.dgate))
    other = FP16 if layer == BF16 else BF16
    for bad in (per_value.to(other), vector.view((1,) + many[1:]).expand(many)):
        with pytest.raises(ValueError, match="gate"):
            cc.block_norm_fwd(x, b, gate=bad, norm_dims=dims, dtype=layer)
    with pytest.raises(ValueError):
        cc.block_norm_fwd(one(x), one(b), gate=one(per_value).to(other), norm_dims=dims, dtype=layer)

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



@pytest.mark.parametrize("gate", [None, "shared", "full"])
@pytest.mark.parametrize("width,types", KERNELS, ids=lambda v: v if isinstance(v, int) else None)
def test_each_backward_output_may_be_left_out(width, types, gate):
    """Through the C ABI: every output by itself, and all but one, is what it is among all; the memory of one that
    is not wanted stays as it was."""
    layer, stream, branch = types
    rows = 37
    y, b, dh, dy = (rows_of(rows, width, t, k) for k, t in enumerate((stream, branch, layer, stream)))
    rpre, rpost = (torch.rsqrt(t.double().square().mean(1) + 1e-6).float() for t in (y, b))
    wpre, wpost = (torch.rand(width, device="cuda") + 0.5 for _ in range(2))
    g = None if gate is None else rows_of(rows, width, layer, 8) if gate == "full" else torch.rand(width, device="cuda")
    code = {FP32: cc.FP32, BF16: cc.BF16, FP16: cc.FP16}
    block = cc.BlockArgs(rows, width, code[layer], code[stream], code[branch], 1,
                         {None: cc.GATE_NONE, "shared": cc.GATE_SHARED, "full": cc.GATE_FULL}[gate], cc.ACT_SILU, 0.9, 0.5, 1e-6)
    need = cc.capscaps_block_norm_bwd_workspace_bytes(block)
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    types_of = {"dx": stream, "dbranch": layer, "dpre_weight": FP32, "dpost_weight": FP32}
    if gate:
        types_of["dgate"] = layer if gate == "full" else FP32

    def run(wanted):
        out = {k: torch.full((width,) if k.endswith("weight") or k == "dgate" and gate == "shared" else (rows, width), 7.0,
                             dtype=t, device="cuda") for k, t in types_of.items()}
        sums = any(k.endswith("weight") or k == "dgate" and gate == "shared" for k in wanted)
        args = cc.BlockBwdArgs(y=y.data_ptr(), branch=b.data_ptr(), gate=None if g is None else g.data_ptr(),
                               pre_weight=wpre.data_ptr(), post_weight=wpost.data_ptr(), rstd_pre=rpre.data_ptr(),
                               rstd_post=rpost.data_ptr(), dh=dh.data_ptr(), dy=dy.data_ptr(),
                               **{k: out[k].data_ptr() for k in wanted},
                               **{k + "_stride": width for k in ("y", "branch", "gate", "dh", "dy", "dx", "dbranch", "dgate")})
        stream_ = torch.cuda.current_stream().cuda_stream
        rc = cc.capscaps_block_norm_bwd(block, args, workspace.data_ptr() if sums else None, need if sums else 0, stream_)
        assert rc == cc.OK, (wanted, rc)
        return out

    names = list(types_of)
    every = run(names)
    for wanted in [[k] for k in names] + [[j for j in names if j != k] for k in names]:
        got = run(wanted)
        for k in names:
            if k in wanted:
                assert torch.equal(got[k], every[k]), (wanted, k)
            else:
                assert (got[k] == 7.0).all(), (wanted, k)


@pytest.mark.parametrize("gate", ["shared", "full"])
@pytest.mark.parametrize("width,types", KERNELS[1:] + [(27, (BF16, BF16, BF16)), (512, (FP16, FP16, FP16)), (40000, (FP16, FP16, FP16))],
                         ids=lambda v: v if isinstance(v, int) else None)
def test_zeros_infinities_and_nan_stay_in_their_rows(width, types, gate):
    """In every kind of kernel: what is not finite in a row makes NaN or zeros of that row alone, next to it in a workgroup
    and in memory included; sums over rows are NaN where it reaches."""
    layer, stream, branch = types
    rows, inf, nan = 16, float("inf"), float("nan")
    x, b, dh, dy, full = (rows_of(rows, width, t, k) for k, t in enumerate((stream, branch, layer, stream, layer)))
    g = full if gate == "full" else torch.rand(width, device="cuda") + 0.5
    same = dict(gate=g, gate_act="sigmoid", pre_weight=torch.rand(width, device="cuda") + 0.5,
                post_weight=torch.rand(width, device="cuda") + 0.5, dtype=layer)

    def stats(y, b):
        return [torch.rsqrt(t.double().square().mean(1) + 1e-6).float() for t in (y, b)]

    clean = cc.block_norm_fwd(x, b, save=True, **same)
    back = cc.block_norm_bwd(x, b, *stats(x, b), dh, dy, **same)
    good = [0, 2, 5, 7, 8, 10, 12, 14, 15]
    xs, bs = x.clone(), b.clone()
    xs[1], bs[1] = 0.0, 0.0
    xs[3, width // 2], xs[4, 0], xs[6, width - 1] = inf, nan, -inf
    bs[9, width - 1], bs[11, 0], bs[13, width // 2] = nan, inf, -inf
    r = cc.block_norm_fwd(xs, bs, save=True, **same)
    assert (r.y[1] == 0).all() and (r.h[1] == 0).all()
    for k in (3, 4, 6):       # an infinity in the stream: its root mean square is infinite, so the row is zeros but for it
        at = {3: width // 2, 4: 0, 6: width - 1}[k]
        rest = [j for j in range(width) if j != at]
        assert not torch.isfinite(r.y[k, at]) and torch.isnan(r.h[k, at])
        assert torch.equal(r.y[k, rest], clean.y[k, rest])
        assert torch.isnan(r.h[k]).all() if k == 4 else (r.h[k, rest] == 0).all()
    for k, at in ((9, width - 1), (11, 0), (13, width // 2)):   # in the branch: the norm after it spreads it
        assert torch.isnan(r.y[k, at]) and torch.isnan(r.h[k]).all()
        if k == 9:
            assert torch.isnan(r.y[k]).all()
        else:
            rest = [j for j in range(width) if j != at]
            assert torch.equal(r.y[k, rest], x[k, rest])
    for k in good:
        assert torch.equal(r.y[k], clean.y[k]) and torch.equal(r.h[k], clean.h[k])
    dhs, dys = dh.clone(), dy.clone()
    dhs[3, width // 2], dhs[4, 0], dys[6, width - 1], dys[9, 0] = inf, nan, nan, -inf
    got = cc.block_norm_bwd(x, b, *stats(x, b), dhs, dys, **same)
    for k in (3, 4):
        assert not torch.isfinite(got.dx[k]).any() and torch.isnan(got.dbranch[k]).all()
    for k, at in ((6, width - 1), (9, 0)):
        rest = [j for j in range(width) if j != at]
        assert not torch.isfinite(got.dx[k, at]) and torch.equal(got.dx[k, rest], back.dx[k, rest])
        assert not torch.isfinite(got.dbranch[k]).any()   # (e infinite in one place: the mean is, and -inf + inf there)
    for k in good + [1, 11, 13]:
        if k != 9:
            assert torch.equal(got.dx[k], back.dx[k]) and torch.equal(got.dbranch[k], back.dbranch[k])
            if gate == "full":
                assert torch.equal(got.dgate[k], back.dgate[k])
    assert not torch.isfinite(got.dpre_weight[[0, width // 2]]).any()

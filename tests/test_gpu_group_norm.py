"""GPU parity of the group norm with its activation (forward and backward) against its formulas in 64 bits: every element
type and activation, groups of one value to groups wider than a workgroup's columns, one position to many, rows at
odd strides and addresses, in place, values far from zero, infinities and NaN, other streams, graphs.  Tolerances:
tests/group_norm_ref.py, from the number of roundings."""
import numpy as np
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import group_norm_ref as ref

pytestmark = pytest.mark.gpu

FP32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(FP32, FP32), (FP32, BF16), (BF16, BF16), (FP32, FP16), (FP16, FP16)]
NAMES = {FP32: "fp32", BF16: "bf16", FP16: "fp16"}
IDS = [f"{NAMES[x]}-{NAMES[d]}" for x, d in TYPES]
ACTS = ["linear", "sigmoid", "silu"]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def close(got, want, err, what):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - err
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}{at}: {got[at]} for {want[at]}, bound {err[at]}"


class Case:
    def __init__(self, images, positions, width, groups, types, kind="silu", affine=True, gap=0, shift=0, offset=0.0,
                 seed=0):
        self.groups, self.kind, self.eps, self.gap, self.shift = groups, kind, 1e-5, gap, shift
        self.xt, self.layer = types
        rng = torch.Generator().manual_seed(seed + 7 * images + 11 * positions + width)
        scale = torch.exp(0.5 * torch.randn((images, 1, width), generator=rng))
        shape = (images, positions, width)
        self.x = self.place((torch.randn(shape, generator=rng) * scale + offset).to(self.xt))
        self.dy = self.place(torch.randn(shape, generator=rng).to(self.layer))
        self.w = self.b = None
        if affine:
            self.w, self.b = (1 + 0.3 * torch.randn(width, generator=rng)).cuda(), torch.randn(width, generator=rng).cuda()

    def place(self, t):
        """On the GPU, rows `gap` values apart, the first `shift` values into its allocation."""
        if not self.gap and not self.shift:
            return t.cuda()
        n, p, w = t.shape
        wide = torch.full((n * p * (w + self.gap) + self.shift,), float("nan"), dtype=t.dtype, device="cuda")
        view = wide[self.shift:].view(n, p, w + self.gap)[:, :, :w]
        view.copy_(t)
        return view

    def forward(self, **more):
        return cc.group_norm_fwd(self.x, self.groups, weight=self.w, bias=self.b, act=self.kind, eps=self.eps,
                                 dtype=self.layer, save=True, **more)

    def backward(self, r):
        return cc.group_norm_bwd(self.x, self.groups, r.mean, r.rstd, self.dy, weight=self.w, bias=self.b, act=self.kind)

    def check(self):
        x, w, b = f64(self.x), f64(self.w), f64(self.b)
        r = self.forward()
        y, mean, rstd, ey, em, er = ref.forward(x, self.groups, w, b, self.kind, self.eps, NAMES[self.layer])
        assert r.y.dtype == self.layer
        close(r.mean, mean, em, "mean")
        close(r.rstd, rstd, er, "rstd")
        close(r.y, y, ey, "y")
        g = self.backward(r)
        dx, dw, db, edx, edw, edb = ref.backward(x, self.groups, f64(r.mean), f64(r.rstd), f64(self.dy), w, b, self.kind,
                                                 NAMES[self.layer])
        assert g.dx.dtype == self.layer
        close(g.dx, dx, edx, "dx")
        if self.w is not None:
            close(g.dweight, dw, edw, "dweight")
            close(g.dbias, db, edb, "dbias")
        else:
            assert g.dweight is None and g.dbias is None
        return r, g


# one value, one position; whole vectors, halves, odd columns; groups narrower than a vector; many images; groups that fill a
# workgroup's registers and that do not; groups wider than a workgroup's columns; more groups than threads
SHAPES = [(1, 1, 1, 1), (2, 1, 8, 2), (3, 5, 12, 3), (2, 7, 27, 1), (2, 49, 54, 2), (1, 64, 256, 32), (5, 33, 96, 32),
          (2, 64, 864, 32), (1, 1024, 108, 4), (3, 1, 4096, 32), (2, 1, 4096, 1), (1, 256, 1024, 4), (1, 1200, 512, 2),
          (1, 700, 2050, 1), (1, 300, 6000, 2), (2, 9, 2000, 1000), (300, 2, 64, 4), (1, 3000, 30, 10), (2, 513, 1300, 4)]


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, types):
    Case(*shape, types).check()


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("positions", [240, 560])
def test_many_images_of_odd_groups(positions, types):
    """Vectors that straddle groups: slabs that share a CU, and that would fill it alone."""
    Case(520, positions, 120, 4, types).check()


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("affine", [True, False])
def test_activations(kind, affine, types):
    Case(3, 40, 128, 4, types, kind, affine).check()
    Case(1, 2500, 256, 2, types, kind, affine).check()


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("gap,shift", [(8, 0), (5, 0), (0, 3), (1, 1), (64, 8)])
def test_strides_and_addresses(gap, shift, types):
    Case(2, 21, 120, 3, types, gap=gap, shift=shift).check()
    Case(1, 1300, 640, 2, types, gap=gap, shift=shift).check()


@pytest.mark.parametrize("shape", [(2, 64, 128, 4), (1, 3000, 640, 2)])
@pytest.mark.parametrize("offset", [100.0, -3e4])
def test_values_far_from_zero(shape, offset):
    """The variance does not come from the difference of two large numbers."""
    Case(*shape, (FP32, FP32), offset=offset).check()


@pytest.mark.parametrize("shape", [(2, 64, 128, 4), (1, 3000, 640, 2)])
def test_equal_values(shape):
    """A group without variance: y = act(bias)."""
    c = Case(*shape, (FP32, FP32))
    c.x.fill_(7.25)
    r = c.forward()
    assert (r.mean == 7.25).all()
    close(r.rstd, np.full(r.rstd.shape, 1e-5 ** -0.5), np.full(r.rstd.shape, 1e-5 ** -0.5 * 1e-6), "rstd")
    want = ref.act("silu", f64(c.b))
    close(r.y[0], np.broadcast_to(want, c.x.shape[1:]), np.full(c.x.shape[1:], 1e-5), "y")


@pytest.mark.parametrize("shape", [(3, 64, 128, 4), (2, 3000, 640, 2), (2, 50, 27, 1)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_infinities_and_nan_stay_in_their_group(shape, value):
    c = Case(*shape, (BF16, BF16))
    good = c.forward()
    bad = (1, 11, shape[2] // shape[3])  # the second group's first column, where there is one
    at = bad if shape[3] > 1 else (1, 11, 3)
    c.x[at] = value
    r = c.forward()
    n, g = 1, at[2] // (shape[2] // shape[3])
    keep = torch.ones((shape[0], shape[3]), dtype=torch.bool, device="cuda")
    keep[n, g] = False
    of = lambda t: t.reshape(shape[0], shape[1], shape[3], -1).transpose(1, 2)[keep]  # noqa: E731
    assert torch.equal(of(r.y), of(good.y)) and torch.isnan(r.rstd[n, g])
    d = c.backward(r)
    assert torch.isfinite(of(d.dx)).all()


@pytest.mark.parametrize("shape", [(2, 64, 128, 4), (1, 3000, 640, 2)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_in_place(shape, dtype):
    c = Case(*shape, (dtype, dtype))
    want = c.forward()
    again = cc.group_norm_fwd(c.x, c.groups, weight=c.w, bias=c.b, act=c.kind, dtype=dtype, y=c.x)
    assert again.y is c.x and torch.equal(again.y, want.y) and again.mean is None


def test_positions_and_channels_of_an_activation():
    """[N,H,W,C,D0,D1,D2] with all capsules of a pixel as its channels."""
    c = Case(2, 6 * 5, 4 * 2 * 3 * 4, 4, (BF16, BF16))
    want = c.forward()
    x = c.x.view(2, 6, 5, 4, 2, 3, 4)
    got = cc.group_norm_fwd(x, 4, weight=c.w.view(4, 2, 3, 4), bias=c.b, act=c.kind, channel_dims=4, save=True)
    assert got.y.shape == x.shape and torch.equal(got.y.view_as(want.y), want.y)
    g, k = c.backward(want), cc.group_norm_bwd(x, 4, got.mean, got.rstd, c.dy.view_as(x), weight=c.w, bias=c.b, act=c.kind,
                                              channel_dims=4)
    assert torch.equal(g.dx.view_as(x), k.dx) and torch.equal(g.dweight, k.dweight)


@pytest.mark.parametrize("shape", [(3, 64, 128, 4), (1, 2000, 512, 2)])
def test_broadcast_gradient(shape):
    """A gradient that is the same at all positions (that of a mean over them), of stride 0."""
    c = Case(*shape, (FP32, FP32))
    r = c.forward()
    c.dy = c.dy[:1, :1].expand(c.dy.shape)
    got = c.backward(r)
    c.dy = c.dy.contiguous()
    want = c.backward(r)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(3, 64, 128, 4), (1, 2000, 512, 2)])
def test_graph_and_stream(shape):
    """Captured and replayed with other values, between eager calls; on another stream."""
    c = Case(*shape, (BF16, BF16))
    first = c.x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = c.forward()
        g = c.backward(r)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cr = c.forward()
        cg = c.backward(cr)
    for k in range(4):
        c.x.copy_(first * (1.0 + 0.5 * k))
        graph.replay()
        want = c.forward()
        grads = c.backward(want)
        torch.cuda.synchronize()
        for a, b in zip((*cr, *cg), (*want, *grads)):
            assert torch.equal(a, b), k
    c.x.copy_(first)
    again = c.forward()
    for a, b in zip((*again, *c.backward(again)), (*r, *g)):
        assert torch.equal(a, b)


def test_offsets_past_32_bits():
    images, positions, width = 3, 70, 16384
    wide = torch.empty((images, positions, 1 << 24), dtype=BF16, device="cuda")  # 7 GB: rows 32 MB apart
    x = wide[:, :, :width]
    small = torch.randn((images, positions, width), generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    x.copy_(small)
    got = cc.group_norm_fwd(x, 32, act="silu", save=True)
    want = cc.group_norm_fwd(small, 32, act="silu", save=True)
    assert torch.equal(got.y, want.y)
    dy = small.flip(0).contiguous()
    a, b = (cc.group_norm_bwd(t, 32, want.mean, want.rstd, dy, act="silu") for t in (x, small))
    assert torch.equal(a.dx, b.dx)


@pytest.mark.parametrize("types", [(FP32, FP32)])
@pytest.mark.parametrize("shape", [(2, 6, 12, 3), (1, 600, 40, 2)])
@pytest.mark.parametrize("kind", ACTS)
def test_gradients_against_differences(shape, kind, types):
    """Along the gradients themselves, the sum of y * dy changes by their squares."""
    c = Case(*shape, types, kind)
    g = c.backward(c.forward())
    for at, grad in ((c.x, g.dx), (c.w, g.dweight), (c.b, g.dbias)):
        before, step = at.clone(), 1e-2 / float(grad.norm())
        value = []
        for sign in (1, -1):
            at.copy_(before + sign * step * grad)
            value.append(float((f64(c.forward().y) * f64(c.dy)).sum()))
        at.copy_(before)
        slope, want = (value[0] - value[1]) / (2 * step), float(f64(grad.flatten()) @ f64(grad.flatten()))
        # y is off by 1e-6 of values of size 1 at `numel` places, in effect at random, and the quotient of third order in a step
        # of 1e-2 along a gradient; 2 % leaves a factor of ten
        noise = 1e-6 * np.sqrt(c.x.numel()) * 3 / step
        assert abs(slope - want) <= 0.02 * want + noise, (slope, want)

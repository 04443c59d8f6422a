"""GPU parity of the norms around a block (forward and backward) against their formulas in 64 bits: every element type,
gate and activation, rows of one value to rows beyond every kernel's tile, rows at odd strides and addresses, rows of
zeros, infinities and NaN, offsets past 32 bits.  Tolerances: tests/block_norm_ref.py, from the
number of roundings; inputs are what the storage type holds, so both sides read the same values."""
import numpy as np
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import block_norm_ref as ref

pytestmark = pytest.mark.gpu

FP32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(FP32, FP32, FP32), (BF16, BF16, BF16), (BF16, FP32, BF16), (BF16, BF16, FP32), (BF16, FP32, FP32),
         (FP16, FP16, FP16), (FP16, FP32, FP32)]
NAMES = {FP32: "f32", BF16: "bf16", FP16: "f16"}


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def close(got, want, err, what):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - err
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}{at}: {got[at]} for {want[at]}, bound {err[at]}"


class Case:
    def __init__(self, rows, width, types, gate=None, kind="linear", post=True, seed=0, gap=0, shift=0, rs=1.0, bs=1.0):
        self.rows, self.width, self.gate_kind, self.kind, self.post, self.rs, self.bs = rows, width, gate, kind, post, rs, bs
        self.layer, self.stream, self.branch = types
        self.gap, self.shift, self.eps = gap, shift, 1e-6
        rng = torch.Generator().manual_seed(1000 * rows + width + seed)
        scale = torch.exp(torch.randn((rows, 1), generator=rng))

        def make(dtype, sigma):
            return self.place((torch.randn((rows, width), generator=rng) * scale * sigma).to(dtype))

        def vector(mean, sigma):
            return (mean + sigma * torch.randn(width, generator=rng)).cuda()

        self.x, self.b = make(self.stream, 1.0), make(self.branch, 0.5)
        self.dh, self.dy = make(self.layer, 0.1), make(self.stream, 0.1)
        self.wpre, self.wpost = vector(1.0, 0.2), vector(1.0, 0.2)
        self.gate = vector(0.5, 0.5) if gate == "shared" else make(self.layer, 1.0) if gate == "full" else None

    def place(self, t):
        """On the GPU, rows `gap` values apart, the first `shift` values into its allocation."""
        if not self.gap and not self.shift:
            return t.cuda()
        wide = torch.full((t.shape[0] * (t.shape[1] + self.gap) + self.shift,), float("nan"), dtype=t.dtype, device="cuda")
        view = wide[self.shift:].view(t.shape[0], t.shape[1] + self.gap)[:, :t.shape[1]]
        view.copy_(t)
        return view

    def same(self):
        return dict(pre_weight=self.wpre, post_weight=self.wpost if self.post else None, gate=self.gate, gate_act=self.kind,
                    post_norm=self.post, residual_scale=self.rs, branch_scale=self.bs, dtype=self.layer)

    def forward(self, **more):
        return cc.block_norm_fwd(self.x, self.b, eps=self.eps, save=True, **self.same(), **more)

    def check_forward(self, r):
        x, b, g, wpost = f64(self.x), f64(self.b), f64(self.gate), f64(self.wpost)
        y, h, rpre, rpost = ref.forward(x, b, f64(self.wpre), wpost, g, self.kind, self.post, self.rs, self.bs, self.eps)
        e = ref.forward_bounds(x, b, y, h, rpre, wpost, g, self.kind, self.post, self.rs, self.bs, rpost)
        close(r.y, y, ref.stored(e["y"], y, self.stream), "y")
        close(r.h, h, ref.stored(e["h"], h, self.layer), "h")
        close(r.rstd_pre, rpre, e["rpre"] + 4 * ref.U * rpre, "rstd_pre")
        if self.post:
            close(r.rstd_post, rpost, e["rpost"] + 4 * ref.U * rpost, "rstd_post")
        else:
            assert r.rstd_post is None
        assert r.y.dtype == self.stream and r.h.dtype == self.layer

    def stats(self):
        """Of x as the stored y, as fp32."""
        rpre, rpost = (torch.from_numpy((1.0 / np.sqrt((f64(t) ** 2).mean(1) + self.eps)).astype(np.float32)).cuda()
                       for t in (self.x, self.b))
        return rpre, rpost if self.post else None

    def backward(self, dh=True, dy=True):
        return cc.block_norm_bwd(self.x, self.b, *self.stats(), self.dh if dh else None, self.dy if dy else None, **self.same())

    def check_backward(self, r, dh=True, dy=True):
        rpre, rpost = self.stats()
        want = ref.backward(f64(self.x), f64(self.b), f64(rpre), f64(rpost), f64(self.dh) if dh else None,
                            f64(self.dy) if dy else None, f64(self.wpre), f64(self.wpost), f64(self.gate), self.kind,
                            self.post, self.rs, self.bs)
        outs = {"dx": (r.dx, self.stream), "db": (r.dbranch, self.layer), "dpre": (r.dpre_weight, FP32),
                "dpost": (r.dpost_weight, FP32), "dgate": (r.dgate, self.layer if self.gate_kind == "full" else FP32)}
        if not dh:
            assert r.dpre_weight is None
        for name, (got, dtype) in outs.items():
            if name not in want or name == "dpre" and not dh:
                assert got is None, name
                continue
            assert got.dtype == dtype, name
            close(got, want[name][0], ref.stored(want[name][1], want[name][0], dtype), name)


# rows of one value; rows that fill no vector, one, some lanes, a wave, several waves; rows beyond the widest tile
WIDTHS = [1, 2, 7, 8, 9, 16, 27, 63, 64, 100, 255, 512, 520, 600, 864, 1024, 1027, 2048, 2600, 4096, 5000, 8192, 16384,
          20001, 33000, 70000]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(NAMES[x] for x in t))
def test_widths_and_types(width, types):
    rows = 1 if width % 2 else 5
    if width <= 64:
        rows = 300 + width  # several rows in a wave, the last wave ragged
    c = Case(rows, width, types, gate="shared" if width % 3 else "full", kind="linear" if width % 5 else "silu", bs=0.5, rs=0.9)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("gate", [None, "shared", "full"])
@pytest.mark.parametrize("kind", ["linear", "sigmoid", "silu"])
@pytest.mark.parametrize("post", [True, False], ids=["post", "nopost"])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[2], TYPES[5]], ids=lambda t: "-".join(NAMES[x] for x in t))
def test_gates_and_norms(gate, kind, post, types):
    for rows, width in ((33, 72), (4, 1500)):
        c = Case(rows, width, types, gate, kind, post, rs=1.1, bs=-0.7)
        c.check_forward(c.forward())
        c.check_backward(c.backward())


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 1000, 4099, 20000])
@pytest.mark.parametrize("width", [20, 640])
def test_row_counts(rows, width):
    c = Case(rows, width, TYPES[rows % 2], "shared")
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("rows,width,types,gate", [
    (1100, 9000, TYPES[1], "shared"), (1100, 9001, TYPES[0], "shared"), (700, 16384, TYPES[6], "full"),
    (2300, 5003, TYPES[0], "full"), (2300, 6000, TYPES[2], None), (9001, 1100, TYPES[1], "shared"),
    (9000, 1027, TYPES[3], "full"), (150001, 27, TYPES[0], "full"), (300001, 16, TYPES[1], "shared"),
    (300001, 13, TYPES[5], "full"), (70001, 64, TYPES[4], "shared"), (1000003, 3, TYPES[1], None)],
    ids=lambda v: v if isinstance(v, (int, str)) else None)
def test_more_rows_than_workgroups(rows, width, types, gate):
    """Each kernel with workgroups that take several rounds of rows, the last one ragged."""
    c = Case(rows, width, types, gate, "silu" if gate == "full" else "linear", rs=0.9)
    c.check_forward(c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("width", [8, 27, 64, 600, 2048, 4100])
@pytest.mark.parametrize("gap,shift", [(0, 1), (8, 0), (5, 0), (3, 3)])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[1], TYPES[4]], ids=lambda t: "-".join(NAMES[x] for x in t))
def test_strides_and_addresses(width, gap, shift, types):
    """Rows apart and rows off every vector's alignment, outputs too; what lies between the rows is NaN before and after."""
    c = Case(37, width, types, "full", "sigmoid", gap=gap, shift=shift)
    y, h = (c.place(torch.zeros((37, width), dtype=t)) for t in (c.stream, c.layer))
    c.check_forward(c.forward(y=y, h=h))
    for t in (y, h):
        if gap:
            wide = t.as_strided((36, gap), (width + gap, 1), t.storage_offset() + width)
            assert torch.isnan(wide).all()
    c.check_backward(c.backward())


@pytest.mark.parametrize("width", [13, 64, 1027])
def test_one_row_broadcast_to_many(width):
    """Inputs of stride 0, and rows that overlap their neighbours: nothing behind the last value is read."""
    c = Case(1, width, TYPES[1])
    many = [t.expand(70, width) for t in (c.x, c.b, c.dh, c.dy)]
    dense = [t.contiguous() for t in many]
    stats = [torch.rsqrt(t.double().square().mean(1) + c.eps).float() for t in dense[:2]]
    for a, b in zip(cc.block_norm_fwd(*many[:2], pre_weight=c.wpre), cc.block_norm_fwd(*dense[:2], pre_weight=c.wpre)):
        assert a is None or torch.equal(a, b)
    for a, b in zip(cc.block_norm_bwd(*many[:2], *stats, *many[2:], pre_weight=c.wpre),
                    cc.block_norm_bwd(*dense[:2], *stats, *dense[2:], pre_weight=c.wpre)):
        assert a is None or torch.equal(a, b)
    line = torch.randn(width + 30, device="cuda").to(BF16)
    sliding = line.as_strided((31, width), (1, 1))
    assert torch.equal(cc.block_norm_fwd(sliding).h, cc.block_norm_fwd(sliding.contiguous()).h)


def test_without_a_branch_and_with_one_gradient():
    for types in (TYPES[0], TYPES[2]):
        c = Case(19, 200, types, "shared")
        r = cc.block_norm_fwd(c.x, pre_weight=c.wpre, eps=c.eps, dtype=c.layer, save=True)
        assert r.y is None and r.rstd_post is None
        x = f64(c.x)
        y, h, rpre, _ = ref.forward(x, None, f64(c.wpre), None, None, "linear", False, 1, 1, c.eps)
        e = ref.forward_bounds(x, None, y, h, rpre, None, None, "linear", False, 1, 1, None)
        close(r.h, h, ref.stored(e["h"], h, c.layer), "h")
        g = cc.block_norm_bwd(c.x, None, r.rstd_pre, None, c.dh, c.dy, pre_weight=c.wpre)
        want = ref.backward(x, None, f64(r.rstd_pre), None, f64(c.dh), f64(c.dy), f64(c.wpre), None, None, "linear", False, 1, 1)
        close(g.dx, want["dx"][0], ref.stored(want["dx"][1], want["dx"][0], c.stream), "dx")
        close(g.dpre_weight, want["dpre"][0], want["dpre"][1] + 1e-30, "dpre")
        assert g.dbranch is None and g.dgate is None and g.dpost_weight is None
        c.check_backward(c.backward(dh=False), dh=False)
        c.check_backward(c.backward(dy=False), dy=False)


def test_wanted_outputs_only_and_in_place():
    c = Case(50, 264, TYPES[2], "shared")
    both = c.forward()
    assert torch.equal(cc.block_norm_fwd(c.x, c.b, want_y=False, eps=c.eps, **c.same()).h, both.h)
    only = cc.block_norm_fwd(c.x, c.b, want_h=False, eps=c.eps, **c.same())
    assert only.h is None and torch.equal(only.y, both.y)
    for width in (264, 40000):   # y in the place of x
        c = Case(6, width, TYPES[2], "shared")
        both = c.forward()
        again = c.forward(y=c.x)
        assert again.y is c.x and torch.equal(c.x, both.y) and torch.equal(again.h, both.h)


def test_seven_axes_as_the_layers_have_them():
    """[N,H,W,C,D0,D1,D2]: all capsules of a pixel together, each by itself, and channels cut out of a wider tensor."""
    x = torch.randn((2, 3, 4, 5, 1, 4, 6), generator=torch.Generator().manual_seed(5)).cuda()
    wide = torch.zeros((2, 3, 4, 9, 1, 4, 6), device="cuda")
    wide[:, :, :, 2:7] = x
    for dims, width in ((4, 120), (3, 24)):
        w = torch.randn(width, device="cuda")
        flat = cc.block_norm_fwd(x.reshape(-1, width), pre_weight=w).h
        assert torch.equal(cc.block_norm_fwd(x, pre_weight=w, norm_dims=dims).h.reshape(-1, width), flat)
    w = torch.randn(120, device="cuda")
    assert torch.equal(cc.block_norm_fwd(wide[:, :, :, 2:7], pre_weight=w, norm_dims=4).h,
                       cc.block_norm_fwd(x, pre_weight=w, norm_dims=4).h)
    with pytest.raises(ValueError, match="equal distances"):   # capsules of a cut: two distances
        cc.block_norm_fwd(wide[:, :, :, 2:7], norm_dims=3)
    with pytest.raises(ValueError, match="next to each other"):
        cc.block_norm_fwd(x.transpose(5, 6), norm_dims=3)


@pytest.mark.parametrize("width", [27, 512, 6000, 40000])
def test_rows_of_zeros_infinities_and_nan(width):
    c = Case(8, width, TYPES[0], "shared")
    clean, grads = c.forward(), c.backward()
    c.x[1], c.b[1], c.dh[1], c.dy[1] = 0.0, 0.0, 0.0, 0.0
    c.x[3, width // 2] = float("inf")
    c.b[4, width - 1] = float("nan")
    c.x[6] = 1e30   # squares pass the largest float: as infinity
    r = c.forward()
    assert (r.y[1] == 0).all() and (r.h[1] == 0).all()
    assert torch.isnan(r.h[4]).all() and torch.isnan(r.y[4]).all()
    assert torch.isinf(r.y[3, width // 2]) and torch.isnan(r.h[3, width // 2])
    assert (r.h[6] == 0).all() and (r.rstd_pre[6] == 0).all()
    for k in (0, 2, 5, 7):
        assert torch.equal(r.h[k], clean.h[k]) and torch.equal(r.y[k], clean.y[k])
    c.b[4, width - 1] = 0.0
    c.x[3, width // 2] = 0.0
    c.x[6] = 0.0
    stats = [torch.rsqrt(t.double().square().mean(1) + c.eps).float() for t in (c.x, c.b)]
    c.dh[4, 0] = float("nan")
    g = cc.block_norm_bwd(c.x, c.b, *stats, c.dh, c.dy, **c.same())
    assert (g.dx[1] == 0).all() and (g.dbranch[1] == 0).all()
    assert torch.isnan(g.dx[4]).all() and torch.isnan(g.dpre_weight[0])
    assert torch.isfinite(g.dpre_weight[1:]).all()   # (the mean of row 4 reaches the other sums)
    for k in (0, 2, 5, 7):
        assert torch.equal(g.dx[k], grads.dx[k]) and torch.equal(g.dbranch[k], grads.dbranch[k])


def test_differences_of_the_kernel_itself():
    """The kernels' own forward pass moved along a direction, in fp32 with steps of 2^-7: the loss is a sum of 2 * 5120
    products of magnitude around 0.1, off by about sqrt(10240) * 0.1 * 2^-23, over 2^-6; the third derivative adds 2^-14 of the derivative's magnitude."""
    c = Case(16, 320, TYPES[0], "full", "silu")
    r = c.forward()
    g = cc.block_norm_bwd(r.y, c.b, r.rstd_pre, r.rstd_post, c.dh, c.dy, **c.same())

    def loss():
        r = c.forward()
        return float((r.y.double() * c.dy.double()).sum() + (r.h.double() * c.dh.double()).sum())

    for t, d in ((c.x, g.dx), (c.b, g.dbranch), (c.gate, g.dgate), (c.wpre, g.dpre_weight), (c.wpost, g.dpost_weight)):
        way = torch.randn(t.shape, generator=torch.Generator().manual_seed(3)).cuda() * t.abs().mean()
        keep = t.clone()
        step = 2.0 ** -7
        t.copy_(keep + step * way)
        up = loss()
        t.copy_(keep - step * way)
        down = loss()
        t.copy_(keep)
        want = float((d.double() * way.double()).sum())
        size = float((d.double() * way.double()).abs().sum())
        assert abs((up - down) / (2 * step) - want) <= 1e-2 * size + 1e-3


def test_runs_repeat_bit_for_bit_and_on_a_side_stream():
    c = Case(3000, 136, TYPES[2], "shared", "sigmoid")
    a, b = c.backward(), c.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s, f = c.backward(), c.forward()
    torch.cuda.synchronize()
    for x, y, z in zip(a, b, s):
        assert torch.equal(x, y) and torch.equal(x, z)
    c.check_forward(f)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_offsets_past_32_bits(dtype):
    """Two rows more than 2^31 values apart, and 2^31 values in dense rows."""
    apart = (1 << 31) + 8
    buf = torch.empty(apart + 64, dtype=dtype, device="cuda")
    x = buf.as_strided((2, 64), (apart, 1))
    x.copy_(torch.randn((2, 64), generator=torch.Generator().manual_seed(1)))
    near = x.clone()
    assert torch.equal(cc.block_norm_fwd(x).h, cc.block_norm_fwd(near).h)
    out = buf.as_strided((2, 64), (apart, 1))
    want = cc.block_norm_fwd(near, near)
    got = cc.block_norm_fwd(x, near, y=out)
    assert torch.equal(got.y, want.y) and torch.equal(got.h, want.h)
    del buf, x, out, got
    if dtype == FP32:
        return
    rows = (1 << 31) // 4096 + 3
    x = torch.zeros((rows, 4096), dtype=dtype, device="cuda")
    x[-3:] = torch.randn((3, 4096), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    r = cc.block_norm_fwd(x, save=True)
    assert torch.equal(r.h[-3:], cc.block_norm_fwd(x[-3:].contiguous()).h)
    dh = torch.zeros_like(x)
    dh[-3:] = x[-3:]
    g = cc.block_norm_bwd(x, None, r.rstd_pre, None, dh, None)
    few = cc.block_norm_bwd(x[-3:].contiguous(), None, r.rstd_pre[-3:].contiguous(), None, dh[-3:].contiguous(), None)
    assert torch.equal(g.dx[-3:], few.dx)

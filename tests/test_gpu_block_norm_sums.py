"""The block norm's sums over rows, bit for bit.  Gradients, stream and branch are 1 or 2, statistics 1, scales and weights powers
of two, so that every product is a whole number from 1 on, and every sum of them, in any order, is exact in fp32 (below
2^24).  Each row adds at least 1 to each column: a row, a workgroup or a round that is lost or taken twice
changes every sum.  (A bound on the rounding of sums over so many rows is as large as the sums.)  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests.test_gpu_block_norm import Case

pytestmark = pytest.mark.gpu

FP32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16


def ones_and_twos(rows, width, dtype, gen, gap=0):
    t = torch.randint(1, 3, (rows, width), generator=gen, device="cuda", dtype=torch.uint8).to(dtype)
    if not gap:
        return t
    wide = torch.full((rows * (width + gap),), float("nan"), dtype=dtype, device="cuda").view(rows, width + gap)
    wide[:, :width] = t
    return wide[:, :width]


def check(rows, width, layer, stream, branch, gap=0):
    gen = torch.Generator(device="cuda").manual_seed(rows + width)
    y, b, dh, dy = (ones_and_twos(rows, width, t, gen, gap) for t in (stream, branch, layer, stream))
    one = torch.ones(rows, device="cuda")
    wpre, wpost, gate = (2.0 ** torch.randint(-1, 2, (width,), generator=gen, device="cuda").float() for _ in range(3))

    def columns(s, t):
        return (s.double() * t.double()).sum(0)

    r = cc.block_norm_bwd(y, b, one, one, dh, None, pre_weight=wpre, post_weight=wpost, gate=gate, dtype=layer)
    assert torch.equal(r.dpre_weight.double(), columns(dh, y))
    sums = columns(dy, b)
    r = cc.block_norm_bwd(y, b, None, one, None, dy, post_weight=wpost, gate=gate, branch_scale=0.5, dtype=layer)
    assert torch.equal(r.dpost_weight.double(), sums * 0.5 * gate.double())
    assert torch.equal(r.dgate.double(), sums * 0.5 * wpost.double())
    if gap:   # what lies between the rows stays as it was
        for t in (y, b, dh, dy):
            assert torch.isnan(t.as_strided((rows - 1, gap), (width + gap, 1), t.storage_offset() + width)).all()


TYPES = {"fp32": (FP32, FP32, FP32), "bf16": (BF16, BF16, BF16), "bf16-32-16": (BF16, FP32, BF16),
         "fp16-16-32": (FP16, FP16, FP32), "fp16-32-32": (FP16, FP32, FP32)}


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,width", [
    (1, 4096), (5, 27), (255, 640), (1000003, 3), (300001, 16), (150001, 27), (70001, 64), (20011, 280), (9001, 640),
    (9001, 1100), (9000, 1027), (2300, 4096), (2300, 5003), (1100, 8192), (1100, 9001), (700, 16384), (3001, 20001)])
def test_every_row_is_in_the_sums_once(rows, width, types):
    check(rows, width, *TYPES[types])


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,width", [(2, 64), (600, 27), (600, 64), (600, 1000), (300, 4100), (300, 9000)])
def test_rows_far_apart(rows, width, types):
    """Past the reach of a workgroup's 32-bit offsets, where each row is a workgroup's by itself."""
    check(rows, width, *TYPES[types], gap=(1 << 18) + 5)


@pytest.mark.parametrize("types", ["fp32", "bf16", "fp16-32-32"])
@pytest.mark.parametrize("rows,width,gate", [(300, 27, "full"), (300, 64, "shared"), (60, 1000, "full"), (60, 9000, "shared")])
def test_rows_far_apart_one_by_one(rows, width, gate, types):
    c = Case(rows, width, TYPES[types], gate, "silu" if gate == "full" else "linear", gap=(1 << 18) + 5, bs=0.5)
    c.check_forward(c.forward())
    c.check_backward(c.backward())

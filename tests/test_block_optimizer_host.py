"""Host-side checks of the block norm, the gradient norm and AdamW that need no GPU: refusals before anything is
launched, sizes of scratch, layouts of the argument structures, the hash that rounds 8-bit moments."""
import ctypes
import re
import subprocess
from pathlib import Path

import numpy as np
import pytest

from paper_2104_02621_amd import capscaps as cc
from tests import adamw_ref as ref

ROOT = Path(__file__).resolve().parent.parent
FAKE = 0x10000  # an aligned non-null "pointer"; never dereferenced on these error paths
NAN, INF = float("nan"), float("inf")


def block(**over):
    a = dict(rows=4, width=8, dtype=cc.BF16, stream_dtype=cc.FP32, branch_dtype=cc.BF16, post_norm=1,
             gate=cc.GATE_SHARED, gate_act=cc.ACT_LINEAR, residual_scale=1.0, branch_scale=1.0, eps=1e-6)
    a.update(over)
    return cc.BlockArgs(**a)


def fwd(**over):
    a = dict(x=FAKE, branch=FAKE, gate=FAKE, pre_weight=FAKE, post_weight=FAKE, y=2 * FAKE, h=FAKE, rstd_pre=FAKE,
             rstd_post=FAKE, x_stride=8, branch_stride=8, gate_stride=0, y_stride=8, h_stride=8)
    a.update(over)
    return cc.BlockFwdArgs(**a)


def bwd(**over):
    a = dict(y=FAKE, branch=FAKE, gate=FAKE, pre_weight=FAKE, post_weight=FAKE, rstd_pre=FAKE, rstd_post=FAKE, dh=FAKE,
             dy=FAKE, dx=FAKE, dbranch=FAKE, dgate=FAKE, dpre_weight=FAKE, dpost_weight=FAKE, y_stride=8,
             branch_stride=8, gate_stride=0, dh_stride=8, dy_stride=8, dx_stride=8, dbranch_stride=8, dgate_stride=8)
    a.update(over)
    return cc.BlockBwdArgs(**a)


BAD_BLOCKS = [dict(rows=0), dict(rows=-1), dict(width=0), dict(dtype=3), dict(dtype=cc.FP16), dict(stream_dtype=cc.FP16),
              dict(branch_dtype=7), dict(post_norm=2), dict(gate=3), dict(gate=-1), dict(gate_act=3), dict(eps=0.0),
              dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(residual_scale=NAN), dict(branch_scale=INF),
              dict(rows=1 << 62), dict(width=(1 << 30) + 1), dict(gate=cc.GATE_NONE)]


@pytest.mark.parametrize("over", BAD_BLOCKS, ids=str)
def test_blocks_are_refused(over):
    b = block(**over)
    assert cc.capscaps_block_norm_fwd(b, fwd()) == cc.EINVAL
    assert cc.capscaps_block_norm_bwd(b, bwd(), FAKE, 1 << 40) == cc.EINVAL
    if "gate" not in over or over["gate"] != cc.GATE_NONE:
        assert cc.capscaps_block_norm_bwd_workspace_bytes(b) == 0
    assert cc.capscaps_block_norm_fwd(None, fwd()) == cc.EINVAL
    assert cc.capscaps_block_norm_fwd(block(), None) == cc.EINVAL
    assert cc.capscaps_block_norm_bwd(block(), None, FAKE, 1 << 40) == cc.EINVAL


@pytest.mark.parametrize("over", [dict(x=None), dict(y=None, h=None), dict(branch=None), dict(gate=None),
                                  dict(x=FAKE + 2), dict(branch=FAKE + 1), dict(gate=FAKE + 2), dict(h=FAKE + 1),
                                  dict(pre_weight=FAKE + 2), dict(rstd_post=FAKE + 1), dict(x_stride=-8),
                                  dict(y_stride=7), dict(h_stride=0), dict(x_stride=1 << 60),
                                  dict(x=2 * FAKE, x_stride=16)], ids=str)
def test_forward_arguments_are_refused(over):
    assert cc.capscaps_block_norm_fwd(block(), fwd(**over)) == cc.EINVAL


@pytest.mark.parametrize("over", [dict(dh=None, dy=None), dict(y=None), dict(rstd_pre=None), dict(rstd_post=None),
                                  dict(branch=None), dict(gate=None), dict(dh=None),
                                  dict(dx=None, dbranch=None, dgate=None, dpre_weight=None, dpost_weight=None),
                                  dict(dx=FAKE + 1), dict(dgate=FAKE + 2), dict(dbranch_stride=4), dict(dy_stride=-1),
                                  dict(dpost_weight=FAKE + 2)], ids=str)
def test_backward_arguments_are_refused(over):
    assert cc.capscaps_block_norm_bwd(block(), bwd(**over), FAKE, 1 << 40) == cc.EINVAL
    assert cc.capscaps_block_norm_bwd(block(post_norm=0), bwd(), FAKE, 1 << 40) == cc.EINVAL   # dpost_weight


def test_backward_workspace_is_checked():
    need = cc.capscaps_block_norm_bwd_workspace_bytes(block())
    assert need > 0
    assert cc.capscaps_block_norm_bwd(block(), bwd(), None, 0) == cc.EWORKSPACE
    assert cc.capscaps_block_norm_bwd(block(), bwd(), FAKE, need - 1) == cc.EWORKSPACE
    assert cc.capscaps_block_norm_bwd(block(), bwd(), FAKE + 4, need) == cc.EINVAL


def grads(*items):
    return (cc.GradTensor * max(1, len(items)))(*items)


@pytest.mark.parametrize("call", [
    lambda: cc.capscaps_grad_norm(None, 1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads(), -1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, 1.0, None, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, 1.0, FAKE + 4, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 3)), 1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, -5, 0)), 1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((None, 5, 0)), 1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE + 2, 5, 0)), 1, 1.0, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, NAN, 1.0, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, NAN, FAKE, FAKE, 65536),
    lambda: cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, 1.0, FAKE, FAKE + 8, 65536),
])
def test_gradient_norm_arguments_are_refused(call):
    assert call() == cc.EINVAL


def test_gradient_norm_workspace_is_checked():
    assert cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, 1.0, FAKE, None, 0) == cc.EWORKSPACE
    assert cc.capscaps_grad_norm(grads((FAKE, 5, 0)), 1, 1.0, 1.0, FAKE, FAKE, 65535) == cc.EWORKSPACE
    assert cc.capscaps_grad_norm(grads((FAKE, 1 << 50, 0)), 1, 1.0, 1.0, FAKE, FAKE, 65536) == cc.EUNSUPPORTED
    many = grads(*[(FAKE, 1 << 32, 0)] * 100)
    assert cc.capscaps_grad_norm(many, 100, 1.0, 1.0, FAKE, FAKE, 65536) == cc.EUNSUPPORTED


def tensor(**over):
    a = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_exp=FAKE, v_exp=FAKE, copy=FAKE, n=10, weight_decay=0.1,
             grad_dtype=cc.FP32, copy_dtype=cc.BF16)
    a.update(over)
    return (cc.AdamwTensor * 1)(cc.AdamwTensor(**a))


def adamw(t, bits=32, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1, control=None, count=1):
    return cc.capscaps_adamw_step(t, count, bits, lr, b1, b2, eps, step, 0, control)


@pytest.mark.parametrize("over", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1),
                                  dict(weight_decay=NAN), dict(grad_dtype=5), dict(copy_dtype=cc.FP32),
                                  dict(param=FAKE + 2), dict(grad=FAKE + 2), dict(copy=FAKE + 1)], ids=str)
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_tensors_are_refused(over, bits):
    assert adamw(tensor(**over), bits) == cc.EINVAL


def test_adamw_arguments_are_refused():
    t = tensor()
    for over in (dict(bits=16), dict(lr=NAN), dict(b1=1.0), dict(b1=-0.1), dict(b2=NAN), dict(eps=0.0), dict(eps=1e-60),
                 dict(step=0), dict(step=-1), dict(step=1 << 40), dict(control=FAKE + 8), dict(count=-1)):
        assert adamw(t, **over) == cc.EINVAL, over
    assert adamw(None) == cc.EINVAL
    assert adamw(tensor(m=FAKE + 2)) == cc.EINVAL
    for over in (dict(m_exp=None), dict(v_exp=None)):
        assert adamw(tensor(**over), 8) == cc.EINVAL
    assert adamw(tensor(n=1 << 50)) == cc.EUNSUPPORTED
    # nothing to do is no error, and touches no GPU
    assert adamw(None, count=0) == cc.OK
    assert adamw(tensor(n=0, param=None, grad=None, m=None, v=None)) == cc.OK


def test_state_values_arguments_are_refused():
    out = (ctypes.c_void_p * 1)(FAKE)
    none = (ctypes.c_void_p * 1)(None)
    odd = (ctypes.c_void_p * 1)(FAKE + 1)
    assert cc.capscaps_adamw_state_values(tensor(), 1, out, none) == cc.EINVAL
    assert cc.capscaps_adamw_state_values(tensor(), 1, odd, out) == cc.EINVAL
    assert cc.capscaps_adamw_state_values(tensor(m_exp=None), 1, out, out) == cc.EINVAL
    assert cc.capscaps_adamw_state_values(tensor(), 1, None, out) == cc.EINVAL
    assert cc.capscaps_adamw_state_values(None, 0, None, None) == cc.OK


def test_python_wrappers_refuse_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU only"):
        cc.block_norm_fwd(x)
    with pytest.raises(ValueError, match="no rows"):
        cc.block_norm_fwd(x, norm_dims=3)
    with pytest.raises(ValueError, match="no rows"):
        cc.block_norm_fwd(torch.zeros(0, 8))
    with pytest.raises(ValueError, match="float32"):
        cc.block_norm_fwd(x.double())
    with pytest.raises(ValueError, match="gate_act"):
        cc.block_norm_fwd(x, gate_act="tanh")
    with pytest.raises(ValueError, match="dh or dy"):
        cc.block_norm_bwd(x, None, None, None, None, None)
    with pytest.raises(ValueError, match="contiguous device"):
        cc.AdamW([x])
    with pytest.raises(ValueError, match="float32"):
        cc.AdamW([x.half()])
    with pytest.raises(ValueError, match="state_bits"):
        cc.AdamW([x], state_bits=16)
    with pytest.raises(ValueError, match="needs parameters"):
        cc.AdamW([])
    with pytest.raises(ValueError, match="as many"):
        cc.AdamW([x], weight_decay=[0.1, 0.2])
    with pytest.raises(ValueError, match="no tensors"):
        cc.grad_norm([])


def test_argument_structures_have_the_headers_layout(tmp_path):
    structures = {"capscaps_block": cc.BlockArgs, "capscaps_block_fwd_args": cc.BlockFwdArgs,
                  "capscaps_block_bwd_args": cc.BlockBwdArgs, "capscaps_grad_tensor": cc.GradTensor,
                  "capscaps_adamw_tensor": cc.AdamwTensor}
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/capscaps.h"', "int main(void) {"]
    for name, s in structures.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in s._fields_]
    lines += ['printf("scratch %u\\n", CAPSCAPS_GRAD_NORM_WORKSPACE_BYTES);', "return 0; }"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "layout")], check=True)
    said = dict(line.split() for line in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True,
                                                        check=True).stdout.splitlines())
    for name, s in structures.items():
        assert int(said[name]) == ctypes.sizeof(s)
        for f, _ in s._fields_:
            assert int(said[f"{name}.{f}"]) == getattr(s, f).offset, f
    assert int(said["scratch"]) == cc.GRAD_NORM_WORKSPACE_BYTES
    header = (ROOT / "include" / "capscaps.h").read_text()
    for name, value in re.findall(r"#define CAPSCAPS_((?:GATE|ACT)_\w+) (\d)", header):
        assert getattr(cc, name) == int(value)


def test_random_bits_are_even_and_independent():
    """65536 values' bits, of several seeds, steps and tensors: means of 16-bit numbers and of their products, each within
    five standard deviations."""
    n = 65536
    for seed, step, k in ((0, 1, 0), (1, 1, 0), (0, 2, 0), (0, 1, 1), (12345, 999, 43)):
        a, b = (r / 65536 - 0.5 for r in ref.random16(0, n, seed, step, k))
        c, _ = (r / 65536 - 0.5 for r in ref.random16(0, n, seed, step + 1, k))
        d, _ = (r / 65536 - 0.5 for r in ref.random16(0, n, seed, step, k + 1))
        sigma = 1 / np.sqrt(12 * n)
        assert abs(a.mean()) < 5 * sigma and abs(b.mean()) < 5 * sigma
        for x, y in ((a, b), (a[1:], a[:-1]), (a, c), (a, d), (a[256:], a[:-256])):
            assert abs((x * y).mean()) < 5 / 12 / np.sqrt(n)


def test_reference_codes_come_back():
    """Each code, decoded and encoded with any random bits, is itself (the reference the GPU tests compare with)."""
    for signed, below, top in ((True, 15, 127), (False, 31, 255)):
        for e in (below + 1, 100, 127, 254):
            codes = np.arange(top + 1, dtype=np.uint8)
            codes = codes if e < 254 else codes[codes < top - 7]
            codes[0] = 0
            exps = np.array([e], dtype=np.uint8)
            values = ref.decode(codes, exps, signed)
            for r in (0, 65535):
                got, ge = ref.encode(values, np.full(len(values), r), signed)
                if ge[0] == e:
                    assert np.array_equal(got, codes)

"""ctypes binding of ``libcapscaps.so`` (C ABI in ``include/capscaps.h``).

Argument marshalling only: every step of the capsule convolution runs in the HIP library.
Functions carry the C names; ``conv_fwd`` is a convenience wrapper that takes torch tensors
(torch is used for device memory and streams only).  There is no CPU fallback: if the
library is missing or no GPU is present, calls fail.  They take no part in autograd: results have no history, also of inputs
that require gradients; the gradients are calls of their own.
"""
from __future__ import annotations

import ctypes
import math
import os
from collections import namedtuple
from pathlib import Path

FP32, BF16, FP16 = 0, 1, 2
PATH_AUTO, PATH_DIRECT, PATH_MFMA, PATH_MFMA_GENERIC, PATH_MFMA_TUNED16 = 0, 1, 2, 3, 4
PATH_MFMA_TUNED32 = 5
PATH_MFMA_SMALL = 6
OK, EINVAL, EWORKSPACE, EUNSUPPORTED, EHIP, ESCRATCH = 0, -1, -2, -3, -4, -5
STATIC_SCRATCH_BYTES = 80 << 20
GATE_NONE, GATE_SHARED, GATE_FULL = 0, 1, 2
ACT_LINEAR, ACT_SIGMOID, ACT_SILU = 0, 1, 2
GRAD_NORM_WORKSPACE_BYTES = 65536
MOST_ROW_VALUES = 1 << 30

# CAPSCAPS_SANITIZE=1 selects the build whose host code is instrumented (see build.py)
_LIB_PATH = Path(__file__).resolve().parent / (
    "libcapscaps.san.so" if os.environ.get("CAPSCAPS_SANITIZE") == "1" else "libcapscaps.so")
_lib = None


def _fields(names, ctype):
    return [(name, ctype) for name in names.split()]


class BlockArgs(ctypes.Structure):
    """capscaps_block"""
    _fields_ = (_fields("rows", ctypes.c_longlong)
                + _fields("width dtype stream_dtype branch_dtype post_norm gate gate_act", ctypes.c_int)
                + _fields("residual_scale branch_scale eps", ctypes.c_float))


class BlockFwdArgs(ctypes.Structure):
    """capscaps_block_fwd_args"""
    _fields_ = (_fields("x branch gate pre_weight post_weight y h rstd_pre rstd_post", ctypes.c_void_p)
                + _fields("x_stride branch_stride gate_stride y_stride h_stride", ctypes.c_longlong))


class BlockBwdArgs(ctypes.Structure):
    """capscaps_block_bwd_args"""
    _fields_ = (_fields("y branch gate pre_weight post_weight rstd_pre rstd_post dh dy dx dbranch dgate "
                        "dpre_weight dpost_weight", ctypes.c_void_p)
                + _fields("y_stride branch_stride gate_stride dh_stride dy_stride dx_stride dbranch_stride "
                          "dgate_stride", ctypes.c_longlong))


class GroupNormArgs(ctypes.Structure):
    """capscaps_group_norm"""
    _fields_ = (_fields("images positions", ctypes.c_longlong)
                + _fields("width groups x_dtype dtype act", ctypes.c_int) + [("eps", ctypes.c_float)])


class GroupFwdArgs(ctypes.Structure):
    """capscaps_group_fwd_args"""
    _fields_ = (_fields("x weight bias y mean rstd", ctypes.c_void_p) + _fields("x_stride y_stride", ctypes.c_longlong))


class GroupBwdArgs(ctypes.Structure):
    """capscaps_group_bwd_args"""
    _fields_ = (_fields("x weight bias mean rstd dy dx dweight dbias", ctypes.c_void_p)
                + _fields("x_stride dy_stride dx_stride", ctypes.c_longlong))


class HeadArgs(ctypes.Structure):
    """capscaps_head"""
    _fields_ = ([("rows", ctypes.c_longlong)]
                + _fields("width classes dtype index_bits top teacher_dtype", ctypes.c_int)
                + [("temperature", ctypes.c_float), ("gradient_terms", ctypes.c_int)])


_HEAD_TENSORS = (_fields("x weight bias index teacher", ctypes.c_void_p)
                 + _fields("x_stride weight_stride index_stride teacher_stride", ctypes.c_longlong))


class HeadFwdArgs(ctypes.Structure):
    """capscaps_head_fwd_args"""
    _fields_ = _HEAD_TENSORS + _fields("loss lse logq", ctypes.c_void_p)


class HeadBwdArgs(ctypes.Structure):
    """capscaps_head_bwd_args"""
    _fields_ = (_HEAD_TENSORS + _fields("loss lse logq dloss dx dweight dbias", ctypes.c_void_p)
                + [("dloss_stride", ctypes.c_longlong)])


class GradTensor(ctypes.Structure):
    """capscaps_grad_tensor"""
    _fields_ = [("grad", ctypes.c_void_p), ("n", ctypes.c_longlong), ("dtype", ctypes.c_int)]


class AdamwTensor(ctypes.Structure):
    """capscaps_adamw_tensor"""
    _fields_ = (_fields("param grad m v m_exp v_exp copy", ctypes.c_void_p) + [("n", ctypes.c_longlong)]
                + [("weight_decay", ctypes.c_float)] + _fields("grad_dtype copy_dtype", ctypes.c_int))


class CapscapsError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        detail = f" ({capscaps_last_hip_error()})" if status == EHIP else ""
        super().__init__(f"capscaps status {status}: {capscaps_strerror(status)}{detail}")


def library_path() -> Path:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise FileNotFoundError(
            f"{_LIB_PATH} is not built; run `python -m paper_2104_02621_amd.build`")
    # One HIP runtime per process: PyTorch ships its own libamdhip64 under the same soname as
    # ROCm's.  Importing torch first makes the dynamic loader resolve this library's dependency
    # to the copy torch already mapped, so streams and device pointers are shared.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(str(_LIB_PATH))
    i, p, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    ip = ctypes.POINTER(ctypes.c_int)
    lib.capscaps_out_shape.argtypes = [i] * 6 + [ip, ip]
    lib.capscaps_out_shape.restype = i
    lib.capscaps_conv_fwd.argtypes = [p, p, p] + [i] * 13 + [p]
    lib.capscaps_conv_fwd.restype = i
    lib.capscaps_conv_fwd_ex.argtypes = [p, p, p] + [i] * 14 + [p, sz, p]
    lib.capscaps_conv_fwd_ex.restype = i
    lib.capscaps_conv_fwd_static.argtypes = [p, p, p] + [i] * 14 + [p]
    lib.capscaps_conv_fwd_static.restype = i
    lib.capscaps_conv_fwd_out16_workspace_bytes.argtypes = [i] * 14
    lib.capscaps_conv_fwd_out16_workspace_bytes.restype = sz
    lib.capscaps_conv_fwd_out16.argtypes = [p, p, p] + [i] * 14 + [p, sz, p]
    lib.capscaps_conv_fwd_out16.restype = i
    lib.capscaps_conv_fwd_path.argtypes = [p, p, p] + [i] * 15 + [p, sz, p]
    lib.capscaps_conv_fwd_path.restype = i
    lib.capscaps_conv_fwd_workspace_bytes.argtypes = [i] * 14
    lib.capscaps_conv_fwd_workspace_bytes.restype = sz
    lib.capscaps_select_path.argtypes = [i] * 14
    lib.capscaps_select_path.restype = i
    for name in ("capscaps_conv_bwd_input", "capscaps_conv_bwd_kernel"):
        getattr(lib, name).argtypes = [p, p, p] + [i] * 14 + [p, sz, p]
        getattr(lib, name).restype = i
        getattr(lib, name + "_workspace_bytes").argtypes = [i] * 14
        getattr(lib, name + "_workspace_bytes").restype = sz
    lib.capscaps_conv_bwd_input_out16.argtypes = [p, p, p] + [i] * 14 + [p, sz, p]
    lib.capscaps_conv_bwd_input_out16.restype = i
    lib.capscaps_conv_bwd_input_out16_workspace_bytes.argtypes = [i] * 14
    lib.capscaps_conv_bwd_input_out16_workspace_bytes.restype = sz
    lib.capscaps_scheme2_index_bytes.argtypes = [i] * 14
    lib.capscaps_scheme2_index_bytes.restype = sz
    lib.capscaps_scheme2_build_index.argtypes = [p, sz] + [i] * 14 + [p]
    lib.capscaps_scheme2_build_index.restype = i
    lib.capscaps_scheme2_fwd.argtypes = [p, p, p, p, sz] + [i] * 14 + [p]
    lib.capscaps_scheme2_fwd.restype = i
    ll, f, d = ctypes.c_longlong, ctypes.c_float, ctypes.c_double
    lib.capscaps_block_norm_fwd.argtypes = [p, p, p]
    lib.capscaps_block_norm_fwd.restype = i
    lib.capscaps_block_norm_bwd_workspace_bytes.argtypes = [p]
    lib.capscaps_block_norm_bwd_workspace_bytes.restype = sz
    lib.capscaps_block_norm_bwd.argtypes = [p, p, p, sz, p]
    lib.capscaps_block_norm_bwd.restype = i
    for name in ("capscaps_group_norm_fwd", "capscaps_group_norm_bwd"):
        getattr(lib, name).argtypes = [p, p, p, sz, p]
        getattr(lib, name).restype = i
        getattr(lib, name + "_workspace_bytes").argtypes = [p]
        getattr(lib, name + "_workspace_bytes").restype = sz
    for name in ("capscaps_class_loss", "capscaps_distill_loss"):
        for way in ("_fwd", "_bwd"):
            getattr(lib, name + way).argtypes = [p, p, p, sz, p]
            getattr(lib, name + way).restype = i
        getattr(lib, name + "_workspace_bytes").argtypes = [p, i]
        getattr(lib, name + "_workspace_bytes").restype = sz
    lib.capscaps_grad_norm.argtypes = [p, i, f, f, p, p, sz, p]
    lib.capscaps_grad_norm.restype = i
    lib.capscaps_adamw_step.argtypes = [p, i, i, d, d, d, d, ll, ctypes.c_uint, p, p]
    lib.capscaps_adamw_step.restype = i
    lib.capscaps_adamw_state_values.argtypes = [p, i, p, p, p]
    lib.capscaps_adamw_state_values.restype = i
    lib.capscaps_mfma_yardstick.argtypes = [p, p, i, i, i, p]
    lib.capscaps_mfma_yardstick.restype = i
    lib.capscaps_mfma_yardstick_flops.argtypes = [i, i, i]
    lib.capscaps_mfma_yardstick_flops.restype = ctypes.c_double
    lib.capscaps_strerror.argtypes = [i]
    lib.capscaps_strerror.restype = ctypes.c_char_p
    lib.capscaps_last_hip_error.argtypes = []
    lib.capscaps_last_hip_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


# ------------------------------------------------------------------ C ABI, same names
def capscaps_strerror(status: int) -> str:
    return _load().capscaps_strerror(int(status)).decode()


def capscaps_last_hip_error() -> str:
    return _load().capscaps_last_hip_error().decode()


def capscaps_out_shape(H, W, kh, kw, stride, pad):
    """Returns (status, Ho, Wo)."""
    ho, wo = ctypes.c_int(0), ctypes.c_int(0)
    rc = _load().capscaps_out_shape(H, W, kh, kw, stride, pad, ctypes.byref(ho), ctypes.byref(wo))
    return rc, ho.value, wo.value


def capscaps_conv_fwd(input, kernel, out, N, H, W, C, M, kh, kw, stride, D0, D1, D2, D3, dtype,
                      stream=None) -> int:
    """Device pointers as ints; returns the status code."""
    return _load().capscaps_conv_fwd(input, kernel, out, N, H, W, C, M, kh, kw, stride, D0, D1,
                                     D2, D3, dtype, stream)


def capscaps_conv_fwd_ex(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                         dtype, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_fwd_ex(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad,
                                        D0, D1, D2, D3, dtype, workspace, workspace_bytes, stream)


def capscaps_conv_fwd_static(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                             dtype, stream=None) -> int:
    return _load().capscaps_conv_fwd_static(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad,
                                            D0, D1, D2, D3, dtype, stream)


def capscaps_conv_fwd_out16_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                                            dtype) -> int:
    return int(_load().capscaps_conv_fwd_out16_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad,
                                                               D0, D1, D2, D3, dtype))


def capscaps_conv_fwd_out16(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                            dtype, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_fwd_out16(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad,
                                           D0, D1, D2, D3, dtype, workspace, workspace_bytes,
                                           stream)


def capscaps_conv_fwd_path(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2,
                           D3, dtype, path, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_fwd_path(input, kernel, out, N, H, W, C, M, kh, kw, stride, pad,
                                          D0, D1, D2, D3, dtype, path, workspace,
                                          workspace_bytes, stream)


def capscaps_conv_fwd_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                                      dtype) -> int:
    return int(_load().capscaps_conv_fwd_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0,
                                                         D1, D2, D3, dtype))


def capscaps_select_path(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3, dtype) -> int:
    return int(_load().capscaps_select_path(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                                            dtype))


def capscaps_conv_bwd_input(dout, kernel, dinput, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2,
                            D3, dtype, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_bwd_input(dout, kernel, dinput, N, H, W, C, M, kh, kw, stride,
                                           pad, D0, D1, D2, D3, dtype, workspace, workspace_bytes,
                                           stream)


def capscaps_conv_bwd_input_out16(dout, kernel, dinput, N, H, W, C, M, kh, kw, stride, pad, D0, D1,
                                  D2, D3, dtype, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_bwd_input_out16(dout, kernel, dinput, N, H, W, C, M, kh, kw,
                                                 stride, pad, D0, D1, D2, D3, dtype, workspace,
                                                 workspace_bytes, stream)


def capscaps_conv_bwd_input_out16_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2,
                                                  D3, dtype) -> int:
    return int(_load().capscaps_conv_bwd_input_out16_workspace_bytes(N, H, W, C, M, kh, kw, stride,
                                                                     pad, D0, D1, D2, D3, dtype))


def capscaps_conv_bwd_kernel(input, dout, dkernel, N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2,
                             D3, dtype, workspace, workspace_bytes, stream=None) -> int:
    return _load().capscaps_conv_bwd_kernel(input, dout, dkernel, N, H, W, C, M, kh, kw, stride,
                                            pad, D0, D1, D2, D3, dtype, workspace,
                                            workspace_bytes, stream)


def capscaps_conv_bwd_input_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                                            dtype) -> int:
    return int(_load().capscaps_conv_bwd_input_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad,
                                                               D0, D1, D2, D3, dtype))


def capscaps_conv_bwd_kernel_workspace_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3,
                                             dtype) -> int:
    return int(_load().capscaps_conv_bwd_kernel_workspace_bytes(N, H, W, C, M, kh, kw, stride,
                                                                pad, D0, D1, D2, D3, dtype))


def capscaps_scheme2_index_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3, dtype) -> int:
    return int(_load().capscaps_scheme2_index_bytes(N, H, W, C, M, kh, kw, stride, pad, D0, D1,
                                                    D2, D3, dtype))


def capscaps_scheme2_build_index(index, index_bytes, N, H, W, C, M, kh, kw, stride, pad, D0, D1,
                                 D2, D3, dtype, stream=None) -> int:
    return _load().capscaps_scheme2_build_index(index, index_bytes, N, H, W, C, M, kh, kw, stride,
                                                pad, D0, D1, D2, D3, dtype, stream)


def capscaps_scheme2_fwd(input, kernel, out, index, index_bytes, N, H, W, C, M, kh, kw, stride,
                         pad, D0, D1, D2, D3, dtype, stream=None) -> int:
    return _load().capscaps_scheme2_fwd(input, kernel, out, index, index_bytes, N, H, W, C, M, kh,
                                        kw, stride, pad, D0, D1, D2, D3, dtype, stream)


def capscaps_block_norm_fwd(block, args, stream=None) -> int:
    """`block`, `args`: BlockArgs and BlockFwdArgs."""
    return _load().capscaps_block_norm_fwd(_ref(block), _ref(args), stream)


def capscaps_block_norm_bwd_workspace_bytes(block) -> int:
    return int(_load().capscaps_block_norm_bwd_workspace_bytes(_ref(block)))


def capscaps_block_norm_bwd(block, args, workspace, workspace_bytes, stream=None) -> int:
    """`block`, `args`: BlockArgs and BlockBwdArgs."""
    return _load().capscaps_block_norm_bwd(_ref(block), _ref(args), workspace, workspace_bytes, stream)


def capscaps_group_norm_fwd_workspace_bytes(norm) -> int:
    return int(_load().capscaps_group_norm_fwd_workspace_bytes(_ref(norm)))


def capscaps_group_norm_fwd(norm, args, workspace, workspace_bytes, stream=None) -> int:
    """`norm`, `args`: GroupNormArgs and GroupFwdArgs."""
    return _load().capscaps_group_norm_fwd(_ref(norm), _ref(args), workspace, workspace_bytes, stream)


def capscaps_group_norm_bwd_workspace_bytes(norm) -> int:
    return int(_load().capscaps_group_norm_bwd_workspace_bytes(_ref(norm)))


def capscaps_group_norm_bwd(norm, args, workspace, workspace_bytes, stream=None) -> int:
    """`norm`, `args`: GroupNormArgs and GroupBwdArgs."""
    return _load().capscaps_group_norm_bwd(_ref(norm), _ref(args), workspace, workspace_bytes, stream)


def capscaps_class_loss_workspace_bytes(head, backward) -> int:
    return int(_load().capscaps_class_loss_workspace_bytes(_ref(head), backward))


def capscaps_class_loss_fwd(head, args, workspace, workspace_bytes, stream=None) -> int:
    """`head`, `args`: HeadArgs and HeadFwdArgs."""
    return _load().capscaps_class_loss_fwd(_ref(head), _ref(args), workspace, workspace_bytes, stream)


def capscaps_class_loss_bwd(head, args, workspace, workspace_bytes, stream=None) -> int:
    """`head`, `args`: HeadArgs and HeadBwdArgs."""
    return _load().capscaps_class_loss_bwd(_ref(head), _ref(args), workspace, workspace_bytes, stream)


def capscaps_distill_loss_workspace_bytes(head, backward) -> int:
    return int(_load().capscaps_distill_loss_workspace_bytes(_ref(head), backward))


def capscaps_distill_loss_fwd(head, args, workspace, workspace_bytes, stream=None) -> int:
    """`head`, `args`: HeadArgs and HeadFwdArgs."""
    return _load().capscaps_distill_loss_fwd(_ref(head), _ref(args), workspace, workspace_bytes, stream)


def capscaps_distill_loss_bwd(head, args, workspace, workspace_bytes, stream=None) -> int:
    """`head`, `args`: HeadArgs and HeadBwdArgs."""
    return _load().capscaps_distill_loss_bwd(_ref(head), _ref(args), workspace, workspace_bytes, stream)


def capscaps_grad_norm(grads, count, grad_scale, max_norm, control, workspace, workspace_bytes, stream=None) -> int:
    """`grads`: an array of GradTensor."""
    return _load().capscaps_grad_norm(grads, count, grad_scale, max_norm, control, workspace, workspace_bytes, stream)


def capscaps_adamw_step(tensors, count, state_bits, lr, beta1, beta2, eps, step, seed, control, stream=None) -> int:
    """`tensors`: an array of AdamwTensor."""
    return _load().capscaps_adamw_step(tensors, count, state_bits, lr, beta1, beta2, eps, step, seed, control, stream)


def capscaps_adamw_state_values(tensors, count, m_out, v_out, stream=None) -> int:
    """`tensors`: an array of AdamwTensor; `m_out`, `v_out`: arrays of device pointers (c_void_p)."""
    return _load().capscaps_adamw_state_values(tensors, count, m_out, v_out, stream)


def _ref(structure):
    return None if structure is None else ctypes.addressof(structure)


def capscaps_mfma_yardstick(seed, sink, dtype, blocks, iters, stream=None) -> int:
    return _load().capscaps_mfma_yardstick(seed, sink, dtype, blocks, iters, stream)


def capscaps_mfma_yardstick_flops(dtype, blocks, iters) -> float:
    return float(_load().capscaps_mfma_yardstick_flops(dtype, blocks, iters))


# ------------------------------------------------------------------ torch convenience
def _torch_dtype_code(t):
    import torch
    return {torch.float32: FP32, torch.bfloat16: BF16, torch.float16: FP16}[t.dtype]


def conv_fwd(input, kernel, stride=1, pad=0, path=PATH_AUTO, out=None, workspace=None,
             out16=False):
    """input [N,H,W,C,D0,D1,D2], kernel [kh,kw,C,M,D0,D2,D3] (contiguous device tensors of one
    dtype: float32, bfloat16 or float16) -> float32 [N,H',W',M,D0,D1,D3] (with `out16`: of the
    operands' 16-bit type, library's own path choice).  Enqueues on torch's current stream; does
    not synchronise."""
    import torch
    if not (input.is_cuda and kernel.is_cuda):
        raise ValueError("capscaps runs on the GPU only: pass device tensors")
    if input.dtype != kernel.dtype or input.dim() != 7 or kernel.dim() != 7:
        raise ValueError("input and kernel must be 7-D tensors of one dtype")
    if not (input.is_contiguous() and kernel.is_contiguous()):
        raise ValueError("input and kernel must be contiguous")
    N, H, W, C, D0, D1, D2 = input.shape
    kh, kw, Ck, M, D0k, D2k, D3 = kernel.shape
    if (Ck, D0k, D2k) != (C, D0, D2):
        raise ValueError(f"kernel {tuple(kernel.shape)} does not match input {tuple(input.shape)}")
    dt = _torch_dtype_code(input)
    rc, Ho, Wo = capscaps_out_shape(H, W, kh, kw, stride, pad)
    if rc != OK:
        raise CapscapsError(rc)
    if out is None:
        out = torch.empty((N, Ho, Wo, M, D0, D1, D3),
                          dtype=input.dtype if out16 else torch.float32, device=input.device)
    need = (capscaps_conv_fwd_out16_workspace_bytes if out16 else
            capscaps_conv_fwd_workspace_bytes)(N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3, dt)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=input.device)
    stream = torch.cuda.current_stream(input.device).cuda_stream
    if out16:
        rc = capscaps_conv_fwd_out16(input.data_ptr(), kernel.data_ptr(), out.data_ptr(), N, H, W,
                                     C, M, kh, kw, stride, pad, D0, D1, D2, D3, dt,
                                     workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), stream)
    else:
        rc = capscaps_conv_fwd_path(input.data_ptr(), kernel.data_ptr(), out.data_ptr(), N, H, W,
                                    C, M, kh, kw, stride, pad, D0, D1, D2, D3, dt, path,
                                    workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), stream)
    if rc != OK:
        raise CapscapsError(rc)
    return out


def _bwd_common(a, b):
    if not (a.is_cuda and b.is_cuda):
        raise ValueError("capscaps runs on the GPU only: pass device tensors")
    if a.dtype != b.dtype or a.dim() != 7 or b.dim() != 7:
        raise ValueError("operands must be 7-D tensors of one dtype")
    if not (a.is_contiguous() and b.is_contiguous()):
        raise ValueError("operands must be contiguous")


def conv_bwd_input(dout, kernel, input_hw, stride=1, pad=0, out16=False):
    """dout [N,H',W',M,D0,D1,D3], kernel [kh,kw,C,M,D0,D2,D3] (one dtype), input_hw = (H, W) of
    the forward input -> float32 dinput [N,H,W,C,D0,D1,D2] (with `out16`: of the operands' 16-bit
    type)."""
    import torch
    _bwd_common(dout, kernel)
    N, Ho, Wo, M, D0, D1, D3 = dout.shape
    kh, kw, C, Mk, D0k, D2, D3k = kernel.shape
    H, W = input_hw
    rc, ho, wo = capscaps_out_shape(H, W, kh, kw, stride, pad)
    if rc != OK:
        raise CapscapsError(rc)
    if (Mk, D0k, D3k, ho, wo) != (M, D0, D3, Ho, Wo):
        raise ValueError("dout, kernel and input_hw do not describe one convolution")
    dt = _torch_dtype_code(dout)
    shape = (N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3, dt)
    need = (capscaps_conv_bwd_input_out16_workspace_bytes if out16 else
            capscaps_conv_bwd_input_workspace_bytes)(*shape)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dout.device)
    din = torch.empty((N, H, W, C, D0, D1, D2), dtype=dout.dtype if out16 else torch.float32,
                      device=dout.device)
    call = capscaps_conv_bwd_input_out16 if out16 else capscaps_conv_bwd_input
    rc = call(dout.data_ptr(), kernel.data_ptr(), din.data_ptr(), *shape, ws.data_ptr(), ws.numel(),
              torch.cuda.current_stream(dout.device).cuda_stream)
    if rc != OK:
        raise CapscapsError(rc)
    return din


def conv_bwd_kernel(input, dout, kernel_hw, stride=1, pad=0):
    """input [N,H,W,C,D0,D1,D2], dout [N,H',W',M,D0,D1,D3] (one dtype), kernel_hw = (kh, kw)
    -> float32 dkernel [kh,kw,C,M,D0,D2,D3]."""
    import torch
    _bwd_common(input, dout)
    N, H, W, C, D0, D1, D2 = input.shape
    Ng, Ho, Wo, M, D0g, D1g, D3 = dout.shape
    kh, kw = kernel_hw
    rc, ho, wo = capscaps_out_shape(H, W, kh, kw, stride, pad)
    if rc != OK:
        raise CapscapsError(rc)
    if (Ng, D0g, D1g, ho, wo) != (N, D0, D1, Ho, Wo):
        raise ValueError("input, dout and kernel_hw do not describe one convolution")
    dt = _torch_dtype_code(input)
    shape = (N, H, W, C, M, kh, kw, stride, pad, D0, D1, D2, D3, dt)
    need = capscaps_conv_bwd_kernel_workspace_bytes(*shape)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=input.device)
    dk = torch.empty((kh, kw, C, M, D0, D2, D3), dtype=torch.float32, device=input.device)
    rc = capscaps_conv_bwd_kernel(input.data_ptr(), dout.data_ptr(), dk.data_ptr(), *shape,
                                  ws.data_ptr(), ws.numel(),
                                  torch.cuda.current_stream(input.device).cuda_stream)
    if rc != OK:
        raise CapscapsError(rc)
    return dk


# ------------------------------------------------------------------ norms around a block
BlockNorm = namedtuple("BlockNorm", "y h rstd_pre rstd_post")
BlockNormGrads = namedtuple("BlockNormGrads", "dx dbranch dpre_weight dpost_weight dgate")
_ACTS = {"linear": ACT_LINEAR, "sigmoid": ACT_SIGMOID, "silu": ACT_SILU}
_codes = None
_raw_stream = None


def _stream(device):
    """Handle of torch's current stream on `device`, by the short way (1.8 us less than through a Stream object, of the 20
    that a call on small tensors takes) where this torch has it."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device.index)


def _current_gpu():
    """Index of torch's current GPU, the one that kernels go to, whatever the stream."""
    global _current_gpu
    import torch
    _current_gpu = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _current_gpu()


def _enqueue(call, device, *args):
    """A call of the library on torch's current stream of the tensors' GPU, made the current one where it is not."""
    if _current_gpu() != device.index:
        import torch
        with torch.cuda.device(device):
            return _enqueue(call, device, *args)
    rc = call(*args, _stream(device))
    if rc != OK:
        raise CapscapsError(rc)


def _overwritten(tensors):
    """Tells autograd that the caller's tensors have other values now, as torch's own in-place operations do."""
    global _overwritten
    import torch
    _overwritten = torch.autograd.graph.increment_version
    _overwritten(tensors)


def _code(dtype):
    """The library's code of a torch dtype."""
    global _codes
    if _codes is None:
        import torch
        _codes = {torch.float32: FP32, torch.bfloat16: BF16, torch.float16: FP16}
    try:
        return _codes[dtype]
    except KeyError:
        raise ValueError(f"{dtype}: float32, bfloat16 and float16 are supported") from None


def _gpu_of(t):
    if not t.is_cuda:
        raise ValueError("capscaps runs on the GPU only: pass device tensors")
    return t.get_device()


def _row_stride(t, shape, width, norm_dims, name, gpu):
    """Distance between the rows of `t`, whose last `norm_dims` axes are one dense row and whose other axes follow
    each other at equal distances; it has to be on that `gpu`."""
    if t.get_device() != gpu:
        raise ValueError(f"{name} is not on the GPU that the other tensors are on")
    if t.shape == shape and t.is_contiguous():
        return width
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    strides, dense = t.stride(), 1
    for k in range(len(shape) - 1, len(shape) - 1 - norm_dims, -1):
        if shape[k] != 1 and strides[k] != dense:
            raise ValueError(f"{name}: a row's values must lie next to each other")
        dense *= shape[k]
    row, expect = None, None
    for k in range(len(shape) - 1 - norm_dims, -1, -1):
        if shape[k] == 1:
            continue
        if row is None:
            row = expect = strides[k]
        if strides[k] != expect:
            raise ValueError(f"{name}: its rows must lie at equal distances")
        expect *= shape[k]
    return width if row is None else row


def _vector(t, width, device, name):
    if t is None:
        return None
    if t.numel() != width or _code(t.dtype) != FP32 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be {width} contiguous float32 values on {device}")
    return t.data_ptr()


def _block(x, branch, gate, gate_act, dtype, norm_dims, post_norm, residual_scale, branch_scale, eps):
    """(BlockArgs, pointers and strides of branch and gate): what both directions check."""
    shape = x.shape
    if not 1 <= norm_dims <= len(shape) or x.numel() == 0:
        raise ValueError(f"{norm_dims} axes of a tensor of shape {tuple(shape)} are no rows")
    width = math.prod(shape[len(shape) - norm_dims:])
    if width > MOST_ROW_VALUES:  # (a C int, to which ctypes would cut it without a word)
        raise ValueError(f"rows of {width} values: up to 2^30 are supported")
    layer, stream = _code(dtype), _code(x.dtype)
    kind, gate_ptr, gate_stride = GATE_NONE, None, 0
    if gate is not None:
        # (for one row the type says which it is: a vector is float32, a gate for every value `dtype`)
        if gate.shape == shape and (x.numel() > width or
                                    gate.dtype == dtype and (layer != FP32 or gate.dim() > norm_dims)):
            if gate.dtype != dtype:
                raise ValueError(f"a gate for every value must be {dtype}")
            kind, gate_stride = GATE_FULL, _row_stride(gate, shape, width, norm_dims, "gate", _gpu_of(x))
            gate_ptr = gate.data_ptr()
        else:
            kind, gate_ptr = GATE_SHARED, _vector(gate, width, x.device, "gate")
    if gate_act not in _ACTS:
        raise ValueError(f"gate_act is one of {', '.join(_ACTS)}")
    branch_ptr, branch_stride, branch_code = None, 0, FP32
    if branch is not None:
        branch_stride = _row_stride(branch, shape, width, norm_dims, "branch", _gpu_of(x))
        branch_ptr, branch_code = branch.data_ptr(), _code(branch.dtype)
    elif gate is not None:
        raise ValueError("a gate needs a branch")
    if stream not in (FP32, layer) or branch_code not in (FP32, layer):
        raise ValueError(f"x and branch must be float32 or {dtype}")
    block = BlockArgs(x.numel() // width, width, layer, stream, branch_code, 1 if post_norm else 0, kind,
                      _ACTS[gate_act], residual_scale, branch_scale, eps)
    return block, branch_ptr, branch_stride, gate_ptr, gate_stride


def block_norm_fwd(x, branch=None, *, pre_weight=None, post_weight=None, gate=None, gate_act="linear",
                   post_norm=True, residual_scale=1.0, branch_scale=1.0, eps=1e-6, norm_dims=1, dtype=None,
                   save=False, want_y=True, want_h=True, y=None, h=None):
    """Between two blocks of layers, in one launch: the norm after the block, its gate, the residual sum, the norm
    before the next block.

        u = branch / rms(branch) * post_weight            (post_norm=False: u = branch)
        y = residual_scale * x + branch_scale * act(gate) * u
        h = y / rms(y) * pre_weight

    The last `norm_dims` axes of x [N, ...] are a row: of an activation [N,H,W,C,D0,D1,D2], 4 normalises all
    capsules of a pixel together, 3 every capsule by itself.  `dtype` is the layers' element type (that of h; default: x's): x, the
    residual stream, and branch, a layer's output, are each float32 or `dtype`.  Weights are float32 of a row's
    size; the gate is such a vector, or a tensor of x's shape and `dtype` (of one row, the type says which).  Without a branch only h is computed.
    Returns BlockNorm(y, h, rstd_pre, rstd_post); the statistics only with `save`, for block_norm_bwd.  `y` and `h`
    may be given to write to; y may be x.  The results have no autograd history: gradients are block_norm_bwd's.  Enqueues on torch's current stream; does not synchronise (tensors made on another
    stream have to be ready and, if they are freed early, recorded there, as for torch's own operations)."""
    import torch
    dtype = x.dtype if dtype is None else dtype
    block, bp, bs, gp, gs = _block(x, branch, gate, gate_act, dtype, norm_dims, post_norm, residual_scale,
                                   branch_scale, eps)
    shape, width, device, gpu = x.shape, block.width, x.device, _gpu_of(x)
    xs = _row_stride(x, shape, width, norm_dims, "x", gpu)
    if branch is None and y is not None:
        raise ValueError("without a branch there is no y")
    if y is not None and y.dtype != x.dtype or h is not None and h.dtype != dtype:
        raise ValueError("y has x's type, h has `dtype`")
    given = [t for t in (y, h) if t is not None]
    ys = width if y is None else _row_stride(y, shape, width, norm_dims, "y", gpu)
    hs = width if h is None else _row_stride(h, shape, width, norm_dims, "h", gpu)
    if y is None and want_y and branch is not None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    if h is None and want_h:
        h = torch.empty(shape, dtype=dtype, device=device)
    rpre = rpost = None
    if save:
        if h is not None:
            rpre = torch.empty(shape[:len(shape) - norm_dims], dtype=torch.float32, device=device)
        if branch is not None and post_norm:
            rpost = torch.empty(shape[:len(shape) - norm_dims], dtype=torch.float32, device=device)
    args = BlockFwdArgs(
        x.data_ptr(), bp, gp, _vector(pre_weight, width, device, "pre_weight"),
        _vector(post_weight, width, device, "post_weight"), None if y is None else y.data_ptr(),
        None if h is None else h.data_ptr(), None if rpre is None else rpre.data_ptr(),
        None if rpost is None else rpost.data_ptr(), xs, bs, gs, ys, hs)
    _enqueue(capscaps_block_norm_fwd, device, block, args)
    if given:
        _overwritten(given)
    return BlockNorm(y, h, rpre, rpost)


def block_norm_bwd(y, branch, rstd_pre, rstd_post, dh, dy, *, pre_weight=None, post_weight=None, gate=None,
                   gate_act="linear", post_norm=True, residual_scale=1.0, branch_scale=1.0, norm_dims=1, dtype=None):
    """The gradients of block_norm_fwd, from what it returned with `save` and the gradients of h and y (`dh` of the
    layers' type `dtype`, `dy` of the stream's; either may be None = zero).  `y` is the stream after the
    block (without a branch: x).  Returns BlockNormGrads(dx, dbranch, dpre_weight, dpost_weight, dgate): dx in
    the stream's type, dbranch and the gradient of a gate for every value in `dtype`, the other gates' and the weights' float32 sums over
    rows; None where there is no such operand."""
    import torch
    if dh is None and dy is None:
        raise ValueError("block_norm_bwd needs dh or dy")
    if dtype is None:
        dtype = y.dtype if dh is None else dh.dtype
    block, bp, bs, gp, gs = _block(y, branch, gate, gate_act, dtype, norm_dims, post_norm, residual_scale,
                                   branch_scale, 1.0)
    shape, width, device, gpu = y.shape, block.width, y.device, _gpu_of(y)
    if dh is not None and dh.dtype != dtype or dy is not None and dy.dtype != y.dtype:
        raise ValueError("dh has `dtype`, dy has y's type")
    post = branch is not None and post_norm

    def vector():
        return torch.empty(width, dtype=torch.float32, device=device)

    dx = torch.empty(shape, dtype=y.dtype, device=device)
    db = torch.empty(shape, dtype=dtype, device=device) if branch is not None else None
    dpre = vector() if dh is not None and pre_weight is not None else None
    dpost = vector() if post and post_weight is not None else None
    dgate = None
    if gate is not None:
        dgate = vector().view(gate.shape) if block.gate == GATE_SHARED else torch.empty(shape, dtype=dtype, device=device)
    need = capscaps_block_norm_bwd_workspace_bytes(block)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    args = BlockBwdArgs(
        y.data_ptr(), bp, gp, _vector(pre_weight, width, device, "pre_weight"),
        _vector(post_weight, width, device, "post_weight"),
        _vector(rstd_pre, block.rows, device, "rstd_pre") if dh is not None else None,
        _vector(rstd_post, block.rows, device, "rstd_post") if post else None,
        None if dh is None else dh.data_ptr(), None if dy is None else dy.data_ptr(), dx.data_ptr(),
        None if db is None else db.data_ptr(), None if dgate is None else dgate.data_ptr(),
        None if dpre is None else dpre.data_ptr(), None if dpost is None else dpost.data_ptr(),
        _row_stride(y, shape, width, norm_dims, "y", gpu), bs, gs,
        0 if dh is None else _row_stride(dh, shape, width, norm_dims, "dh", gpu),
        0 if dy is None else _row_stride(dy, shape, width, norm_dims, "dy", gpu), width, width, width)
    _enqueue(capscaps_block_norm_bwd, device, block, args, ws.data_ptr(), need)
    return BlockNormGrads(dx, db, dpre, dpost, dgate)


# ------------------------------------------------------------------ group norm
GroupNorm = namedtuple("GroupNorm", "y mean rstd")
GroupNormGrads = namedtuple("GroupNormGrads", "dx dweight dbias")


def _group(x, groups, act, dtype, eps, channel_dims):
    """(GroupNormArgs, width): what both directions check."""
    shape = x.shape
    if not 1 <= channel_dims < len(shape) or x.numel() == 0:
        raise ValueError(f"a tensor of shape {tuple(shape)} has no images and {channel_dims} axes of channels")
    width = math.prod(shape[len(shape) - channel_dims:])
    if width > MOST_ROW_VALUES:
        raise ValueError(f"{width} values of a position: up to 2^30 are supported")
    if not 1 <= groups <= width or width % groups:
        raise ValueError(f"{width} values of a position are not {groups} groups")
    if act not in _ACTS:
        raise ValueError(f"act is one of {', '.join(_ACTS)}")
    layer, code = _code(dtype), _code(x.dtype)
    if code not in (FP32, layer):
        raise ValueError(f"x must be float32 or {dtype}")
    images = shape[0]
    return GroupNormArgs(images, x.numel() // (width * images), width, groups, code, layer, _ACTS[act], eps), width


def group_norm_fwd(x, groups, *, weight=None, bias=None, act="linear", eps=1e-5, channel_dims=1, dtype=None, save=False,
                   y=None):
    """Group norm and activation, channels last:

        y = act((x - mean) / sqrt(var + eps) * weight + bias)

    x is [N, ..., channels]: its last `channel_dims` axes are the values of a position (of an activation
    [N,H,W,C,D0,D1,D2], 4), cut into `groups` groups of neighbours, and mean and variance are those of a group over all
    positions of an image.  `dtype` is the layers' element type (that of y; default: x's); x is float32 or `dtype`.  Weight
    and bias are float32, of a position's size.  Returns GroupNorm(y, mean, rstd); the statistics [N, groups] only with
    `save`, for group_norm_bwd.  `y` may be given to write to, and may be x.  The results have no autograd history.  Enqueues on torch's
    current stream; does not synchronise."""
    import torch
    dtype = x.dtype if dtype is None else dtype
    norm, width = _group(x, groups, act, dtype, eps, channel_dims)
    shape, device, gpu, given = x.shape, x.device, _gpu_of(x), y is not None
    xs = _row_stride(x, shape, width, channel_dims, "x", gpu)
    if given:
        if y.dtype != dtype:
            raise ValueError("y has `dtype`")
        ys = _row_stride(y, shape, width, channel_dims, "y", gpu)
    else:
        y, ys = torch.empty(shape, dtype=dtype, device=device), width
    mean = rstd = None
    if save:
        mean = torch.empty((shape[0], groups), dtype=torch.float32, device=device)
        rstd = torch.empty((shape[0], groups), dtype=torch.float32, device=device)
    need = capscaps_group_norm_fwd_workspace_bytes(norm)
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    args = GroupFwdArgs(x.data_ptr(), _vector(weight, width, device, "weight"), _vector(bias, width, device, "bias"),
                        y.data_ptr(), None if mean is None else mean.data_ptr(),
                        None if rstd is None else rstd.data_ptr(), xs, ys)
    _enqueue(capscaps_group_norm_fwd, device, norm, args, ws.data_ptr() if need else None, need)
    if given:
        _overwritten([y])
    return GroupNorm(y, mean, rstd)


def group_norm_bwd(x, groups, mean, rstd, dy, *, weight=None, bias=None, act="linear", channel_dims=1):
    """The gradients of group_norm_fwd, from its input, the statistics that it returned with `save` and the gradient of y.
    dy has the layers' type, and so has dx; x is float32 or of that type.  Returns GroupNormGrads(dx, dweight, dbias), the latter
    two float32 of a position's size, None without a weight or bias."""
    import torch
    norm, width = _group(x, groups, act, dy.dtype, 1.0, channel_dims)
    shape, device, gpu = x.shape, x.device, _gpu_of(x)
    dx = torch.empty(shape, dtype=dy.dtype, device=device)
    dweight, dbias = (None if t is None else torch.empty(t.shape, dtype=torch.float32, device=device)
                      for t in (weight, bias))
    need = capscaps_group_norm_bwd_workspace_bytes(norm)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    many = shape[0] * groups
    args = GroupBwdArgs(
        x.data_ptr(), _vector(weight, width, device, "weight"), _vector(bias, width, device, "bias"),
        _vector(mean, many, device, "mean"), _vector(rstd, many, device, "rstd"), dy.data_ptr(), dx.data_ptr(),
        None if dweight is None else dweight.data_ptr(), None if dbias is None else dbias.data_ptr(),
        _row_stride(x, shape, width, channel_dims, "x", gpu), _row_stride(dy, shape, width, channel_dims, "dy", gpu), width)
    if args.mean is None or args.rstd is None:
        raise ValueError("group_norm_bwd needs the mean and rstd that group_norm_fwd returned with `save`")
    _enqueue(capscaps_group_norm_bwd, device, norm, args, ws.data_ptr(), need)
    return GroupNormGrads(dx, dweight, dbias)


# ------------------------------------------------------------------ losses of a head over many classes
ClassLoss = namedtuple("ClassLoss", "loss lse")
DistillLoss = namedtuple("DistillLoss", "loss lse logq")
HeadGrads = namedtuple("HeadGrads", "dx dweight dbias")
MOST_ROWS, MOST_WIDTH, MOST_CLASSES, MOST_TOP = 1 << 20, 1 << 20, 1 << 26, 1024


def _head(x, weight, bias, index, teacher, temperature, gradient_terms=0):
    """(HeadArgs, what the tensors are as HeadFwdArgs and HeadBwdArgs have them): what both losses and directions check."""
    import torch
    gpu, device = _gpu_of(x), x.device
    if x.dim() < 1 or weight.dim() != 2 or weight.shape[1] != x.shape[-1] or not weight.numel():
        raise ValueError(f"x [..., width] and weight [classes, width]: not {tuple(x.shape)} and {tuple(weight.shape)}")
    if weight.dtype != x.dtype:
        raise ValueError("x and weight have one dtype")
    shape, (classes, width) = x.shape[:-1], weight.shape
    rows = math.prod(shape)
    if rows > MOST_ROWS or width > MOST_WIDTH or classes > MOST_CLASSES:  # (C ints, to which ctypes would cut them)
        raise ValueError(f"{rows} rows of {width} values, {classes} classes: up to 2^20, 2^20 and 2^26 are supported")
    if index.dtype not in (torch.int64, torch.int32):
        raise ValueError("indices of classes are int64 or int32")
    top, teacher_dtype, teacher_ptr, ts = 1, FP32, None, 0
    if teacher is None:
        ins = _row_stride(index, shape, 1, 0, "targets", gpu)
    else:
        if teacher.dim() != len(shape) + 1 or not 1 <= teacher.shape[-1] <= MOST_TOP:
            raise ValueError(f"the teacher has 1 to {MOST_TOP} logits for each of {tuple(shape)} rows")
        top, teacher_dtype, teacher_ptr = teacher.shape[-1], _code(teacher.dtype), teacher.data_ptr()
        ins = _row_stride(index, (*shape, top), top, 1, "teacher_index", gpu)
        ts = _row_stride(teacher, (*shape, top), top, 1, "teacher_logits", gpu)
    if not 1e-6 <= temperature <= 1e6:
        raise ValueError("temperature is 1e-6 to 1e6")
    if gradient_terms not in (0, 1, 2):
        raise ValueError("gradient_terms is 1 or 2, or 0 for the rule")
    head = HeadArgs(rows, width, classes, _code(x.dtype), 64 if index.dtype == torch.int64 else 32, top, teacher_dtype,
                    temperature, gradient_terms)
    return head, (x.data_ptr(), weight.data_ptr(), _vector(bias, classes, device, "bias"), index.data_ptr(), teacher_ptr,
                  _row_stride(x, x.shape, width, 1, "x", gpu), _row_stride(weight, weight.shape, width, 1, "weight", gpu),
                  ins, ts)


def _head_fwd(call, need, x, head, tensors, logq_shape=None):
    import torch
    device, shape = x.device, x.shape[:-1]
    loss, lse = (torch.empty(shape, dtype=torch.float32, device=device) for _ in range(2))
    logq = None if logq_shape is None else torch.empty(logq_shape, dtype=torch.float32, device=device)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    args = HeadFwdArgs(*tensors, loss.data_ptr(), lse.data_ptr(), None if logq is None else logq.data_ptr())
    _enqueue(call, device, head, args, ws.data_ptr(), need)
    return loss, lse, logq


def _head_bwd(call, need, x, weight, bias, head, tensors, loss, lse, logq, dloss, want_dx, want_dweight):
    import torch
    device, rows = x.device, head.rows
    if not (want_dx or want_dweight or bias is not None):
        raise ValueError("no gradient is wanted")
    if dloss.dtype != torch.float32 or dloss.device != device or dloss.numel() not in (1, rows):
        raise ValueError(f"dloss is a float32 for each of {rows} rows, or one for all, on {device}")
    if dloss.numel() == 1 or all(s == 0 for s in dloss.stride()):
        step = 0
    elif dloss.is_contiguous():
        step = 1
    else:
        raise ValueError("dloss must be contiguous, or one value for all rows")
    dx = torch.empty(x.shape, dtype=x.dtype, device=device) if want_dx else None
    dweight = torch.empty(weight.shape, dtype=weight.dtype, device=device) if want_dweight else None
    dbias = None if bias is None else torch.empty(bias.shape, dtype=torch.float32, device=device)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    args = HeadBwdArgs(*tensors, _vector(loss, rows, device, "loss"), _vector(lse, rows, device, "lse"),
                       _vector(logq, rows * head.top, device, "logq"), dloss.data_ptr(),
                       *(None if t is None else t.data_ptr() for t in (dx, dweight, dbias)), step)
    _enqueue(call, device, head, args, ws.data_ptr(), need)
    return HeadGrads(dx, dweight, dbias)


def class_loss_fwd(x, weight, targets, *, bias=None):
    """Softmax cross entropy of a linear head over many classes, the logits z = x weight^T + bias computed piece by piece
    and never kept:

        loss = lse - z[target]          lse = log(sum(exp(z)))

    x [..., width] and weight [classes, width] of one dtype, targets [...] int64 or int32, bias [classes] float32 (-inf
    rules a class out).  A row whose target is no class (any negative one) is left out: its loss is 0.  Returns
    ClassLoss(loss, lse), float32 [...].  The results have no autograd history: gradients are class_loss_bwd's.  Enqueues on torch's current
    stream; does not synchronise."""
    head, tensors = _head(x, weight, bias, targets, None, 1.0)
    loss, lse, _ = _head_fwd(capscaps_class_loss_fwd, capscaps_class_loss_workspace_bytes(head, 0), x, head, tensors)
    return ClassLoss(loss, lse)


def class_loss_bwd(x, weight, targets, loss, lse, dloss, *, bias=None, want_dx=True, want_dweight=True, gradient_terms=0):
    """The gradients of class_loss_fwd, from its arguments, what it returned and the gradient of the loss: float32, one for each row
    or one for all (a mean's: 1 / rows that have a target).  Returns HeadGrads(dx, dweight, dbias): dx and dweight in x's dtype
    (None where not wanted), dbias float32, None without a bias.

    In 16 bits the gradient of z, which the products for dx and dweight read, is rounded to x's dtype once (`gradient_terms` 1: about as
    large an error again as that of storing dx and dweight), or held in two terms of it (2: no more than that one rounding, for
    products of twice the length).  0 takes 2 where rows or classes are 256 or fewer, else 1."""
    head, tensors = _head(x, weight, bias, targets, None, 1.0, gradient_terms)
    return _head_bwd(capscaps_class_loss_bwd, capscaps_class_loss_workspace_bytes(head, 1), x, weight, bias, head, tensors,
                     loss, lse, None, dloss, want_dx, want_dweight)


def distill_loss_fwd(x, weight, teacher_index, teacher_logits, *, bias=None, temperature=1.0):
    """Distillation from a teacher's top logits through a linear head, z = x weight^T + bias as in class_loss_fwd:

        loss = temperature^2 * sum_k t_k (log t_k - logq_k)
        t = softmax(teacher_logits / temperature)      logq_k = z[teacher_index_k] / temperature - lse

    teacher_index [..., top] (int64 or int32) and teacher_logits [..., top] (float32, bfloat16 or float16) are a row's entries;
    those whose index is no class (any negative one) do not count, and a row without entries is left out.  Returns
    DistillLoss(loss, lse, logq), float32 [...] and [..., top]; lse is that of z / temperature."""
    head, tensors = _head(x, weight, bias, teacher_index, teacher_logits, temperature)
    return DistillLoss(*_head_fwd(capscaps_distill_loss_fwd, capscaps_distill_loss_workspace_bytes(head, 0), x, head, tensors,
                                  teacher_index.shape))


def distill_loss_bwd(x, weight, teacher_index, teacher_logits, lse, logq, dloss, *, bias=None, temperature=1.0, want_dx=True,
                     want_dweight=True, gradient_terms=0):
    """The gradients of distill_loss_fwd, as class_loss_bwd's, from the lse and logq that it returned."""
    head, tensors = _head(x, weight, bias, teacher_index, teacher_logits, temperature, gradient_terms)
    return _head_bwd(capscaps_distill_loss_bwd, capscaps_distill_loss_workspace_bytes(head, 1), x, weight, bias, head, tensors,
                     None, lse, logq, dloss, want_dx, want_dweight)


# ------------------------------------------------------------------ gradient norm, AdamW
def _dense(t, what, gpu):
    """Address of a contiguous tensor on that GPU."""
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{what} must be contiguous device tensors")
    if t.get_device() != gpu:
        raise ValueError(f"{what} must be on one GPU")
    return t.data_ptr()


def _grad_codes(grads, gpu):
    """Type codes of gradients that the library can read where they are.  (No call for each: lists are long, steps short.)"""
    if not all([g.get_device() == gpu and g.is_contiguous() for g in grads]) or (grads and not grads[0].is_cuda):
        raise ValueError("gradients must be contiguous device tensors, on the GPU of the other tensors")
    try:
        return [_codes[g.dtype] for g in grads]
    except (KeyError, TypeError):  # a type of no code, or the first call: no codes yet
        return [_code(g.dtype) for g in grads]


def _control_ptr(control, gpu):
    if control.nbytes != 16:
        raise ValueError("control is 16 bytes: norm, scale (float32), skip, step (int32)")
    return _dense(control, "control and gradients", gpu)


def grad_norm(grads, max_norm=None, grad_scale=1.0, control=None, workspace=None):
    """The 2-norm of all gradients together, on the device: writes `control`, four values of 4 bytes that AdamW.step
    reads: the norm (of grad_scale * gradients), the factor that scales and clips the gradients to `max_norm`
    (None, or 0 and below: no clipping), whether the step is to be skipped because the norm is not finite (int32), and the number of steps
    not skipped so far (int32, counted up here).  Returns it.  `control`: an optimizer's `control`, or a tensor of zeros
    that is kept for the whole training.  Without one a new tensor is returned, for this step alone: it counts nothing
    but this step, and AdamW.step counts the steps itself then."""
    import torch
    if not grads and control is None:
        raise ValueError("grad_norm of no tensors needs a control to write to")
    first = control if control is not None else grads[0]
    device, gpu = first.device, first.get_device()
    codes = _grad_codes(grads, gpu)
    if control is None:
        control = torch.zeros(4, dtype=torch.float32, device=device)
        control.capscaps_for_one_step = True
    if workspace is None:
        workspace = torch.empty(GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=device)
    elif workspace.get_device() != gpu or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the gradients' GPU")
    items = (GradTensor * max(1, len(grads)))(
        *[(g.data_ptr(), g.numel(), code) for g, code in zip(grads, codes)])
    _enqueue(capscaps_grad_norm, device, items, len(grads), grad_scale, 0.0 if max_norm is None else max_norm,
             _control_ptr(control, gpu), workspace.data_ptr(), workspace.numel())
    return control


class AdamW:
    """AdamW over a list of float32 device tensors, all in one launch (44 tensors a launch).

    `weight_decay`: a number, or one for each tensor.  `copies`: None, a 16-bit dtype (copies of that type are made), or
    a list of 16-bit tensors (None where there is none) of the parameters' sizes; each step writes the rounded
    parameters there, for the layers to read.  `state_bits`: 32 (float32 moments) or 8 (a byte for each, and a
    byte for each 256 values that share an exponent; rounded at random by a hash of `seed`, the step and the
    position).  `state`: moments to go on from, (m, v) or (m, v, m_exp, v_exp), lists of tensors in that format (those
    of another AdamW, saved); kept, not copied; `steps`: the steps they have seen (`steps` of that AdamW).

    Steps are counted on the host, or, so that one that is not finite can be skipped without waiting for the GPU, on the
    device.  For the latter give `step` what grad_norm returned: grad_norm(grads, max_norm, control=opt.control) counts in
    `control`, the optimizer's own, which begins at `steps`; grad_norm(grads, max_norm) leaves the counting to `step`. A
    control of the caller's own counts by itself, from zero, and is refused by an optimizer that has counted steps
    otherwise.  `steps` is the number of steps taken either way (on the device, reading it waits for the GPU).

    Tensors of `params`, `m`, `v`, `m_exp`, `v_exp` and `copies` may get other storage, or be replaced in the lists, between
    steps (a captured step keeps the ones it was captured with)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, state_bits=32, copies=None,
                 seed=0, state=None, steps=0):
        import torch
        if state_bits not in (32, 8):
            raise ValueError("state_bits is 32 or 8")
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamW needs parameters")
        count, eight = len(self.params), state_bits == 8
        self.lr, self.betas, self.eps, self.state_bits, self.seed = lr, betas, eps, state_bits, seed
        # steps counted on the host; the control that counts them on the device, if one does; the optimizer's own control, and
        # the steps that it has not counted
        self._control = torch.zeros(4, dtype=torch.float32, device=self.params[0].device)
        self._host, self._counter, self._lacking, self._int32 = steps, None, 0, torch.int32
        if steps:
            self.steps = steps
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
        if isinstance(copies, torch.dtype):
            copies = [p.detach().to(copies) for p in self.params]
        self.copies = [None] * count if copies is None else list(copies)
        if state is None:
            kind = torch.uint8 if eight else torch.float32
            self.m, self.v = ([torch.zeros(p.shape, dtype=kind, device=p.device) for p in self.params]
                              for _ in range(2))
            self.m_exp, self.v_exp = ([torch.zeros((p.numel() + 255) // 256, dtype=torch.uint8, device=p.device)
                                       for p in self.params] if eight else [None] * count for _ in range(2))
        else:
            if len(state) != (4 if eight else 2):
                raise ValueError("state is (m, v), or (m, v, m_exp, v_exp) in 8 bits")
            self.m, self.v, self.m_exp, self.v_exp = [list(s) for s in state] + (
                [] if eight else [[None] * count, [None] * count])
        # (methods of the class, to map over lists: these are long, steps short)
        self._decay, self._address, self._contiguous = decay, torch.Tensor.data_ptr, torch.Tensor.is_contiguous
        self._fill()

    def _fill(self):
        """Checks the tensors and writes the library's table of them."""
        import torch
        count, eight = len(self.params), self.state_bits == 8
        if any(len(s) != count for s in (self._decay, self.copies, self.m, self.v, self.m_exp, self.v_exp)):
            raise ValueError(f"{count} parameters need as many copies, moments and decays")
        self._held = None  # (nothing to step with if a check below fails)
        self._device, self._gpu = self.params[0].device, self.params[0].get_device()
        gpu = self._gpu
        self._items = (AdamwTensor * count)()
        self._sizes = [p.numel() for p in self.params]
        for t, p, m, v, me, ve, c, d in zip(self._items, self.params, self.m, self.v, self.m_exp, self.v_exp,
                                            self.copies, self._decay):
            kind, n = (torch.uint8 if eight else torch.float32), p.numel()
            if p.dtype != torch.float32:
                raise ValueError("parameters are float32")
            if m.dtype != kind or v.dtype != kind or m.numel() != n or v.numel() != n:
                raise ValueError(f"moments are {kind} of the parameters' sizes")
            if eight and any(e.dtype != torch.uint8 or e.numel() != (n + 255) // 256 for e in (me, ve)):
                raise ValueError("exponents are bytes, one for each 256 values")
            if c is not None and (c.numel() != n or _code(c.dtype) == FP32):
                raise ValueError("copies are 16-bit tensors of the parameters' sizes")
            t.param, t.n, t.weight_decay = _dense(p, "parameters", gpu), n, d
            t.m, t.v = _dense(m, "parameters and moments", gpu), _dense(v, "parameters and moments", gpu)
            t.m_exp, t.v_exp = [_dense(e, "parameters and exponents", gpu) for e in (me, ve)] if eight else (None, None)
            t.copy, t.copy_dtype = (None, BF16) if c is None else (_dense(c, "parameters and copies", gpu), _code(c.dtype))
        if self._control.get_device() != gpu:  # the parameters moved
            own = self._counter is self._control
            self._control = self._control.to(self.params[0].device)
            self._counter = self._control if own else self._counter
        self._written = self.params + [c for c in self.copies if c is not None]
        self._held = self._addresses()

    def _addresses(self):
        """Where the tensors lie now: storage may be replaced (`p.data = ...`), and so may entries of the lists."""
        held = [*self.params, *self.m, *self.v]
        if self.state_bits == 8:
            held += [*self.m_exp, *self.v_exp]
        return [*map(self._address, held)] + [0 if c is None else c.data_ptr() for c in self.copies]

    def _refresh(self):
        """Before each call: the table is of the tensors as they are."""
        if self._held != self._addresses() or not all(map(self._contiguous, self.params)):
            self._fill()

    def step(self, grads, control=None, lr=None):
        """One step with these gradients (float32, bfloat16 or float16, contiguous).  With `control`, what
        grad_norm returned: their scale, the number of the step and whether it is skipped come from there;
        without, steps are counted here.  Enqueues on torch's current stream."""
        self._refresh()
        if _current_gpu() != self._device.index:
            import torch
            with torch.cuda.device(self._device):
                return self.step(grads, control, lr)
        if len(grads) != len(self._items):
            raise ValueError(f"{len(self._items)} parameters need as many gradients")
        if [g.numel() for g in grads] != self._sizes:
            raise ValueError("gradients have the parameters' sizes")
        for t, at, code in zip(self._items, map(self._address, grads), _grad_codes(grads, self._gpu)):
            t.grad, t.grad_dtype = at, code
        step = self.steps + 1 if control is None else 0
        counter = None if control is None else _control_ptr(self._counting(control), self._gpu)
        rc = capscaps_adamw_step(self._items, len(self._items), self.state_bits, self.lr if lr is None else lr,
                                 self.betas[0], self.betas[1], self.eps, step, self.seed & 0xFFFFFFFF, counter,
                                 _stream(self._device))
        if rc != OK:
            raise CapscapsError(rc)
        _overwritten(self._written)
        if control is None:  # what the optimizer's control has not counted
            if self._counter is not None:
                self._lacking = 0 if self._counter is self._control else step - 1
            self._lacking += 1
            self._host, self._counter = step, None

    def _counting(self, control):
        """The control that counts this step, for the one that `step` was given."""
        if control is self._counter:
            return control
        own, single = self._control, getattr(control, "capscaps_for_one_step", False)
        _control_ptr(control, self._gpu)
        if not single and control.data_ptr() != own.data_ptr():
            if self._host or self._counter is own:
                raise ValueError("this optimizer has counted steps without this control: give grad_norm the "
                                 "optimizer's `control`, or none")
            self._counter = control
            return control
        if self._counter is not None and self._counter is not own:  # the caller's has counted until now
            self._lacking = self.steps
        self._own_control()
        if single:
            own[:3].copy_(control[:3])
            own.view(self._int32)[3:].add_(control.view(self._int32)[2:3] == 0)
        self._counter = own
        return own

    def _own_control(self):
        """The optimizer's control, with the steps that were counted elsewhere."""
        import torch
        if self._lacking:
            if torch.cuda.is_current_stream_capturing():  # (each replay would count them again)
                raise RuntimeError("steps were counted on the host: read the optimizer's `control` once before the capture")
            self._control.view(self._int32)[3:].add_(self._lacking)
            self._lacking = 0
        return self._control

    @property
    def control(self):
        """The optimizer's own control, for grad_norm to write: it counts the steps on the device."""
        return self._own_control()

    @property
    def steps(self):
        """Steps taken.  Where the device counts them, this waits for it."""
        if self._counter is None:
            return self._host
        return self._counter.cpu().flatten().view(self._int32)[3].item()

    @steps.setter
    def steps(self, steps):
        self._host, self._counter, self._lacking = steps, None, 0
        self._control.view(self._int32)[3:].fill_(steps)

    def state_values(self, out=None):
        """The moments (m, v) as lists of tensors; in 8 bits, the values their codes stand for, in bfloat16, which
        holds them exactly (written to `out`, two lists of tensors, if given)."""
        import torch
        if self.state_bits == 32:
            return self.m, self.v
        self._refresh()
        if out is None:
            out = [[torch.empty(p.shape, dtype=torch.bfloat16, device=p.device) for p in self.params]
                   for _ in range(2)]
        for t, n in zip(out[0] + out[1], self._sizes + self._sizes):
            if t.dtype != torch.bfloat16 or t.numel() != n:
                raise ValueError("moments' values are bfloat16 of the parameters' sizes")
        count = len(self._items)
        pointers = [(ctypes.c_void_p * count)(*[_dense(t, "parameters and values", self._gpu) for t in o]) for o in out]
        _enqueue(capscaps_adamw_state_values, self._device, self._items, count, *pointers)
        return out[0], out[1]

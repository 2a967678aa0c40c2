"""ctypes binding of libslim.so: one Python method per C entry point, same names, argument
marshalling only.  PyTorch supplies device memory and the HIP stream; every step of the pass runs
in the library's kernels.  There is no fallback: if the library is missing, `load()` raises."""
from __future__ import annotations

import array
import ctypes
import os
import struct
from typing import NamedTuple, Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslim.so")

SLIM_OK = 0
ERR_INVALID_ARG, ERR_NOT_PD, ERR_ALLOC, ERR_HIP, ERR_UNSUPPORTED = -1, -2, -3, -4, -5
F16, BF16, F32, F64 = 0, 1, 2, 3
WEIGHT_MASK_MEAN, WEIGHT_UNIFORM, WEIGHT_ELEMENT = 0, 1, 2
Q1_SIGN, Q1_AFFINE = 0, 1
SCOPE_BLOCK, SCOPE_ROW = 0, 1
SAL_HINV_DIAG, SAL_CHOL_DIAG = 0, 1
OBJ_KL, OBJ_MSE = 0, 1
ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

_DT = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32, torch.float64: F64}

# every symbol include/slim.h declares
EXPORTS = [
    "slim_default_params", "slim_default_tau", "slim_create", "slim_destroy", "slim_last_error",
    "slim_workspace_bytes", "slim_workspace_query", "slim_hessian_accumulate", "slim_hessian_inverse", "slim_salience",
    "slim_sba_allocate", "slim_sba_prepare", "slim_sqc_calibrate", "slim_gptq_quantize", "slim_pack", "slim_dequant_matmul",
    "slim_dequant_matmul_noalloc", "slim_dequant_matmul_zp", "slim_dequant_matmul_handover",
    "slim_transpose_16", "slim_pack_zeros", "slim_unpack_zeros", "slim_lwc_quantize",
    "slim_fp8_quantize_weights", "slim_fp8_linear_workspace", "slim_fp8_linear", "slim_fp8_linear_backward_workspace",
    "slim_fp8_linear_backward", "slim_layer_norm", "slim_layer_norm_backward_workspace", "slim_layer_norm_backward",
    "slim_distill_workspace", "slim_distill_loss", "slim_distill_loss_grad",
    "slim_fp8_linear_act_workspace", "slim_fp8_linear_act", "slim_fp8_linear_act_backward_workspace", "slim_fp8_linear_act_backward",
    "slim_head_loss_workspace", "slim_head_loss", "slim_head_loss_grad_workspace", "slim_head_loss_grad",
    "slim_add_norm", "slim_add_norm_backward", "slim_grad_norm_workspace", "slim_grad_norm", "slim_clip_gradients",
    "slim_profile_enable", "slim_profile_collect", "slim_profile_entry", "slim_profile_reset",
]


class SlimParams(ctypes.Structure):
    _fields_ = [("sqc_weight_mode", ctypes.c_int), ("mask_scope", ctypes.c_int),
                ("q1_mode", ctypes.c_int), ("sal_mode", ctypes.c_int)]


class SlimShape(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int), ("m", ctypes.c_int), ("beta", ctypes.c_int), ("t_c", ctypes.c_int64),
                ("t_s", ctypes.c_int64), ("t_x", ctypes.c_int), ("lwc_steps", ctypes.c_int)]


class SlimEpilogue(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("bias_dtype", ctypes.c_int), ("act", ctypes.c_int), ("R", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("Z", ctypes.c_void_p), ("ldz", ctypes.c_int64)]


_EPILOGUE = struct.Struct("PiiPqPq")          # the same as bytes, which are made in a fifth of the time


class AddNorm(NamedTuple):
    """What Slim.add_norm returns; what was not asked for is None."""
    H: torch.Tensor                  # the residual stream
    Y: Optional[torch.Tensor]        # its norm
    q: Optional[torch.Tensor]        # the same in 8 bits: numbers and scales
    s: Optional[torch.Tensor]
    mean: Optional[torch.Tensor]     # of the rows, for the backward pass
    rstd: Optional[torch.Tensor]


def workspace_query(n: int, m: int, beta: int, t_c: int = 0, t_s: int = 0, t_x: int = 0, num_cus: int = 0,
                    lwc_steps: int = 0) -> int:
    """Bytes of workspace the entry points need for a layer of this shape (host only, no GPU needed)."""
    return int(load().slim_workspace_query(ctypes.byref(SlimShape(n, m, beta, t_c, t_s, t_x, lwc_steps)), num_cus))


def zero_bits_for(N: int) -> int:
    """Width of a packed zero point (the stored value is 2 z) for a layer of target width N (App. B.2)."""
    return int(N) + 2


def bit_base_for(N: int) -> int:
    """The width that the 2-bit group value 0 of the stored form stands for, for a layer of target width N (App. B.2):
    1 for the targets 2 and 3, N - 2 above them, so that N - 1, N, N + 1 always fit the four values."""
    return max(1, int(N) - 2)


class SlimError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("libslim status %d: %s" % (status, message))
        self.status = status


_lib = None


def load() -> ctypes.CDLL:
    """Loads the built library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2405_14917_amd.build`" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    c_void_p, c_int, c_i64, c_double = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double
    P = ctypes.POINTER
    lib.slim_default_params.argtypes = [P(SlimParams)]
    lib.slim_default_params.restype = None
    lib.slim_default_tau.argtypes = [P(c_double), c_int]
    lib.slim_default_tau.restype = c_int
    lib.slim_create.argtypes = [P(c_void_p), c_void_p, c_void_p, ctypes.c_size_t]
    lib.slim_workspace_query.argtypes = [P(SlimShape), c_int]
    lib.slim_workspace_query.restype = ctypes.c_size_t
    lib.slim_destroy.argtypes = [c_void_p]
    lib.slim_last_error.argtypes = [c_void_p]
    lib.slim_last_error.restype = ctypes.c_char_p
    lib.slim_workspace_bytes.argtypes = [c_void_p]
    lib.slim_workspace_bytes.restype = ctypes.c_size_t
    lib.slim_hessian_accumulate.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_i64, c_void_p, c_i64, P(c_i64)]
    lib.slim_hessian_inverse.argtypes = [c_void_p, c_void_p, c_i64, c_int, c_i64, c_double, c_void_p, c_i64,
                                         c_void_p, P(c_int)]
    lib.slim_salience.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64, c_void_p, c_i64, c_void_p, c_int,
                                  c_int, c_void_p, c_void_p, c_void_p]
    lib.slim_sba_allocate.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64, c_void_p, c_int, c_int, c_int,
                                      c_void_p, c_int, c_i64, c_i64, P(SlimParams), c_void_p, P(c_int), P(c_double)]
    lib.slim_sba_prepare.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64, c_int, c_int, c_int, c_void_p,
                                     c_int, c_i64, c_i64, P(SlimParams)]
    lib.slim_sqc_calibrate.argtypes = [c_void_p, c_void_p, c_i64, c_int, c_int, c_int, c_void_p, c_void_p,
                                       P(SlimParams), c_void_p, c_int, c_void_p, c_void_p, c_void_p]
    lib.slim_gptq_quantize.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64, c_void_p, c_i64, c_void_p,
                                       c_int, c_int, P(SlimParams), c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_int, c_void_p]
    lib.slim_dequant_matmul.argtypes = [c_void_p, c_void_p, c_i64, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                        c_int, c_int, c_int, c_void_p, c_int, c_int, c_i64, c_void_p, c_i64]
    lib.slim_dequant_matmul_noalloc.argtypes = lib.slim_dequant_matmul.argtypes
    lib.slim_dequant_matmul_handover.argtypes = lib.slim_dequant_matmul.argtypes + [c_void_p, c_i64]
    lib.slim_transpose_16.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_void_p, c_i64]
    lib.slim_dequant_matmul_zp.argtypes = [c_void_p, c_void_p, c_i64, c_void_p, c_void_p, c_void_p, c_void_p, c_i64, c_int,
                                           c_int, c_int, c_int, c_int, c_void_p, c_int, c_int, c_i64, c_void_p, c_i64]
    lib.slim_pack.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_void_p, c_int, c_int, c_void_p, c_i64,
                              c_void_p, c_void_p, P(c_int)]
    lib.slim_pack_zeros.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_int, c_void_p, c_i64, P(c_int)]
    lib.slim_unpack_zeros.argtypes = [c_void_p, c_void_p, c_i64, c_int, c_int, c_int, c_void_p, c_i64]
    lib.slim_lwc_quantize.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64, c_void_p, c_i64, c_i64, c_void_p,
                                      c_int, c_int, c_double, c_double, c_double, c_double, c_double, c_void_p, c_void_p,
                                      c_void_p, c_void_p, c_int, P(c_double)]
    c_size_t = ctypes.c_size_t
    lib.slim_fp8_quantize_weights.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_i64] + [c_void_p, c_i64] * 4
    lib.slim_fp8_linear_workspace.argtypes = [c_int] * 5
    lib.slim_fp8_linear.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_void_p, c_i64, c_void_p, c_i64, c_int, c_int, c_void_p,
                                    c_int, c_i64]
    lib.slim_fp8_linear_backward_workspace.argtypes = [c_int] * 7
    lib.slim_fp8_linear_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_i64, c_i64, c_void_p, c_i64, c_void_p, c_i64,
                                             c_int, c_int, c_void_p, c_i64, c_void_p, c_int, c_i64]
    lib.slim_layer_norm.argtypes = [c_void_p, c_void_p, c_int, c_i64, c_int, c_i64, c_void_p, c_void_p, c_int, c_double, c_int, c_void_p,
                                    c_i64, c_void_p, c_void_p]
    lib.slim_layer_norm_backward_workspace.argtypes = [c_i64, c_int, c_int, c_int, c_int]
    lib.slim_layer_norm_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_i64, c_int, c_i64, c_i64, c_void_p, c_int, c_void_p,
                                             c_void_p, c_void_p, c_i64, c_void_p, c_void_p]
    lib.slim_distill_loss.argtypes = [c_void_p, c_void_p, c_int, c_i64, c_int, c_i64, c_void_p, c_int, c_void_p, c_int, c_int, c_i64,
                                      c_void_p, c_double, c_void_p]
    lib.slim_distill_loss_grad.argtypes = lib.slim_distill_loss.argtypes[:-1] + [c_void_p, c_void_p, c_void_p, c_i64]
    lib.slim_distill_workspace.argtypes = [c_i64, c_int, c_int]
    lib.slim_fp8_linear_act_workspace.argtypes = [c_int] * 6
    lib.slim_fp8_linear_act.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64] + [c_void_p, c_i64] * 4 + [c_int, c_int, c_void_p, c_void_p,
                                                                                                          c_int, c_i64]
    lib.slim_fp8_linear_act_backward_workspace.argtypes = [c_int] * 8
    lib.slim_fp8_linear_act_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int, c_i64, c_i64, c_i64, c_void_p, c_i64,
                                                 c_void_p, c_i64, c_int, c_int, c_void_p, c_i64, c_void_p, c_int, c_i64, c_void_p, c_int]
    lib.slim_add_norm.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_i64, c_int, c_i64, c_i64, c_void_p, c_void_p, c_int, c_double, c_int,
                                  c_void_p, c_i64, c_void_p, c_i64, c_void_p, c_i64, c_void_p, c_i64, c_void_p, c_void_p]
    lib.slim_add_norm_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_i64, c_int, c_i64, c_i64, c_i64, c_void_p, c_int,
                                           c_void_p, c_void_p, c_void_p, c_i64, c_void_p, c_void_p]
    lib.slim_head_loss_workspace.argtypes = [c_int] * 4
    lib.slim_head_loss.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64, c_void_p, c_i64, c_void_p, c_i64, c_int, c_int, c_void_p, c_int, c_void_p]
    lib.slim_head_loss_grad_workspace.argtypes = [c_int] * 7
    lib.slim_head_loss_grad.argtypes = [c_void_p, c_void_p, c_int, c_int, c_i64] + [c_void_p, c_i64] * 4 + [c_int, c_int, c_void_p, c_int, c_void_p,
                                                                                                          c_void_p, c_void_p, c_i64, c_void_p, c_int, c_i64]
    lib.slim_grad_norm_workspace.argtypes = [c_int, c_int]
    lib.slim_grad_norm.argtypes = [c_void_p, c_void_p, c_int, c_void_p]
    lib.slim_clip_gradients.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_double, c_void_p]
    for fn in (lib.slim_head_loss_workspace, lib.slim_head_loss_grad_workspace, lib.slim_fp8_linear_act_workspace, lib.slim_fp8_linear_act_backward_workspace, lib.slim_grad_norm_workspace, lib.slim_distill_workspace, lib.slim_fp8_linear_workspace, lib.slim_fp8_linear_backward_workspace, lib.slim_layer_norm_backward_workspace):
        fn.restype = c_size_t
    lib.slim_profile_enable.argtypes = [c_void_p, c_int]
    lib.slim_profile_collect.argtypes = [c_void_p]
    lib.slim_profile_collect.restype = c_int
    lib.slim_profile_entry.argtypes = [c_void_p, c_int, P(ctypes.c_char_p), P(c_double), P(c_int)]
    lib.slim_profile_reset.argtypes = [c_void_p]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("slim_default_params", "slim_default_tau", "slim_last_error", "slim_workspace_bytes",
                        "slim_workspace_query", "slim_profile_collect") and not name.endswith("_workspace"):
            fn.restype = c_int
    _lib = lib
    return lib


def default_tau() -> np.ndarray:
    lib = load()
    n = lib.slim_default_tau(None, 0)
    buf = (ctypes.c_double * n)()
    lib.slim_default_tau(buf, n)
    return np.frombuffer(buf, dtype=np.float64).copy()


def make_params(sqc_weight_mode: int = 0, mask_scope: int = 0, q1_mode: int = 0, sal_mode: int = 0) -> SlimParams:
    return SlimParams(sqc_weight_mode, mask_scope, q1_mode, sal_mode)


def _dtype(t: torch.Tensor) -> int:
    try:
        return _DT[t.dtype]
    except KeyError:
        raise ValueError("libslim has no %s" % t.dtype) from None


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


_E4M3 = torch.float8_e4m3fn
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def fp8_linear_workspace(n: int, m: int, t: int, dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.fp8_linear (host only, no GPU needed)."""
    return int(load().slim_fp8_linear_workspace(n, m, t, _DT[dtype], num_cus))


def fp8_linear_backward_workspace(n: int, m: int, t: int, dx: bool = True, dw: bool = True,
                                  dw_dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.fp8_linear_backward (host only, no GPU needed)."""
    return int(load().slim_fp8_linear_backward_workspace(n, m, t, int(dx), int(dw), _DT[dw_dtype], num_cus))


def layer_norm_backward_workspace(rows: int, cols: int, bias: bool = True, dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.layer_norm_backward (host only, no GPU needed)."""
    return int(load().slim_layer_norm_backward_workspace(rows, cols, _DT[dtype], int(bias), num_cus))


def distill_workspace(rows: int, V: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace of Slim.distill_loss and Slim.distill_loss_grad for logits of `dtype` (host only, no GPU needed)."""
    return int(load().slim_distill_workspace(rows, V, _DT[dtype]))


def fp8_linear_act_workspace(n: int, m: int, t: int, x_8bit: bool = False, dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.fp8_linear_act (host only, no GPU needed)."""
    return int(load().slim_fp8_linear_act_workspace(n, m, t, int(x_8bit), _DT[dtype], num_cus))


def fp8_linear_act_backward_workspace(n: int, m: int, t: int, dx: bool = True, dw: bool = True, dw_dtype: torch.dtype = torch.bfloat16,
                                      db: bool = True, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.fp8_linear_act_backward (host only, no GPU needed)."""
    return int(load().slim_fp8_linear_act_backward_workspace(n, m, t, int(dx), int(dw), _DT[dw_dtype], int(db), num_cus))


def head_loss_workspace(V: int, m: int, t: int, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.head_loss (host only, no GPU needed)."""
    return int(load().slim_head_loss_workspace(V, m, t, num_cus))


def head_loss_grad_workspace(V: int, m: int, t: int, dx: bool = True, dw: bool = True, dw_dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.head_loss_grad (host only, no GPU needed)."""
    return int(load().slim_head_loss_grad_workspace(V, m, t, int(dx), int(dw), _DT[dw_dtype], num_cus))


def grad_norm_workspace(count: int, num_cus: int = 0) -> int:
    """Bytes of workspace of Slim.grad_norm and Slim.clip_gradients for `count` tensors (host only, no GPU needed)."""
    return int(load().slim_grad_norm_workspace(count, num_cus))


_FLOATS = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}


def _tensor_list(tensors, what: str):
    """The descriptions (address, rows, columns, leading dimension, type) that the library takes of a list of tensors."""
    flat = []
    for t in tensors:
        d = _FLOATS.get(t.dtype)
        if d is None:
            raise ValueError("%s have to be float16, bfloat16 or float32" % what)
        if t.is_contiguous():
            n = t.numel()
            flat += (t.data_ptr(), 1, n, n, d)
        elif t.dim() == 2:
            flat += (t.data_ptr(), t.shape[0], t.shape[1], _row_stride(t, what), d)
        else:
            raise ValueError("%s have to be contiguous, or matrices with contiguous rows" % what)
    return array.array("q", flat)


def _address(a: array.array) -> int:
    return a.buffer_info()[0]


def _tensor_rows(tensors, what: str):
    """The same with matrices described by their rows, contiguous or not."""
    flat = _tensor_list(tensors, what)
    for i, t in enumerate(tensors):
        if t.dim() == 2:
            flat[5 * i + 1], flat[5 * i + 2], flat[5 * i + 3] = t.shape[0], t.shape[1], _row_stride(t, what)
    return flat


def _check_act(act):
    if act not in ACTIVATIONS:
        raise ValueError("act has to be one of %s, got %r" % (", ".join(str(a) for a in ACTIVATIONS), act))
    return ACTIVATIONS[act]


def _empty_like(x: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of x's shape and type."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def _row_stride(x: torch.Tensor, what: str) -> int:
    """The leading dimension of a matrix whose rows are contiguous."""
    if x.dim() != 2:
        raise ValueError("%s has to be a matrix, got %d dimensions" % (what, x.dim()))
    rows, cols = x.shape
    ld, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError("libslim takes row-major tensors (last dimension contiguous): %s" % what)
    if rows <= 1 or cols == 0:
        return max(cols, 1)
    if ld < cols:
        raise ValueError("rows of %s overlap" % what)
    return ld


def _stored_strides(q: torch.Tensor, s: torch.Tensor, what: str, rows: int = 128):
    """Leading dimensions of stored 8-bit weights, in blocks of 128 x 128, or of activations (`rows` = 1); raises where they are not what
    Slim.fp8_quantize_weights or Slim.add_norm makes."""
    if q.dtype != _E4M3 or s.dtype != torch.uint8 or q.dim() != 2 or s.dim() != 2:
        raise ValueError("%s has to be a float8_e4m3fn matrix, its scales a uint8 matrix" % what)
    n, m = q.shape
    nb, mb = (n + rows - 1) // rows, (m + 127) // 128
    if s.shape != (nb, mb):
        raise ValueError("%s (%d x %d) needs %d x %d scales, got %d x %d" % (what, n, m, nb, mb, s.shape[0], s.shape[1]))
    (ldq, qstep), (lds, sstep) = q.stride(), s.stride()
    if qstep != 1 and m > 1 or sstep != 1 and mb > 1:
        raise ValueError("libslim takes row-major tensors (last dimension contiguous): %s" % what)
    if ldq % 128 or lds % 4 or ldq < m or lds < mb:
        raise ValueError("rows of %s have to be whole blocks of 128 and those of its scales whole words apart, got %d and %d" % (what, ldq, lds))
    # rows are read to the end of their last block, and scales by the word: the padding of the last row has to be there as well
    if (m % 128 and q.untyped_storage().nbytes() - q.storage_offset() < (n - 1) * ldq + mb * 128 or
            mb % 4 and s.untyped_storage().nbytes() - s.storage_offset() < (nb - 1) * lds + (mb + 3) // 4 * 4):
        raise ValueError("the padding of the last row of %s or of its scales is missing" % what)
    return ldq, lds


def _stored_out(out, n: int, m: int, transposed: bool):
    """Stored weights given to be written over, checked: (q, s, qt, st), the last two None without `transposed`."""
    if len(out) != (4 if transposed else 2):
        raise ValueError("out has to be the %d tensors of an earlier call" % (4 if transposed else 2))
    for q, s, shape in ((out[0], out[1], (n, m)),) + (((out[2], out[3], (m, n)),) if transposed else ()):
        _stored_strides(q, s, "out")
        if q.shape != shape:
            raise ValueError("out holds weights of %d x %d, got %d x %d" % (*q.shape, *shape))
    return (*out, None, None)[:4]


def _no_graph(*tensors):
    """Raises where autograd would expect a recorded call: these calls record none, and their outputs would silently carry no gradient."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("libslim records no graph: a tensor that requires a gradient is taken under torch.no_grad(), or detached")


def _need_cuda(*tensors):
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("libslim takes device tensors")
        if t.dim() >= 1 and t.stride(-1) != 1:
            raise ValueError("libslim takes row-major tensors (last dimension contiguous)")


class Slim:
    """A library context bound to the current torch stream of `device`."""

    def __init__(self, device: str = "cuda:0", workspace_bytes: int = 0):
        """workspace_bytes > 0: the context works in a buffer of that size allocated here, once (see
        workspace_query), and no entry point allocates device memory; 0: the library grows its own on demand."""
        self.lib = load()
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = torch.cuda.current_stream(self.device)
        self._index, self._raw_stream = self.stream.device.index, self.stream.cuda_stream
        self.workspace = (torch.empty(workspace_bytes + 256, dtype=torch.uint8, device=self.device)
                          if workspace_bytes > 0 else None)
        ws_ptr = None
        if self.workspace is not None:
            ws_ptr = ctypes.c_void_p((self.workspace.data_ptr() + 255) // 256 * 256)
        handle = ctypes.c_void_p()
        st = self.lib.slim_create(ctypes.byref(handle), ctypes.c_void_p(self.stream.cuda_stream), ws_ptr,
                                  workspace_bytes)
        if st != SLIM_OK:
            raise SlimError(st, "slim_create failed")
        self.ctx = handle

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.slim_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != SLIM_OK:
            raise SlimError(st, self.lib.slim_last_error(self.ctx).decode())

    def workspace_bytes(self) -> int:
        return int(self.lib.slim_workspace_bytes(self.ctx))

    # ---- a1
    def hessian_accumulate(self, X: torch.Tensor, G: torch.Tensor, n_tokens: int = 0) -> int:
        """G (m x m float32) += X X^T for X of shape (m, t_c) float16 / bfloat16; returns the new token count."""
        _need_cuda(X, G)
        m, t_c = X.shape
        assert X.stride(1) == 1 and G.stride(1) == 1 and G.dtype == torch.float32
        nt = ctypes.c_int64(n_tokens)
        self._check(self.lib.slim_hessian_accumulate(self.ctx, _ptr(X), _DT[X.dtype], m, t_c, X.stride(0), _ptr(G),
                                                     G.stride(0), ctypes.byref(nt)))
        return int(nt.value)

    # ---- a2
    def hessian_inverse(self, G: torch.Tensor, n_tokens: int, percdamp: float = 0.01,
                        U: Optional[torch.Tensor] = None, hinv_diag: Optional[torch.Tensor] = None):
        """Returns (U float64 (m, m) upper, hinv_diag float64 (m,)); raises SlimError(ERR_NOT_PD) otherwise."""
        _need_cuda(G)
        m = G.shape[0]
        U = torch.empty((m, m), dtype=torch.float64, device=G.device) if U is None else U
        hinv_diag = torch.empty(m, dtype=torch.float64, device=G.device) if hinv_diag is None else hinv_diag
        info = ctypes.c_int(0)
        st = self.lib.slim_hessian_inverse(self.ctx, _ptr(G), G.stride(0), m, n_tokens, percdamp, _ptr(U), U.stride(0),
                                           _ptr(hinv_diag), ctypes.byref(info))
        self.last_info = int(info.value)
        self._check(st)
        return U, hinv_diag

    # ---- a3
    def salience(self, W: torch.Tensor, hinv_diag: Optional[torch.Tensor], beta: int, U: Optional[torch.Tensor] = None,
                 sal_mode: int = SAL_HINV_DIAG, want_elem: bool = False):
        _need_cuda(W, hinv_diag, U)
        n, m = W.shape
        col = torch.empty(m, dtype=torch.float64, device=W.device)
        grp = torch.empty(max(m // max(beta, 1), 1), dtype=torch.float64, device=W.device)
        elem = torch.empty((n, m), dtype=torch.float64, device=W.device) if want_elem else None
        self._check(self.lib.slim_salience(self.ctx, _ptr(W), _DT[W.dtype], n, m, W.stride(0), _ptr(U),
                                           0 if U is None else U.stride(0), _ptr(hinv_diag), sal_mode, beta, _ptr(col),
                                           _ptr(grp), _ptr(elem)))
        return col, grp, elem

    # ---- a4
    def sba_prepare(self, W: torch.Tensor, beta: int, N: int, Xs: torch.Tensor, params: Optional[SlimParams] = None,
                    objective: int = OBJ_KL) -> None:
        """Enqueues the part of sba_allocate that needs no salience; the next call on this context must be
        sba_allocate with the same W, Xs, beta, N, params and objective."""
        _need_cuda(W, Xs)
        n, m = W.shape
        self._check(self.lib.slim_sba_prepare(self.ctx, _ptr(W), _DT[W.dtype], n, m, W.stride(0), beta, N, objective,
                                              _ptr(Xs), _DT[Xs.dtype], Xs.shape[1], Xs.stride(0),
                                              ctypes.byref(params) if params is not None else None))

    def sba_allocate(self, W: torch.Tensor, group_sal: torch.Tensor, beta: int, N: int, Xs: torch.Tensor,
                     params: Optional[SlimParams] = None, objective: int = OBJ_KL, host_outputs: bool = True):
        """Returns (bits uint8 device tensor (k,), p_star, obj_curve numpy (k//2+1,)); with host_outputs=False the
        call does not wait for the stream and the last two are None."""
        _need_cuda(W, group_sal, Xs)
        n, m = W.shape
        k = m // beta
        t_s = Xs.shape[1]
        bits = torch.empty(k, dtype=torch.uint8, device=W.device)
        p_star = ctypes.c_int(-1)
        curve = (ctypes.c_double * (k // 2 + 1))()
        self._check(self.lib.slim_sba_allocate(self.ctx, _ptr(W), _DT[W.dtype], n, m, W.stride(0), _ptr(group_sal), beta,
                                               N, objective, _ptr(Xs), _DT[Xs.dtype], t_s, Xs.stride(0),
                                               ctypes.byref(params) if params is not None else None, _ptr(bits),
                                               ctypes.byref(p_star) if host_outputs else None,
                                               curve if host_outputs else None))
        if not host_outputs:
            return bits, None, None
        return bits, int(p_star.value), np.frombuffer(curve, dtype=np.float64).copy()

    # ---- a5 + a6
    def sqc_calibrate(self, Wblk: torch.Tensor, bits: int, params: Optional[SlimParams] = None,
                      omega: Optional[torch.Tensor] = None, hinv_diag_blk: Optional[torch.Tensor] = None,
                      tau: Optional[torch.Tensor] = None):
        """Wblk float64 (n, beta).  Returns (scale, zero float64 (n,), cand_idx int32 (n,))."""
        _need_cuda(Wblk, omega, hinv_diag_blk, tau)
        n, beta = Wblk.shape
        scale = torch.empty(n, dtype=torch.float64, device=Wblk.device)
        zero = torch.empty(n, dtype=torch.float64, device=Wblk.device)
        idx = torch.empty(n, dtype=torch.int32, device=Wblk.device)
        self._check(self.lib.slim_sqc_calibrate(self.ctx, _ptr(Wblk), Wblk.stride(0), n, beta, bits, _ptr(omega),
                                                _ptr(hinv_diag_blk),
                                                ctypes.byref(params) if params is not None else None, _ptr(tau),
                                                0 if tau is None else tau.numel(), _ptr(scale), _ptr(zero), _ptr(idx)))
        return scale, zero, idx

    # ---- a5 - a8
    def gptq_quantize(self, W: torch.Tensor, U: torch.Tensor, bits: torch.Tensor, beta: int,
                      params: Optional[SlimParams] = None, hinv_diag: Optional[torch.Tensor] = None,
                      tau: Optional[torch.Tensor] = None, want_what: Optional[torch.dtype] = None,
                      want_sum_e2: bool = False, gptq_block: Optional[int] = None):
        """Returns dict(codes uint8 (n, m), scale, zero float64 (n, k), What or None, sum_e2 or None)."""
        _need_cuda(W, U, bits, hinv_diag, tau)
        n, m = W.shape
        k = m // beta
        codes = torch.empty((n, m), dtype=torch.uint8, device=W.device)
        scale = torch.empty((n, k), dtype=torch.float64, device=W.device)
        zero = torch.empty((n, k), dtype=torch.float64, device=W.device)
        what = torch.empty((n, m), dtype=want_what, device=W.device) if want_what is not None else None
        se2 = torch.zeros(1, dtype=torch.float64, device=W.device) if want_sum_e2 else None
        self._check(self.lib.slim_gptq_quantize(self.ctx, _ptr(W), _DT[W.dtype], n, m, W.stride(0), _ptr(U), U.stride(0),
                                                _ptr(bits), beta, beta if gptq_block is None else gptq_block,
                                                ctypes.byref(params) if params is not None else None, _ptr(hinv_diag),
                                                _ptr(tau), 0 if tau is None else tau.numel(), _ptr(codes), _ptr(scale),
                                                _ptr(zero), _ptr(what), F32 if what is None else _DT[what.dtype],
                                                _ptr(se2)))
        return dict(codes=codes, scale=scale, zero=zero, What=what, sum_e2=se2)

    # ---- a9
    def pack(self, codes: torch.Tensor, bits: torch.Tensor, beta: int, packed_rows: Optional[int] = None,
             host_outputs: bool = True, bit_base: int = 1):
        """Returns (packed uint32-as-int32 (m_star, n), gbits (ceil(k/16),), row_off int32 (k+1,), m_star); with
        host_outputs=False the call does not wait for the stream: packed then has all rows of its capacity (zero
        from row m_star = row_off[k] on) and m_star is None.  bit_base is the width that the 2-bit group value 0
        stands for (bit_base_for(N) of the layer's target width)."""
        _need_cuda(codes, bits)
        n, m = codes.shape
        k = m // beta
        cap = m * (bit_base + 3) // 32 if packed_rows is None else packed_rows     # the widest width the base allows
        packed = torch.zeros((max(cap, 1), n), dtype=torch.int32, device=codes.device)
        gbits = torch.zeros((k + 15) // 16, dtype=torch.int32, device=codes.device)
        row_off = torch.zeros(k + 1, dtype=torch.int32, device=codes.device)
        m_star = ctypes.c_int(0)
        self._check(self.lib.slim_pack(self.ctx, _ptr(codes), n, m, codes.stride(0), _ptr(bits), beta, bit_base, _ptr(packed), cap,
                                       _ptr(gbits), _ptr(row_off), ctypes.byref(m_star) if host_outputs else None))
        if not host_outputs:
            return packed, gbits, row_off, None
        return packed[: m_star.value], gbits, row_off, int(m_star.value)

    def pack_zeros(self, zero: torch.Tensor, zbits: int, host_outputs: bool = True):
        """zero float64 (n, k) -> (zpacked uint32-as-int32 (k, ceil(n zbits / 32)), number of zeros that did not fit
        or None with host_outputs=False)."""
        _need_cuda(zero)
        n, k = zero.shape
        zp = torch.empty((k, (n * zbits + 31) // 32), dtype=torch.int32, device=zero.device)
        bad = ctypes.c_int(0)
        self._check(self.lib.slim_pack_zeros(self.ctx, _ptr(zero), n, k, zero.stride(0), zbits, _ptr(zp), zp.stride(0),
                                             ctypes.byref(bad) if host_outputs else None))
        return zp, (int(bad.value) if host_outputs else None)

    def unpack_zeros(self, zp: torch.Tensor, n: int, zbits: int):
        _need_cuda(zp)
        k = zp.shape[0]
        zero = torch.empty((n, k), dtype=torch.float64, device=zp.device)
        self._check(self.lib.slim_unpack_zeros(self.ctx, _ptr(zp), zp.stride(0), n, k, zbits, _ptr(zero), zero.stride(0)))
        return zero

    # ---- n4
    def lwc_quantize(self, W: torch.Tensor, G: torch.Tensor, n_tokens: int, bits: torch.Tensor, beta: int, steps: int = 20,
                     lr: float = 1e-2, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, init: float = 4.0,
                     want_what: Optional[torch.dtype] = None, host_outputs: bool = True):
        """SliM-LLM+ on one layer.  Returns dict(codes uint8 (n, m), scale, zero float64 (n, k), What or None,
        loss_curve numpy (steps + 1,) or None with host_outputs=False)."""
        _need_cuda(W, G, bits)
        n, m = W.shape
        k = m // beta
        codes = torch.empty((n, m), dtype=torch.uint8, device=W.device)
        scale = torch.empty((n, k), dtype=torch.float64, device=W.device)
        zero = torch.empty((n, k), dtype=torch.float64, device=W.device)
        what = torch.empty((n, m), dtype=want_what, device=W.device) if want_what is not None else None
        curve = (ctypes.c_double * (steps + 1))()
        self._check(self.lib.slim_lwc_quantize(self.ctx, _ptr(W), _DT[W.dtype], n, m, W.stride(0), _ptr(G), G.stride(0),
                                               n_tokens, _ptr(bits), beta, steps, lr, beta1, beta2, eps, init, _ptr(codes),
                                               _ptr(scale), _ptr(zero), _ptr(what),
                                               F32 if what is None else _DT[what.dtype], curve if host_outputs else None))
        return dict(codes=codes, scale=scale, zero=zero, What=what,
                    loss_curve=np.frombuffer(curve, dtype=np.float64).copy() if host_outputs else None)

    # ---- n1
    def dequant_matmul(self, packed: torch.Tensor, gbits: torch.Tensor, row_off: torch.Tensor, scale: torch.Tensor,
                       zero: torch.Tensor, beta: int, X: torch.Tensor, Y: Optional[torch.Tensor] = None,
                       bit_base: int = 1, noalloc: bool = False):
        """Y (t_x, n) float32 = X (t_x, m) float16 / bfloat16 times the dequantised weights, from the stored form.
        noalloc=True calls slim_dequant_matmul_noalloc (Y must then be passed in, so that nothing is allocated)."""
        _need_cuda(packed, gbits, row_off, scale, zero, X)
        n = packed.shape[1]
        t_x, m = X.shape
        assert scale.dtype == torch.float64 and zero.dtype == torch.float64 and scale.stride(0) == m // beta
        Y = torch.empty((t_x, n), dtype=torch.float32, device=X.device) if Y is None else Y
        fn = self.lib.slim_dequant_matmul_noalloc if noalloc else self.lib.slim_dequant_matmul
        self._check(fn(self.ctx, _ptr(packed), packed.stride(0), _ptr(gbits), _ptr(row_off),
                                                 _ptr(scale), _ptr(zero), n, m, beta, bit_base, _ptr(X), _DT[X.dtype], t_x,
                                                 X.stride(0), _ptr(Y), Y.stride(0)))
        return Y

    def dequant_matmul_zp(self, packed: torch.Tensor, gbits: torch.Tensor, row_off: torch.Tensor, scale: torch.Tensor,
                          zpacked: torch.Tensor, zbits: int, beta: int, X: torch.Tensor, bit_base: int = 1):
        """The linear layer on the stored form with packed zero points (from pack_zeros)."""
        _need_cuda(packed, gbits, row_off, scale, zpacked, X)
        n = packed.shape[1]
        t_x, m = X.shape
        Y = torch.empty((t_x, n), dtype=torch.float32, device=X.device)
        self._check(self.lib.slim_dequant_matmul_zp(self.ctx, _ptr(packed), packed.stride(0), _ptr(gbits), _ptr(row_off),
                                                    _ptr(scale), _ptr(zpacked), zpacked.stride(0), zbits, n, m, beta,
                                                    bit_base, _ptr(X), _DT[X.dtype], t_x, X.stride(0), _ptr(Y), Y.stride(0)))
        return Y

    def dequant_matmul_handover(self, packed: torch.Tensor, gbits: torch.Tensor, row_off: torch.Tensor, scale: torch.Tensor,
                                zero: torch.Tensor, beta: int, X: torch.Tensor, Xn: torch.Tensor, Y: torch.Tensor,
                                bit_base: int = 1):
        """Xn (n, t_x) float16, tokens contiguous: the outputs for X (t_x, m), clamped and rounded; Y (t_x, n) float32 is
        scratch."""
        _need_cuda(packed, gbits, row_off, scale, zero, X, Xn, Y)
        t_x, m = X.shape
        n = packed.shape[1]
        assert scale.dtype == torch.float64 and zero.dtype == torch.float64 and scale.stride(0) == m // beta
        assert Xn.shape == (n, t_x) and Xn.dtype == torch.float16 and Xn.stride(1) == 1 and Y.shape == (t_x, n)
        self._check(self.lib.slim_dequant_matmul_handover(self.ctx, _ptr(packed), packed.stride(0), _ptr(gbits), _ptr(row_off),
                                                          _ptr(scale), _ptr(zero), n, m, beta, bit_base, _ptr(X), _DT[X.dtype],
                                                          t_x, X.stride(0), _ptr(Y), Y.stride(0), _ptr(Xn), Xn.stride(0)))
        return Xn

    def transpose_16(self, X: torch.Tensor, out: torch.Tensor):
        """out (cols, rows) = X (rows, cols) transposed; 16-bit elements, both with contiguous rows."""
        _need_cuda(X, out)
        assert X.element_size() == 2 and out.dtype == X.dtype and out.shape == (X.shape[1], X.shape[0])
        assert X.stride(1) == 1 and out.stride(1) == 1
        self._check(self.lib.slim_transpose_16(self.ctx, _ptr(X), X.shape[0], X.shape[1], X.stride(0), _ptr(out), out.stride(0)))
        return out

    # ---- around a quantised layer: 8-bit linear layer, norms, divergence from a teacher
    def _ready(self, *tensors):
        """Tensors on the context's device, and the context's stream current: outputs are allocated on the current one."""
        index = self._index
        for t in tensors:
            if t is not None and t.get_device() != index:
                raise ValueError("libslim takes tensors of the context's device")
        if _current_stream(index) != self._raw_stream:
            raise ValueError("the context is bound to another stream than the current one")

    def fp8_quantize_weights(self, W: torch.Tensor, transposed: bool = True, out=None):
        """W (n, m) float16 / bfloat16 / float32 as stored 8-bit weights: (q float8_e4m3fn (n, m), s uint8 (n / 128, m / 128 rounded up)),
        and with `transposed` also those of W^T, which the backward pass reads.  Rows are padded: keep the tensors as they are.  `out`: the
        tensors of an earlier call for weights of this shape, to be written over (what a captured graph reads has to stay in its place)."""
        self._ready(W, *(out or ()))
        if W.dim() != 2:
            raise ValueError("W has to be a matrix")
        n, m = W.shape
        nb, mb = (n + 127) // 128, (m + 127) // 128

        def stored(rows, cols, rb, cb):
            # (rows an odd number of blocks apart: they spread over the channels of the L2)
            q = torch.zeros((rows, (cb | 1) * 128), dtype=torch.uint8, device=W.device).view(_E4M3)[:, :cols]
            return q, torch.zeros((rb, (cb + 3) // 4 * 4), dtype=torch.uint8, device=W.device)[:, :cb]

        if out is not None:
            q, s, qt, st = _stored_out(out, n, m, transposed)
        else:
            q, s = stored(n, m, nb, mb)
            qt, st = stored(m, n, mb, nb) if transposed else (None, None)
        self._check(self.lib.slim_fp8_quantize_weights(self.ctx, W.data_ptr(), _dtype(W), n, m, _row_stride(W, "W"), q.data_ptr(), q.stride(0),
                                                       s.data_ptr(), s.stride(0), _ptr(qt), qt.stride(0) if transposed else 0, _ptr(st),
                                                       st.stride(0) if transposed else 0))
        return (q, s, qt, st) if transposed else (q, s)

    def fp8_linear(self, X: torch.Tensor, W: torch.Tensor, Ws: torch.Tensor, dtype: Optional[torch.dtype] = None):
        """Y (t, n) = Q(X) W^T for X (t, m) float16 / bfloat16 and stored 8-bit weights W, Ws; `dtype`: of Y (default: X's).  Records no
        graph: X that requires a gradient is refused outside torch.no_grad() (detach it, and call fp8_linear_backward)."""
        _no_graph(X, W)
        self._ready(X, W, Ws)
        ldq, lds = _stored_strides(W, Ws, "W")
        n, m = W.shape
        if X.dim() != 2 or X.shape[1] != m:
            raise ValueError("X has to be (t, %d), got %s" % (m, tuple(X.shape)))
        t = X.shape[0]
        Y = X.new_empty((t, n), dtype=dtype)
        st = self.lib.slim_fp8_linear(self.ctx, X.data_ptr(), _dtype(X), t, _row_stride(X, "X"), W.data_ptr(), ldq, Ws.data_ptr(), lds, n, m,
                                      Y.data_ptr(), _dtype(Y), n)
        if st:
            self._check(st)
        return Y

    def fp8_linear_backward(self, dY: torch.Tensor, X: Optional[torch.Tensor], Wt: Optional[torch.Tensor], Wts: Optional[torch.Tensor],
                            dw_dtype: Optional[torch.dtype] = None, dx: bool = True, dw: bool = True):
        """(dX (t, m), dW (n, m)) for dY (t, n) and X (t, m) of one 16-bit type and the stored weights of W^T; dw_dtype: of dW (default:
        X's).  Without `dx` Wt and Wts may be None, without `dw` X; the gradient that is not wanted is None."""
        self._ready(dY, X, Wt, Wts)
        if not (dx or dw):
            raise ValueError("neither gradient is wanted")
        if dY.dim() != 2:
            raise ValueError("dY has to be a matrix")
        t, n = dY.shape
        ldqt = ldst = 0
        if dw:
            if X is None or X.dim() != 2 or X.shape[0] != t or X.dtype != dY.dtype:
                raise ValueError("X has to be a matrix of dY's tokens and type")
            m = X.shape[1]
        if dx:
            if Wt is None or Wts is None:
                raise ValueError("dX needs the stored weights of W^T")
            ldqt, ldst = _stored_strides(Wt, Wts, "Wt")
            if Wt.shape[1] != n or dw and Wt.shape[0] != m:
                raise ValueError("Wt has to be (m, n) = (%s, %d), got %s" % (m if dw else "m", n, tuple(Wt.shape)))
            m = Wt.shape[0]
        dX = dY.new_empty((t, m)) if dx else None
        dW = dY.new_empty((n, m), dtype=dw_dtype) if dw else None
        st = self.lib.slim_fp8_linear_backward(self.ctx, dY.data_ptr(), X.data_ptr() if dw else None, _dtype(dY), t, _row_stride(dY, "dY"),
                                               _row_stride(X, "X") if dw else 0, Wt.data_ptr() if dx else None, ldqt,
                                               Wts.data_ptr() if dx else None, ldst, n, m, dX.data_ptr() if dx else None, m,
                                               dW.data_ptr() if dw else None, _dtype(dW) if dw else F32, m)
        if st:
            self._check(st)
        return dX, dW

    def layer_norm(self, X: torch.Tensor, w: torch.Tensor, b: Optional[torch.Tensor] = None, eps: float = 1e-5, rms: bool = False,
                   stats: bool = False):
        """Layer norm of the rows of X (rows, cols), without the mean with `rms`; w, b (cols,) of X's type or float32.  With `stats`
        (Y, mean, rstd) for the backward pass (mean is None with `rms`).  Records no graph: without `stats` tensors that require a gradient
        are refused outside torch.no_grad()."""
        if not stats:                        # (who asks for them calls layer_norm_backward)
            _no_graph(X, w, b)
        self._ready(X, w, b)
        rows, cols = self._norm_shape(X, w, b)
        Y = _empty_like(X)
        mean = rstd = None
        if stats:
            mean = None if rms else X.new_empty(rows, dtype=torch.float32)
            rstd = X.new_empty(rows, dtype=torch.float32)
        st = self.lib.slim_layer_norm(self.ctx, X.data_ptr(), _dtype(X), rows, cols, _row_stride(X, "X"), w.data_ptr(),
                                      None if b is None else b.data_ptr(), _dtype(w), eps, rms, Y.data_ptr(), cols,
                                      None if mean is None else mean.data_ptr(), None if rstd is None else rstd.data_ptr())
        if st:
            self._check(st)
        return (Y, mean, rstd) if stats else Y

    def fp8_linear_act(self, X, W: torch.Tensor, Ws: torch.Tensor, bias: Optional[torch.Tensor] = None, act: Optional[str] = None,
                       residual: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, keep: bool = False):
        """Y (t, n) = act(Q(X) W^T + bias) + residual.  X: (t, m) float16 / bfloat16, or its 8-bit form (q, s) as add_norm makes it; bias (n,)
        of Y's type or float32; act: None, "relu", "gelu", "gelu_tanh" or "silu"; residual (t, n) of Y's type.  `dtype`: of Y (default: the
        residual's, else X's, else bfloat16).  With `keep` (Y, Z): the values before the activation in Y's type, for the backward pass.
        Records no graph (without `keep` tensors that require a gradient are refused outside torch.no_grad())."""
        xq = xs = None
        ldx = ldxq = ldxs = 0
        if isinstance(X, torch.Tensor):
            first = X
        else:
            xq, xs = X
            first = xq
        if not keep:
            _no_graph(first, bias, residual)
        self._ready(first, xs, W, Ws, bias, residual)
        ldq, lds = _stored_strides(W, Ws, "W")
        n, m = W.shape
        if first.dim() != 2 or first.shape[1] != m:
            raise ValueError("X has to be (t, %d), got %s" % (m, tuple(first.shape)))
        t = first.shape[0]
        if xq is None:
            ldx = _row_stride(X, "X")
        else:
            ldxq, ldxs = _stored_strides(xq, xs, "X", 1)
        if dtype is None:
            dtype = residual.dtype if residual is not None else X.dtype if xq is None else torch.bfloat16
        Y = W.new_empty((t, n), dtype=dtype)
        Z = W.new_empty((t, n), dtype=dtype) if keep else None
        y = _dtype(Y)
        b = r = ldr = 0
        b_dtype = y
        if bias is not None:
            if bias.shape != (n,) or not bias.is_contiguous():
                raise ValueError("bias has to be a contiguous vector of %d numbers" % n)
            b, b_dtype = bias.data_ptr(), _dtype(bias)
        if residual is not None:
            if residual.shape != (t, n) or residual.dtype != dtype:
                raise ValueError("residual has to be (%d, %d) of Y's type" % (t, n))
            r, ldr = residual.data_ptr(), _row_stride(residual, "residual")
        e = _EPILOGUE.pack(b, b_dtype, _check_act(act), r, ldr, Z.data_ptr() if keep else 0, n)
        st = self.lib.slim_fp8_linear_act(self.ctx, X.data_ptr() if xq is None else None, _dtype(X) if xq is None else F16, t, ldx,
                                          None if xq is None else xq.data_ptr(), ldxq, None if xs is None else xs.data_ptr(), ldxs,
                                          W.data_ptr(), ldq, Ws.data_ptr(), lds, n, m, e, Y.data_ptr(), y, n)
        if st:
            self._check(st)
        return (Y, Z) if keep else Y

    def fp8_linear_act_backward(self, dY: torch.Tensor, Z: Optional[torch.Tensor], act: Optional[str], X: Optional[torch.Tensor],
                                Wt: Optional[torch.Tensor], Wts: Optional[torch.Tensor], dw_dtype: Optional[torch.dtype] = None, dx: bool = True,
                                dw: bool = True, db_dtype: Optional[torch.dtype] = None):
        """(dX (t, m), dW (n, m), db (n,)) for dY and Z (t, n) and X (t, m) of one 16-bit type; Z is what fp8_linear_act kept (not
        needed without an activation); dw_dtype: of dW (default: X's); db_dtype: of db, None: not wanted.  Without `dx` Wt and Wts may be
        None, without `dw` X; the gradient that is not wanted is None.  That of the residual is dY."""
        a = _check_act(act)
        Z = Z if a else None
        self._ready(dY, Z, X, Wt, Wts)
        if not (dx or dw or db_dtype):
            raise ValueError("no gradient is wanted")
        if dY.dim() != 2:
            raise ValueError("dY has to be a matrix")
        t, n = dY.shape
        if a and (Z is None or Z.shape != dY.shape or Z.dtype != dY.dtype):
            raise ValueError("Z has to be of dY's shape and type")
        ldqt = ldst = 0
        m = 1
        if dw:
            if X is None or X.dim() != 2 or X.shape[0] != t or X.dtype != dY.dtype:
                raise ValueError("X has to be a matrix of dY's tokens and type")
            m = X.shape[1]
        if dx:
            if Wt is None or Wts is None:
                raise ValueError("dX needs the stored weights of W^T")
            ldqt, ldst = _stored_strides(Wt, Wts, "Wt")
            if Wt.shape[1] != n or dw and Wt.shape[0] != m:
                raise ValueError("Wt has to be (m, n) = (%s, %d), got %s" % (m if dw else "m", n, tuple(Wt.shape)))
            m = Wt.shape[0]
        dX = dY.new_empty((t, m)) if dx else None
        dW = dY.new_empty((n, m), dtype=dw_dtype) if dw else None
        db = dY.new_empty(n, dtype=db_dtype) if db_dtype else None
        st = self.lib.slim_fp8_linear_act_backward(
            self.ctx, dY.data_ptr(), None if Z is None else Z.data_ptr(), a, X.data_ptr() if dw else None, _dtype(dY), t, _row_stride(dY, "dY"),
            0 if Z is None else _row_stride(Z, "Z"), _row_stride(X, "X") if dw else 0, Wt.data_ptr() if dx else None, ldqt,
            Wts.data_ptr() if dx else None, ldst, n, m, dX.data_ptr() if dx else None, m, dW.data_ptr() if dw else None, _dtype(dW) if dw else F32, m,
            None if db is None else db.data_ptr(), F32 if db is None else _dtype(db))
        if st:
            self._check(st)
        return dX, dW, db

    def add_norm(self, X: torch.Tensor, R: Optional[torch.Tensor], w: torch.Tensor, b: Optional[torch.Tensor] = None, eps: float = 1e-5,
                 rms: bool = False, y: bool = True, e4m3: bool = False, stats: bool = False, H: Optional[torch.Tensor] = None) -> AddNorm:
        """The residual stream H = X + R (rounded to their type; R None: X) and its norm Y, as layer_norm's.  y: Y in X's type is wanted; e4m3:
        its 8-bit form (q, s), which fp8_linear_act takes; stats: mean (None with `rms`) and rstd for the backward pass.  H may be given, X or R
        among others.  Records no graph: without `stats` tensors that require a gradient are refused outside torch.no_grad()."""
        if not stats:
            _no_graph(X, R, w, b)
        _no_graph(H)                         # (written over)
        self._ready(X, R, w, b, H)
        rows, cols = self._norm_shape(X, w, b)
        if not (y or e4m3):
            raise ValueError("neither form of the norm is wanted")
        shape, dtype = X.shape, X.dtype
        if R is not None and (R.shape != shape or R.dtype != dtype) or H is not None and (H.shape != shape or H.dtype != dtype):
            raise ValueError("R and H have to be of X's shape and type")
        ldx = _row_stride(X, "X")
        ldr = ldh = cols
        if R is None:
            if H is not None and H.data_ptr() != X.data_ptr():
                raise ValueError("without R the stream is X itself")
            H = X
        else:
            ldr = _row_stride(R, "R")
            if H is None:
                H = _empty_like(X)
            else:
                ldh = _row_stride(H, "H")
        Y = _empty_like(X) if y else None
        q = s = mean = rstd = None
        ldq = lds = 0
        if e4m3:
            # (rows of many an odd number of blocks apart: they spread over the channels of the L2; a few next to one another: no view to be made)
            blocks = (cols + 127) // 128
            ldq, lds = (blocks if rows <= 16 else blocks | 1) * 128, (blocks + 3) // 4 * 4
            q, s = X.new_empty((rows, ldq), dtype=_E4M3), X.new_empty((rows, lds), dtype=torch.uint8)
            if ldq != cols:
                q = q[:, :cols]
            if lds != blocks:
                s = s[:, :blocks]
        if stats:
            mean = None if rms else X.new_empty(rows, dtype=torch.float32)
            rstd = X.new_empty(rows, dtype=torch.float32)
        st = self.lib.slim_add_norm(self.ctx, X.data_ptr(), None if R is None else R.data_ptr(), _dtype(X), rows, cols, ldx, ldr, w.data_ptr(),
                                    None if b is None else b.data_ptr(), _dtype(w), eps, rms, H.data_ptr(), ldh, None if Y is None else Y.data_ptr(),
                                    cols, None if q is None else q.data_ptr(), ldq, None if s is None else s.data_ptr(), lds,
                                    None if mean is None else mean.data_ptr(), None if rstd is None else rstd.data_ptr())
        if st:
            self._check(st)
        return AddNorm(H, Y, q, s, mean, rstd)

    def add_norm_backward(self, dY: torch.Tensor, dH: Optional[torch.Tensor], H: torch.Tensor, w: torch.Tensor, mean: Optional[torch.Tensor],
                          rstd: torch.Tensor, bias: bool = False):
        """(dX, dw, db): the gradient of X and of R alike, of weight and bias, from those of Y and, past the norm, of H (None: none); db is None
        without `bias`."""
        self._ready(dY, dH, H, w, mean, rstd)
        rows, cols = self._norm_shape(H, w, None)
        for v in (dY, dH):
            if v is not None and (v.shape != H.shape or v.dtype != H.dtype):
                raise ValueError("dY and dH have to be of H's shape and type")
        for v in (mean, rstd):
            if v is not None and (v.dtype != torch.float32 or v.shape != (rows,) or not v.is_contiguous()):
                raise ValueError("mean and rstd have to be float32 vectors of H's rows")
        dX, dw = _empty_like(H), torch.empty_like(w)
        db = torch.empty_like(w) if bias else None
        st = self.lib.slim_add_norm_backward(self.ctx, dY.data_ptr(), None if dH is None else dH.data_ptr(), H.data_ptr(), _dtype(H), rows, cols,
                                             _row_stride(dY, "dY"), 0 if dH is None else _row_stride(dH, "dH"), _row_stride(H, "H"), w.data_ptr(),
                                             _dtype(w), None if mean is None else mean.data_ptr(), rstd.data_ptr(), dX.data_ptr(), cols,
                                             dw.data_ptr(), None if db is None else db.data_ptr())
        if st:
            self._check(st)
        return dX, dw, db

    def grad_norm(self, tensors: Sequence[torch.Tensor]) -> torch.Tensor:
        """The norm of all of the tensors together: one float32 number on the device.  Records no graph: tensors that require a gradient are
        refused outside torch.no_grad()."""
        tensors = list(tensors)
        _no_graph(*tensors)
        self._ready(*tensors)
        flat = _tensor_list(tensors, "tensors")
        norm = torch.empty((), dtype=torch.float32, device=self.stream.device)
        st = self.lib.slim_grad_norm(self.ctx, _address(flat), len(tensors), norm.data_ptr())
        if st:
            self._check(st)
        return norm

    def clip_gradients(self, tensors: Sequence[torch.Tensor], limit: float, out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
        """Scales the tensors by min(1, limit / norm), in place or into `out` (tensors of their shapes and types, which do not overlap them or one
        another); returns their norm before that, one float32 number on the device.  A norm that is not finite leaves the values as they are.
        Records no graph, as grad_norm."""
        tensors = list(tensors)
        _no_graph(*tensors)
        if out is not None:
            out = list(out)
            _no_graph(*out)
            self._ready(*out)
        self._ready(*tensors)
        into = None
        if out is not None:
            if len(out) != len(tensors):
                raise ValueError("out has to hold as many tensors")
            into, flat = _tensor_list(out, "out"), _tensor_list(tensors, "tensors")
            for o, t in zip(out, tensors):
                if o.shape != t.shape or o.dtype != t.dtype:
                    raise ValueError("out has to hold tensors of the same shapes and types")
            if into[1::5] != flat[1::5]:
                # (of a tensor and its output one is contiguous, described as one row, and the other is not: both by their rows)
                into, flat = _tensor_rows(out, "out"), _tensor_rows(tensors, "tensors")
        else:
            flat = _tensor_list(tensors, "tensors")
        norm = torch.empty((), dtype=torch.float32, device=self.stream.device)
        st = self.lib.slim_clip_gradients(self.ctx, _address(flat), None if into is None else _address(into), len(tensors), limit, norm.data_ptr())
        if st:
            self._check(st)
        return norm

    @staticmethod
    def _norm_shape(X, w, b):
        if X.dim() != 2 or w.shape != X.shape[1:] or b is not None and (b.shape != w.shape or b.dtype != w.dtype):
            raise ValueError("X has to be a matrix, w and b vectors of its columns and of one type")
        if not w.is_contiguous() or b is not None and not b.is_contiguous():
            raise ValueError("w and b have to be contiguous")
        return X.shape

    def layer_norm_backward(self, dY: torch.Tensor, X: torch.Tensor, w: torch.Tensor, mean: Optional[torch.Tensor], rstd: torch.Tensor,
                            bias: bool = False):
        """(dX, dw, db) from the gradient of the outputs and the statistics of layer_norm; db is None without `bias`."""
        self._ready(dY, X, w, mean, rstd)
        rows, cols = self._norm_shape(X, w, None)
        if dY.shape != X.shape or dY.dtype != X.dtype:
            raise ValueError("dY has to be of X's shape and type")
        for v in (mean, rstd):
            if v is not None and (v.dtype != torch.float32 or v.shape != (rows,) or not v.is_contiguous()):
                raise ValueError("mean and rstd have to be float32 vectors of X's rows")
        dX, dw = _empty_like(X), torch.empty_like(w)
        db = torch.empty_like(w) if bias else None
        st = self.lib.slim_layer_norm_backward(self.ctx, dY.data_ptr(), X.data_ptr(), _dtype(X), rows, cols, _row_stride(dY, "dY"),
                                               _row_stride(X, "X"), w.data_ptr(), _dtype(w), None if mean is None else mean.data_ptr(),
                                               rstd.data_ptr(), dX.data_ptr(), cols, dw.data_ptr(), None if db is None else db.data_ptr())
        if st:
            self._check(st)
        return dX, dw, db

    def _distill_args(self, S, index, teacher, tau, lse):
        if S.dim() != 2 or index.dim() != 2 or index.shape != teacher.shape or index.shape[0] != S.shape[0]:
            raise ValueError("S has to be (rows, V), index and teacher (rows, K)")
        if index.dtype not in (torch.int64, torch.int32):
            raise ValueError("index has to be int64 or int32")
        rows, V = S.shape
        ldk = _row_stride(index, "index")
        if _row_stride(teacher, "teacher") != ldk:
            raise ValueError("index and teacher have to have one row stride")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (rows,) or not lse.is_contiguous()):
            raise ValueError("lse has to be a float32 vector of the rows")
        return (self.ctx, S.data_ptr(), _dtype(S), rows, V, _row_stride(S, "S"), index.data_ptr(), int(index.dtype == torch.int64),
                teacher.data_ptr(), _dtype(teacher), index.shape[1], ldk, None if lse is None else lse.data_ptr(), tau)

    def distill_loss(self, S: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, tau: float = 1.0, lse: Optional[torch.Tensor] = None):
        """loss float32 (rows,): the divergence of softmax(S / tau) from the teacher's top logits (rows, K) of the classes `index`.  Records no
        graph: S that requires a gradient is refused outside torch.no_grad() (distill_loss_grad gives it)."""
        _no_graph(S, teacher)
        self._ready(S, index, teacher, lse)
        args = self._distill_args(S, index, teacher, tau, lse)
        loss = S.new_empty(args[3], dtype=torch.float32)
        st = self.lib.slim_distill_loss(*args, loss.data_ptr())
        if st:
            self._check(st)
        return loss

    def distill_loss_grad(self, S: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, dloss: torch.Tensor, tau: float = 1.0,
                          lse: Optional[torch.Tensor] = None, dS: Optional[torch.Tensor] = None):
        """(loss, dS) with dS (rows, V) of S's type the gradient of sum(dloss * loss); dS may be given, S itself among others."""
        self._ready(S, index, teacher, dloss, lse, dS)
        args = self._distill_args(S, index, teacher, tau, lse)
        if dloss.dtype != torch.float32 or dloss.shape != (S.shape[0],) or not dloss.is_contiguous():
            raise ValueError("dloss has to be a float32 vector of the rows")
        if dS is None:
            dS = _empty_like(S)
        elif dS.shape != S.shape or dS.dtype != S.dtype:
            raise ValueError("dS has to be of S's shape and type")
        loss = S.new_empty(args[3], dtype=torch.float32)
        st = self.lib.slim_distill_loss_grad(*args, dloss.data_ptr(), loss.data_ptr(), dS.data_ptr(), _row_stride(dS, "dS"))
        if st:
            self._check(st)
        return loss, dS

    def _head_shape(self, X, W, Ws, labels):
        ldq, lds = _stored_strides(W, Ws, "W")
        V, m = W.shape
        if X.dim() != 2 or X.shape[1] != m:
            raise ValueError("X has to be (t, %d), got %s" % (m, tuple(X.shape)))
        if labels.shape != X.shape[:1] or labels.dtype not in (torch.int64, torch.int32) or not labels.is_contiguous():
            raise ValueError("labels have to be a contiguous int64 or int32 vector of the tokens")
        return V, m, X.shape[0], ldq, lds

    def head_loss(self, X: torch.Tensor, W: torch.Tensor, Ws: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        """loss float32 (t,): the cross entropy of the labels (t,) in the softmax of fp8_linear(X, W, Ws), whose outputs are not kept; 0 for a label
        that is no class, -100 say.  Records no graph: X that requires a gradient is refused outside torch.no_grad() (head_loss_grad gives it)."""
        _no_graph(X, W)
        self._ready(X, W, Ws, labels)
        V, m, t, ldq, lds = self._head_shape(X, W, Ws, labels)
        loss = X.new_empty(t, dtype=torch.float32)
        st = self.lib.slim_head_loss(self.ctx, X.data_ptr(), _dtype(X), t, _row_stride(X, "X"), W.data_ptr(), ldq, Ws.data_ptr(), lds, V, m,
                                     labels.data_ptr(), int(labels.dtype == torch.int64), loss.data_ptr())
        if st:
            self._check(st)
        return loss

    def head_loss_grad(self, X: torch.Tensor, W: torch.Tensor, Ws: torch.Tensor, Wt: Optional[torch.Tensor], Wts: Optional[torch.Tensor],
                       labels: torch.Tensor, dloss: torch.Tensor, dw_dtype: Optional[torch.dtype] = None, dx: bool = True, dw: bool = True):
        """(loss, dX (t, m), dW (V, m)): head_loss and the gradients of sum(dloss * loss); dw_dtype: of dW (default: X's).  Without `dx` Wt and Wts may be
        None; the gradient that is not wanted is None.  The workspace keeps up to 64 Mi of the t x V outputs in between, 256 MB."""
        self._ready(X, W, Ws, Wt, Wts, labels, dloss)
        if not (dx or dw):
            raise ValueError("neither gradient is wanted")
        V, m, t, ldq, lds = self._head_shape(X, W, Ws, labels)
        if dloss.dtype != torch.float32 or dloss.shape != (t,) or not dloss.is_contiguous():
            raise ValueError("dloss has to be a float32 vector of the tokens")
        ldqt = ldst = 0
        if dx:
            if Wt is None or Wts is None or Wt.shape != (m, V):
                raise ValueError("dX needs the stored weights of W^T, (%d, %d)" % (m, V))
            ldqt, ldst = _stored_strides(Wt, Wts, "Wt")
        loss = X.new_empty(t, dtype=torch.float32)
        dX = X.new_empty((t, m)) if dx else None
        dW = X.new_empty((V, m), dtype=dw_dtype) if dw else None
        st = self.lib.slim_head_loss_grad(self.ctx, X.data_ptr(), _dtype(X), t, _row_stride(X, "X"), W.data_ptr(), ldq, Ws.data_ptr(), lds,
                                          Wt.data_ptr() if dx else None, ldqt, Wts.data_ptr() if dx else None, ldst, V, m, labels.data_ptr(),
                                          int(labels.dtype == torch.int64), dloss.data_ptr(), loss.data_ptr(), dX.data_ptr() if dx else None, m,
                                          dW.data_ptr() if dw else None, _dtype(dW) if dw else F32, m)
        if st:
            self._check(st)
        return loss, dX, dW

    # ---- measurement aid
    def profile_enable(self, on: bool = True):
        self._check(self.lib.slim_profile_enable(self.ctx, 1 if on else 0))

    def profile_reset(self):
        self._check(self.lib.slim_profile_reset(self.ctx))

    def profile_collect(self):
        """Returns {kernel name: (total_ms, launches)} accumulated since the last reset."""
        n = self.lib.slim_profile_collect(self.ctx)
        out = {}
        for i in range(n):
            name = ctypes.c_char_p()
            ms = ctypes.c_double()
            cnt = ctypes.c_int()
            self._check(self.lib.slim_profile_entry(self.ctx, i, ctypes.byref(name), ctypes.byref(ms), ctypes.byref(cnt)))
            out[name.value.decode()] = (ms.value, cnt.value)
        return out

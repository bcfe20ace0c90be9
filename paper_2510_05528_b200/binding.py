"""ctypes binding of libarmor (see include/armor.h).  Argument marshalling only: every step of the
method runs in the library's CUDA kernels.  PyTorch supplies device memory and streams.

The module-level functions carry the names of the C entry points and take torch CUDA tensors.
``ArmorContext`` bundles a configuration with its workspace.  There is no CPU path: if the shared
library is missing, or a tensor is not on a CUDA device, the call raises."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libarmor.so")

H_FULL, H_DIAG = 0, 1
SELECT_L1_RANDOM, SELECT_L1_GREEDY, SELECT_UNIFORM_RANDOM, SELECT_L2_RANDOM = 0, 1, 2, 3
S_EXACT, S_BETA = 0, 1
AB_EXACT, AB_GD, AB_ADAM = 0, 1, 2
PREC_FP32X3, PREC_TF32, PREC_SIMT, PREC_FP16X3 = 0, 1, 2, 3
PHASE_A, PHASE_B, PHASE_S, PHASE_MASK = 1, 2, 4, 8
DTYPE_F32, DTYPE_BF16, DTYPE_BF16_SPARSE, DTYPE_F16, DTYPE_I8 = 0, 1, 2, 3, 4
# element types of the 8-bit products and of the norms
ROW_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}

EXPORTS = ["armor_workspace_bytes", "armor_create", "armor_destroy", "armor_gram", "armor_init",
           "armor_bcd_step", "armor_proxy_loss", "armor_apply", "armor_packed_core_bytes", "armor_pack_core", "armor_apply_packed",
           "armor_packed_layer_bytes", "armor_pack_layer", "armor_apply_layer",
           "armor_quantize_rows", "armor_linear_i8", "armor_packed_layer_i8_bytes", "armor_pack_layer_i8", "armor_apply_layer_i8",
           "armor_block_norm", "armor_block_norm_backward", "armor_kv_write", "armor_kv_read", "armor_kv_attend",
           "armor_get_device_status",
           "armor_status_string", "armor_launch_count", "armor_gemm_timing_enable", "armor_gemm_timing",
           "armor_normalize_noalloc", "armor_block_product", "armor_block_product_dual", "armor_block_product_two_sided", "armor_selftest_wait_timeout", "armor_kernel_timing_enable", "armor_use_graphs", "armor_fuse_grams",
           "armor_kernel_timing"]


class ArmorError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


class armor_config(C.Structure):
    _fields_ = [("d_out", C.c_int64), ("d_in", C.c_int64), ("d_block", C.c_int32), ("n_keep", C.c_int32),
                ("m_group", C.c_int32), ("h_mode", C.c_int32), ("select_mode", C.c_int32),
                ("s_step", C.c_int32), ("precision", C.c_int32), ("normalize", C.c_int32),
                ("phases", C.c_int32), ("ab_step", C.c_int32), ("mask_sweeps", C.c_int32), ("mask_groups", C.c_int32), ("ridge", C.c_float), ("adam_lr", C.c_float),
                ("adam_beta1", C.c_float), ("adam_beta2", C.c_float), ("adam_eps", C.c_float), ("seed", C.c_uint64)]


def _struct(name, *fields):
    return type(name, (C.Structure,), {"_fields_": list(fields)})


def _rows_of(*names):
    return [f for n in names for f in ((n, C.c_void_p), ("ld" + n, C.c_int64))]


_gate_sizes = [("ld_gate", C.c_int64), ("rows_per_gate", C.c_int64), ("n_gates", C.c_int64)]
_norm_tail = [("stream_dtype", C.c_int32), ("branch_dtype", C.c_int32), ("post", C.c_int32), ("pre", C.c_int32),
              ("residual_scale", C.c_float), ("eps", C.c_float)]
armor_block_norm_args = _struct(
    "armor_block_norm_args", ("n_rows", C.c_int64), ("d", C.c_int64), *_rows_of("x", "y", "h", "n", "q"), ("q_scale", C.c_void_p),
    ("w_post", C.c_void_p), ("w_pre", C.c_void_p), ("gate", C.c_void_p), *_gate_sizes, *_norm_tail)
armor_block_norm_grad_args = _struct(
    "armor_block_norm_grad_args", ("n_rows", C.c_int64), ("d", C.c_int64), *_rows_of("h", "y", "dh", "dn", "dx", "dy"),
    ("w_post", C.c_void_p), ("w_pre", C.c_void_p), ("gate", C.c_void_p), *_gate_sizes,
    ("dw_post", C.c_void_p), ("dw_pre", C.c_void_p), ("dgate", C.c_void_p), *_norm_tail)

armor_kv_cache = _struct(
    "armor_kv_cache", *[(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")],
    *[(n, C.c_int64) for n in ("n_pages", "page_size", "kv_heads", "head_dim", "page_stride", "head_stride", "slot_stride",
                               "scale_page_stride", "scale_head_stride", "scale_slot_stride")])
armor_kv_batch = _struct("armor_kv_batch", ("n_seqs", C.c_int64), ("max_pages", C.c_int64), ("ld_pages", C.c_int64),
                         ("pages", C.c_void_p), ("lengths", C.c_void_p), ("starts", C.c_void_p))
armor_kv_rows = _struct("armor_kv_rows", ("k", C.c_void_p), ("v", C.c_void_p), ("n_rows", C.c_int64),
                        *[(n, C.c_int64) for n in ("k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")], ("dtype", C.c_int32))
armor_kv_attend_args = _struct(
    "armor_kv_attend_args", ("q", C.c_void_p), ("o", C.c_void_p),
    *[(n, C.c_int64) for n in ("n_rows", "heads", "q_row_stride", "q_head_stride", "o_row_stride", "o_head_stride", "window", "max_chunk")],
    ("scale", C.c_float), ("dtype", C.c_int32))

STATS_DTYPE = np.dtype([("loss_start", "<f8"), ("loss_A", "<f8"), ("loss_B", "<f8"), ("loss_S", "<f8"),
                        ("loss_mask", "<f8"), ("delta_L_mask", "<f8"), ("tau_B", "<f4"), ("tau_S", "<f4"),
                        ("groups_changed", "<i4"), ("mask_accepted", "<i4"), ("chol_failed", "<i4"),
                        ("reserved", "<i4")])

_lib = None


def lib() -> C.CDLL:
    """Loads libarmor.so on first use; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not found: build it with `python -m paper_2510_05528_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.armor_workspace_bytes.argtypes = [C.POINTER(armor_config), C.POINTER(C.c_size_t)]
        L.armor_create.argtypes = [C.POINTER(vp), C.POINTER(armor_config), vp, C.c_size_t]
        L.armor_destroy.argtypes = [vp]
        L.armor_gram.argtypes = [vp, vp, i32, i64, i64, vp, vp]
        L.armor_init.argtypes = [vp] + [vp] * 9 + [vp]
        L.armor_bcd_step.argtypes = [vp] + [vp] * 6 + [i64, i32, vp, vp]
        L.armor_proxy_loss.argtypes = [vp] + [vp] * 6 + [vp]
        L.armor_apply.argtypes = [vp] + [vp] * 8 + [i32, i64, vp]
        L.armor_packed_core_bytes.argtypes = [C.POINTER(armor_config), C.POINTER(C.c_size_t)]
        L.armor_pack_core.argtypes = [vp, vp, vp, vp, vp]
        L.armor_apply_packed.argtypes = [vp] + [vp] * 7 + [i64, vp]
        L.armor_packed_layer_bytes.argtypes = [C.POINTER(armor_config), C.POINTER(C.c_size_t)]
        L.armor_pack_layer.argtypes = [vp] + [vp] * 7 + [vp]
        L.armor_apply_layer.argtypes = [vp, vp, vp, vp, i64, vp]
        L.armor_quantize_rows.argtypes = [vp, vp, i32, i64, i64, i64, vp, i64, vp, vp]
        L.armor_linear_i8.argtypes = [vp, vp, i32, i64, vp, vp, i64, vp, vp, vp, i32, i64, i64, i64, i64, vp]
        L.armor_packed_layer_i8_bytes.argtypes = [C.POINTER(armor_config), C.POINTER(C.c_size_t)]
        L.armor_pack_layer_i8.argtypes = [vp] + [vp] * 7 + [vp]
        L.armor_apply_layer_i8.argtypes = [vp, vp, vp, vp, i64, vp]
        L.armor_block_norm.argtypes = [vp, C.POINTER(armor_block_norm_args), vp]
        L.armor_block_norm_backward.argtypes = [vp, C.POINTER(armor_block_norm_grad_args), vp]
        for f, g in (("write", armor_kv_rows), ("read", armor_kv_rows), ("attend", armor_kv_attend_args)):
            getattr(L, "armor_kv_" + f).argtypes = [vp, C.POINTER(armor_kv_cache), C.POINTER(armor_kv_batch), C.POINTER(g), vp]
        L.armor_get_device_status.argtypes = [vp, C.POINTER(i32), i32]
        L.armor_status_string.argtypes = [C.c_int]
        L.armor_status_string.restype = C.c_char_p
        L.armor_launch_count.argtypes = [vp]
        L.armor_launch_count.restype = i64
        L.armor_normalize_noalloc.argtypes = [vp, i64, i64, vp, vp, vp, vp]
        L.armor_block_product.argtypes = [vp, i32, i32, vp, vp, vp, i64, i64, C.c_float, vp, C.c_float, i32, vp]
        L.armor_block_product_dual.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp]
        L.armor_block_product_two_sided.argtypes = [vp, vp, i32, vp, vp, i32, vp, C.c_float, i32, vp]
        L.armor_gemm_timing_enable.argtypes = [vp, i32]
        L.armor_gemm_timing.argtypes = [vp, C.POINTER(i64), C.POINTER(C.c_double), C.POINTER(C.c_double)]
        L.armor_kernel_timing_enable.argtypes = [vp, i32]
        L.armor_use_graphs.argtypes = [vp, i32]
        L.armor_fuse_grams.argtypes = [vp, i32]
        L.armor_kernel_timing.argtypes = [vp, i32, C.POINTER(i64), C.POINTER(C.c_double), C.POINTER(C.c_double)]
        L.armor_selftest_wait_timeout.argtypes = [vp, i64, vp, vp]
        for name in EXPORTS:
            if name not in ("armor_status_string", "armor_launch_count"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().armor_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise ArmorError(code, where)


def _ptr(t: torch.Tensor | None, dtype=None, name: str = "tensor") -> int | None:
    # (a plain address, which ctypes converts as it calls: a pointer object each cost 0.2 us of a call that takes 12)
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (this library has no CPU path)")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream() -> int:
    # the raw handle of torch.cuda.current_stream(), without building a Stream object for it (2 us of a 17 us call); the tensors of
    # the call exist, so CUDA is initialised
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def make_config(d_out, d_in, d_block, *, n_keep=2, m_group=4, h_mode=H_FULL, select_mode=SELECT_L1_RANDOM,
                s_step=S_EXACT, precision=PREC_FP16X3, normalize=0, phases=0, ab_step=AB_EXACT, mask_sweeps=1, mask_groups=1, ridge=1e-6,
                adam_lr=0.0, adam_beta1=0.0, adam_beta2=0.0, adam_eps=0.0, seed=0) -> armor_config:
    return armor_config(d_out, d_in, d_block, n_keep, m_group, h_mode, select_mode, s_step, precision,
                        int(normalize), phases, ab_step, mask_sweeps, mask_groups, ridge, adam_lr, adam_beta1, adam_beta2, adam_eps, seed)


# ---------------------------------------------------------------- C entry points, same names
def armor_workspace_bytes(cfg: armor_config) -> int:
    n = C.c_size_t(0)
    _check(lib().armor_workspace_bytes(C.byref(cfg), C.byref(n)), "armor_workspace_bytes")
    return int(n.value)


def armor_create(cfg: armor_config, workspace: torch.Tensor) -> C.c_void_p:
    ctx = C.c_void_p(0)
    _check(lib().armor_create(C.byref(ctx), C.byref(cfg), _ptr(workspace, name="workspace"),
                              workspace.numel() * workspace.element_size()), "armor_create")
    return ctx


def armor_destroy(ctx) -> None:
    _check(lib().armor_destroy(ctx), "armor_destroy")


def armor_gram(ctx, X: torch.Tensor, H: torch.Tensor) -> None:
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be [n_rows, d_in] with unit column stride")
    if not X.is_cuda or X.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("X must be a float32 or bfloat16 CUDA tensor (this library has no CPU path)")
    ldx = X.stride(0) if X.shape[0] > 1 else X.shape[1]
    _check(lib().armor_gram(ctx, C.c_void_p(X.data_ptr()), DTYPE_BF16 if X.dtype == torch.bfloat16 else DTYPE_F32,
                            X.shape[0], ldx,
                            _ptr(H, torch.float32, "H"), _stream()), "armor_gram")


def armor_init(ctx, W, H, Wbar, r1, r2, A, B, S, M) -> None:
    f = torch.float32
    _check(lib().armor_init(ctx, _ptr(W, f, "W"), _ptr(H, f, "H"), _ptr(Wbar, f, "Wbar"), _ptr(r1, f, "r1"),
                            _ptr(r2, f, "r2"), _ptr(A, f, "A"), _ptr(B, f, "B"), _ptr(S, f, "S"),
                            _ptr(M, torch.uint8, "M"), _stream()), "armor_init")


def armor_bcd_step(ctx, Wbar, H, A, B, S, M, t_first: int, n_iters: int, stats: torch.Tensor | None) -> None:
    f = torch.float32
    _check(lib().armor_bcd_step(ctx, _ptr(Wbar, f, "Wbar"), _ptr(H, f, "H"), _ptr(A, f, "A"), _ptr(B, f, "B"),
                                _ptr(S, f, "S"), _ptr(M, torch.uint8, "M"), int(t_first), int(n_iters),
                                _ptr(stats, torch.uint8, "stats"), _stream()), "armor_bcd_step")


def armor_proxy_loss(ctx, Wbar, H, A, B, S, loss: torch.Tensor) -> None:
    f = torch.float32
    _check(lib().armor_proxy_loss(ctx, _ptr(Wbar, f, "Wbar"), _ptr(H, f, "H"), _ptr(A, f, "A"), _ptr(B, f, "B"),
                                  _ptr(S, f, "S"), _ptr(loss, torch.float64, "loss"), _stream()), "armor_proxy_loss")


def armor_apply(ctx, A, B, S, M, r1, r2, x, y, sparse: bool = False) -> None:
    f = torch.float32
    if x.dtype != y.dtype or x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("x and y must both be float32 or both be bfloat16")
    dt = DTYPE_BF16 if x.dtype == torch.bfloat16 else DTYPE_F32
    if sparse:
        if dt != DTYPE_BF16:
            raise ValueError("the sparse tensor-core forward takes bf16 x and y")
        dt = DTYPE_BF16_SPARSE
    _check(lib().armor_apply(ctx, _ptr(A, f, "A"), _ptr(B, f, "B"), _ptr(S, f, "S"), _ptr(M, torch.uint8, "M"),
                             _ptr(r1, f, "r1"), _ptr(r2, f, "r2"), _ptr(x, x.dtype, "x"), _ptr(y, y.dtype, "y"), dt,
                             x.shape[0], _stream()), "armor_apply")


def armor_packed_core_bytes(cfg: armor_config) -> int:
    n = C.c_size_t(0)
    _check(lib().armor_packed_core_bytes(C.byref(cfg), C.byref(n)), "armor_packed_core_bytes")
    return int(n.value)


def armor_pack_core(ctx, S, M, packed) -> None:
    _check(lib().armor_pack_core(ctx, _ptr(S, torch.float32, "S"), _ptr(M, torch.uint8, "M"),
                                 _ptr(packed, torch.uint8, "packed"), _stream()), "armor_pack_core")


def armor_apply_packed(ctx, A, B, packed, r1, r2, x, y) -> None:
    f = torch.float32
    if x.dtype != torch.bfloat16 or y.dtype != torch.bfloat16:
        raise ValueError("the packed forward takes bf16 x and y")
    _check(lib().armor_apply_packed(ctx, _ptr(A, f, "A"), _ptr(B, f, "B"), _ptr(packed, torch.uint8, "packed"),
                                    _ptr(r1, f, "r1"), _ptr(r2, f, "r2"), _ptr(x, x.dtype, "x"), _ptr(y, y.dtype, "y"),
                                    x.shape[0], _stream()), "armor_apply_packed")


def armor_packed_layer_bytes(cfg: armor_config) -> int:
    n = C.c_size_t(0)
    _check(lib().armor_packed_layer_bytes(C.byref(cfg), C.byref(n)), "armor_packed_layer_bytes")
    return int(n.value)


def armor_pack_layer(ctx, A, B, S, M, r1, r2, packed) -> None:
    f = torch.float32
    _check(lib().armor_pack_layer(ctx, _ptr(A, f, "A"), _ptr(B, f, "B"), _ptr(S, f, "S"), _ptr(M, torch.uint8, "M"),
                                  _ptr(r1, f, "r1"), _ptr(r2, f, "r2"), _ptr(packed, torch.uint8, "packed"), _stream()),
           "armor_pack_layer")


def armor_apply_layer(ctx, packed, x, y) -> None:
    bf16 = torch.bfloat16
    if x.dtype is not bf16 or y.dtype is not bf16:
        raise ValueError("the packed layer takes bf16 x and y")
    code = lib().armor_apply_layer(ctx, _ptr(packed, torch.uint8, "packed"), _ptr(x, None, "x"), _ptr(y, None, "y"), x.shape[0], _stream())
    if code:
        _check(code, "armor_apply_layer")


def _row_ptr(t: torch.Tensor, dtype, name: str, cols: int | None = None) -> tuple[int, int]:
    """(address, leading dimension) of rows [n, cols] with unit column stride."""
    if t.dtype is dtype and t.is_cuda and t.dim() == 2 and t.is_contiguous():      # (the common case first: a call takes microseconds)
        c = t.size(1)
        if cols is None or c == cols:
            ld = t.stride(0)                         # (of a single row it may be anything)
            return t.data_ptr(), ld if ld > c else c
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (this library has no CPU path)")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} must be [rows, {'cols' if cols is None else cols}], got {list(shape)}")
    n, c = shape
    ld, one = t.stride()
    if n <= 1 and ld < c:                            # a single row's stride says nothing
        ld = c
    if (one != 1 and c > 1) or ld < c:
        raise ValueError(f"{name} must have unit column stride and rows that do not overlap")
    return t.data_ptr(), ld


def _rows_at(t: torch.Tensor, dtype, cols: int | None, name: str, here: int) -> tuple[int, int, int]:
    """(address, leading dimension, rows) of [rows, cols] on device `here`.  The common case in as few steps as there are: a small call
    takes ten microseconds, most of them its checks."""
    if t.dtype is dtype and t.get_device() == here and t.is_contiguous():
        shape = t.shape
        if len(shape) == 2 and (cols is None or shape[1] == cols):
            n, c = shape
            return t.data_ptr(), (c if n > 1 else max(c, t.stride(0))), n
    if t.is_cuda and t.get_device() != here:
        raise ValueError(f"{name} must be on cuda:{here}, the call's device, not on {t.device}")
    p, ld = _row_ptr(t, dtype, name, cols)
    return p, ld, t.shape[0]


def _cuda_index(t: torch.Tensor, name: str) -> int:
    """The device of a call, which enqueues on that device's current stream."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    here = t.get_device()
    if torch._C._cuda_getDevice() != here:
        raise ValueError(f"{t.device}, which holds {name}, must be the current device")
    return here


def _vector_at(t: torch.Tensor, n: int, name: str, here: int) -> int:
    """The address of n contiguous floats on device `here`."""
    if t.dtype is torch.float32 and t.get_device() == here and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    if t.is_cuda and t.get_device() != here:
        raise ValueError(f"{name} must be on cuda:{here}, the call's device, not on {t.device}")
    _ptr(t, torch.float32, name)
    raise ValueError(f"{name} must have {n} elements, got {t.numel()}")


def _row_dtype(t: torch.Tensor, name: str) -> int:
    code = ROW_DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def armor_quantize_rows(ctx, x, q, scale) -> None:
    """q [n, c] int8 (rows on 16-byte boundaries) and scale [n] fp32 of x [n, c] (see armor.h)."""
    code = _row_dtype(x, "x")
    here = _cuda_index(x, "x")
    xp, ldx, n = _rows_at(x, x.dtype, None, "x", here)
    c = x.size(1)
    qp, ldq, n_q = _rows_at(q, torch.int8, c, "q", here)
    if n_q != n:
        raise ValueError(f"q must have the {n} rows of x")
    _check(lib().armor_quantize_rows(ctx, xp, code, ldx, n, c, qp, ldq, _vector_at(scale, n, "scale", here), _stream()),
           "armor_quantize_rows")


def armor_linear_i8(ctx, x, x_scale, wq, w_scale, bias, y) -> None:
    """y [n, n_out] = x [n, n_in] wq^T with the scales of both (see armor.h); x_scale None: x is rounded on the way."""
    code = DTYPE_I8 if x.dtype is torch.int8 else _row_dtype(x, "x")
    here = _cuda_index(x, "x")
    xp, ldx, n = _rows_at(x, x.dtype, None, "x", here)
    n_in = x.size(1)
    wp, ldw, n_out = _rows_at(wq, torch.int8, n_in, "wq", here)
    yp, ldy, n_y = _rows_at(y, y.dtype, n_out, "y", here)
    if n_y != n:
        raise ValueError(f"y must have the {n} rows of x")
    code = lib().armor_linear_i8(ctx, xp, code, ldx, None if x_scale is None else _vector_at(x_scale, n, "x_scale", here), wp, ldw,
                                 _vector_at(w_scale, n_out, "w_scale", here), None if bias is None else _vector_at(bias, n_out, "bias", here),
                                 yp, _row_dtype(y, "y"), ldy, n, n_out, n_in, _stream())
    if code:
        _check(code, "armor_linear_i8")


def armor_packed_layer_i8_bytes(cfg: armor_config) -> int:
    n = C.c_size_t(0)
    _check(lib().armor_packed_layer_i8_bytes(C.byref(cfg), C.byref(n)), "armor_packed_layer_i8_bytes")
    return int(n.value)


def armor_pack_layer_i8(ctx, A, B, S, M, r1, r2, packed) -> None:
    f = torch.float32
    _check(lib().armor_pack_layer_i8(ctx, _ptr(A, f, "A"), _ptr(B, f, "B"), _ptr(S, f, "S"), _ptr(M, torch.uint8, "M"),
                                     _ptr(r1, f, "r1"), _ptr(r2, f, "r2"), _ptr(packed, torch.uint8, "packed"), _stream()),
           "armor_pack_layer_i8")


def armor_apply_layer_i8(ctx, packed, x, y) -> None:
    bf16 = torch.bfloat16
    if x.dtype is not bf16 or y.dtype is not bf16:
        raise ValueError("the packed layer takes bf16 x and y")
    here = _cuda_index(x, "x")
    for t, name in ((packed, "packed"), (y, "y")):
        if t.is_cuda and t.get_device() != here:
            raise ValueError(f"{name} must be on cuda:{here}, as x is, not on {t.device}")
    if x.dim() != 2 or y.dim() != 2 or y.size(0) != x.size(0):
        raise ValueError(f"x and y must be [tokens, d_in] and [tokens, d_out], got {list(x.shape)} and {list(y.shape)}")
    code = lib().armor_apply_layer_i8(ctx, _ptr(packed, torch.uint8, "packed"), _ptr(x, None, "x"), _ptr(y, None, "y"), x.shape[0], _stream())
    if code:
        _check(code, "armor_apply_layer_i8")


def _norm_params(a, d, n_rows, here, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps):
    """Fills what both directions of the norms share; returns the gate's rows."""
    a.n_rows = n_rows
    a.d = d
    if w_pre is not None:
        a.w_pre = _vector_at(w_pre, d, "w_pre", here)
    if w_post is not None:
        a.w_post = _vector_at(w_post, d, "w_post", here)
    a.post = w_post is not None if post is None else post
    a.pre = pre
    a.residual_scale = residual_scale
    a.eps = eps
    if gate is None:
        return 0
    if gate.dim() == 1:
        gate = gate.unsqueeze(0)
    a.gate, a.ld_gate, n_gates = _rows_at(gate, torch.float32, d, "gate", here)
    if not rows_per_gate:
        if n_gates < 1 or n_rows % n_gates:
            raise ValueError(f"rows_per_gate must be given where {n_gates} gates do not divide {n_rows} rows")
        rows_per_gate = max(1, n_rows // n_gates)
    a.rows_per_gate = rows_per_gate
    a.n_gates = n_gates
    return n_gates


def _block_norm(ctx, here, x, y, h, n, q, q_scale, made, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps) -> None:
    # made: the outputs are this module's own, contiguous and of the right shape
    a = armor_block_norm_args()
    dt = x.dtype
    a.stream_dtype = code = _row_dtype(x, "x")
    a.x, a.ldx, rows = _rows_at(x, dt, None, "x", here)
    d = x.size(1)
    bt = dt
    if y is not None:
        bt = y.dtype
        a.y, a.ldy, n_y = _rows_at(y, bt, d, "y", here)
        if n_y != rows:
            raise ValueError(f"y must have the {rows} rows of x")
    elif n is not None:
        bt = n.dtype
    a.branch_dtype = code if bt is dt else _row_dtype(n if y is None else y, "y")
    if made:
        a.h = h.data_ptr()
        a.ldh = d
        if n is not None:
            a.n = n.data_ptr()
            a.ldn = d
        if q is not None:
            a.q, a.ldq, _ = _rows_at(q, torch.int8, d, "q", here)
    else:
        n_h = n_n = n_q = rows
        if h is not None:
            a.h, a.ldh, n_h = _rows_at(h, dt, d, "h", here)
        if n is not None:
            a.n, a.ldn, n_n = _rows_at(n, bt, d, "n", here)
        if q is not None:
            a.q, a.ldq, n_q = _rows_at(q, torch.int8, d, "q", here)
        if not n_h == n_n == n_q == rows:
            raise ValueError(f"h, n and q must have the {rows} rows of x")
    if q_scale is not None:
        a.q_scale = _vector_at(q_scale, rows, "q_scale", here)
    _norm_params(a, d, rows, here, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps)
    code = lib().armor_block_norm(ctx, a, _stream())
    if code:
        _check(code, "armor_block_norm")


def armor_block_norm(ctx, x, y, h, n, q, q_scale, *, gate=None, rows_per_gate=0, w_post=None, w_pre=None, post=None, pre=True,
                     residual_scale=1.0, eps=1e-6) -> None:
    """h and n (and n as int8 q with q_scale) of the residual stream x and a block's output y (see armor.h).  post: None means with
    w_post."""
    _block_norm(ctx, _cuda_index(x, "x"), x, y, h, n, q, q_scale, False, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps)


def _block_norm_backward(ctx, here, h, y, dh, dn, dx, dy, dw_post, dw_pre, dgate, made, gate, rows_per_gate, w_post, w_pre, post, pre,
                         residual_scale, eps) -> None:
    a = armor_block_norm_grad_args()
    stream = h if h is not None else (dh if dh is not None else dx)
    branch = y if y is not None else (dn if dn is not None else dy)
    one = stream if stream is not None else branch
    ts, tb = one.dtype, (branch if branch is not None else stream).dtype
    if one.dim() != 2:
        raise ValueError("h, y and their gradients must be [rows, cols]")
    rows, d = one.shape
    a.stream_dtype = _row_dtype(one, "h")
    a.branch_dtype = a.stream_dtype if tb is ts else _row_dtype(branch, "y")
    n_h = n_y = n_dh = n_dn = rows
    if h is not None:
        a.h, a.ldh, n_h = _rows_at(h, ts, d, "h", here)
    if y is not None:
        a.y, a.ldy, n_y = _rows_at(y, tb, d, "y", here)
    if dh is not None:
        a.dh, a.lddh, n_dh = _rows_at(dh, ts, d, "dh", here)
    if dn is not None:
        a.dn, a.lddn, n_dn = _rows_at(dn, tb, d, "dn", here)
    if not n_h == n_y == n_dh == n_dn == rows:
        raise ValueError("h, y, dh and dn must have as many rows")
    gates = _norm_params(a, d, rows, here, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps)
    if made:
        a.dx = dx.data_ptr()
        if dy is not None:
            a.dy = dy.data_ptr()
        a.lddx = a.lddy = d
        if dw_post is not None:
            a.dw_post = dw_post.data_ptr()
        if dw_pre is not None:
            a.dw_pre = dw_pre.data_ptr()
        if dgate is not None:
            a.dgate = dgate.data_ptr()
    else:
        n_dx = n_dy = rows
        if dx is not None:
            a.dx, a.lddx, n_dx = _rows_at(dx, ts, d, "dx", here)
        if dy is not None:
            a.dy, a.lddy, n_dy = _rows_at(dy, tb, d, "dy", here)
        if not n_dx == n_dy == rows:
            raise ValueError(f"dx and dy must have {rows} rows")
        for name, t, n in (("dw_post", dw_post, d), ("dw_pre", dw_pre, d), ("dgate", dgate, gates * d)):
            if t is not None:
                setattr(a, name, _vector_at(t, n, name, here))
    code = lib().armor_block_norm_backward(ctx, a, _stream())
    if code:
        _check(code, "armor_block_norm_backward")


def armor_block_norm_backward(ctx, h, y, dh, dn, dx, dy, dw_post, dw_pre, dgate, *, gate=None, rows_per_gate=0, w_post=None,
                              w_pre=None, post=None, pre=True, residual_scale=1.0, eps=1e-6) -> None:
    """The gradient of armor_block_norm (see armor.h)."""
    one = next((t for t in (h, dh, dx, y, dn, dy) if t is not None), None)
    if one is None:
        raise ValueError("h, dh, dx, y, dn and dy are all missing")
    _block_norm_backward(ctx, _cuda_index(one, "h, y and their gradients"), h, y, dh, dn, dx, dy, dw_post, dw_pre, dgate, False, gate, rows_per_gate, w_post, w_pre, post,
                         pre, residual_scale, eps)


class KvCache:
    """A paged cache of int8 keys and values with an fp32 scale for each row: k and v [n_pages, kv_heads, page_size, head_dim], k_scale
    and v_scale [n_pages, kv_heads, page_size], views in any order of the first three dimensions (k and v alike, k_scale and v_scale alike)
    whose rows start on 16-byte boundaries.  It keeps the tensors and their layout; what they hold may change from call to call."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        for name, t, dtype, dims in (("k", k, torch.int8, 4), ("v", v, torch.int8, 4), ("k_scale", k_scale, torch.float32, 3),
                                     ("v_scale", v_scale, torch.float32, 3)):
            if not t.is_cuda:
                raise ValueError(f"{name} must be a CUDA tensor (this library has no CPU path)")
            if t.device != k.device:
                raise ValueError(f"{name} must be on {k.device}, as k is, not on {t.device}")
            if t.dtype is not dtype or t.dim() != dims:
                raise ValueError(f"{name} must be {dtype} with {dims} dimensions, got {t.dtype} {list(t.shape)}")
            if t.shape != k.shape[:dims]:
                raise ValueError(f"{name} must be {list(k.shape[:dims])}, got {list(t.shape)}")
        if k.numel() == 0:
            raise ValueError("the cache must hold a page")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("the rows of k and v must be contiguous")
        steps, scale_steps = _steps(k), _steps(k_scale)
        if steps != _steps(v) or scale_steps != _steps(v_scale):
            raise ValueError("k and v, k_scale and v_scale must be laid out alike")
        if min(steps) < k.size(3) or min(scale_steps) < 1:
            raise ValueError("pages, heads and slots must not overlap")
        if any(n % 16 for n in (*steps, k.data_ptr(), v.data_ptr())):
            raise ValueError("rows of k and v must start on 16-byte boundaries")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.index = k.get_device()
        self.n_pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.args = armor_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.n_pages, self.page_size,
                                   self.kv_heads, self.head_dim, *steps, *scale_steps)


def _steps(t: torch.Tensor) -> list[int]:
    """Strides of pages, heads and slots; of a dimension of one entry, whose stride says nothing, a row's."""
    return [n if size > 1 else (t.size(3) if t.dim() == 4 else 1) for n, size in zip(t.stride()[:3], t.shape[:3])]


class KvBatch:
    """Sequences of a call on a cache (int32 tensors on its device): rows starts[b] .. starts[b + 1] - 1 of the packed arrays are the last
    positions of sequence b, which has lengths[b] and its pages, in order, in pages[b].  It keeps the tensors; what they hold may
    change from call to call, also under a captured one."""

    def __init__(self, pages: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor):
        for name, t, dims in (("pages", pages, 2), ("lengths", lengths, 1), ("starts", starts, 1)):
            if not t.is_cuda:
                raise ValueError(f"{name} must be a CUDA tensor (this library has no CPU path)")
            if t.device != pages.device:
                raise ValueError(f"{name} must be on {pages.device}, as pages is, not on {t.device}")
            if t.dtype is not torch.int32 or t.dim() != dims:
                raise ValueError(f"{name} must be int32 with {dims} dimensions, got {t.dtype} {list(t.shape)}")
        n, m = pages.shape
        if lengths.numel() != n or starts.numel() != n + 1:
            raise ValueError(f"{n} sequences have {n} lengths and {n + 1} starts, got {lengths.numel()} and {starts.numel()}")
        if not lengths.is_contiguous() or not starts.is_contiguous() or (m > 1 and pages.stride(1) != 1) or (n > 1 and pages.stride(0) < m):
            raise ValueError("lengths, starts and the rows of pages must be contiguous")
        self.pages, self.lengths, self.starts = pages, lengths, starts
        self.index = pages.get_device()
        self.n_seqs = n
        self.args = armor_kv_batch(n, m, pages.stride(0) if n > 1 else max(m, 1), pages.data_ptr(), lengths.data_ptr(), starts.data_ptr())


def _heads_at(t: torch.Tensor, dtype, rows: int | None, heads: int | None, dim: int, name: str, here: int) -> tuple[int, int, int]:
    """(address, stride of rows, stride of heads) of [rows, heads, dim] on device `here`."""
    if t.get_device() != here:
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor (this library has no CPU path)")
        raise ValueError(f"{name} must be on cuda:{here}, the call's device, not on {t.device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 3 or shape[2] != dim or (rows is not None and shape[0] != rows) or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {'heads' if heads is None else heads}, {dim}], got {list(shape)}")
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return t.data_ptr(), row if shape[0] > 1 else max(row, dim), head if shape[1] > 1 else max(head, dim)


def _kv_here(cache: KvCache, batch: KvBatch, here: int) -> None:
    if cache.index != here or batch.index != here:
        raise ValueError(f"the cache is on cuda:{cache.index}, the batch on cuda:{batch.index}, the call's device is cuda:{here}")


def _kv_rows(cache: KvCache, batch: KvBatch, k, v, here) -> armor_kv_rows:
    _kv_here(cache, batch, here)
    code = _row_dtype(k, "k")
    kp, kr, kh = _heads_at(k, k.dtype, None, cache.kv_heads, cache.head_dim, "k", here)
    vp, vr, vh = _heads_at(v, k.dtype, k.size(0), cache.kv_heads, cache.head_dim, "v", here)
    return armor_kv_rows(kp, vp, k.size(0), kr, kh, vr, vh, code)


def _kv_write(ctx, here, cache, batch, k, v) -> None:
    code = lib().armor_kv_write(ctx, cache.args, batch.args, _kv_rows(cache, batch, k, v, here), _stream())
    if code:
        _check(code, "armor_kv_write")


def _kv_read(ctx, cache, batch, rows) -> None:
    code = lib().armor_kv_read(ctx, cache.args, batch.args, rows, _stream())
    if code:
        _check(code, "armor_kv_read")


def armor_kv_write(ctx, cache: KvCache, batch: KvBatch, k, v) -> None:
    """The rows of k and v [rows, kv_heads, head_dim] rounded into the cache's pages (see armor.h)."""
    _kv_write(ctx, _cuda_index(k, "k"), cache, batch, k, v)


def armor_kv_read(ctx, cache: KvCache, batch: KvBatch, k, v) -> None:
    """The same rows of the cache, to k and v."""
    _kv_read(ctx, cache, batch, _kv_rows(cache, batch, k, v, _cuda_index(k, "k")))


def _kv_attend(ctx, here, cache, batch, q, o, scale, window, max_chunk) -> torch.Tensor:
    _kv_here(cache, batch, here)
    code = _row_dtype(q, "q")
    dim = cache.head_dim
    qp, qr, qh = _heads_at(q, q.dtype, None, None, dim, "q", here)
    rows, heads, _ = q.shape
    if o is None:
        o = q.new_empty((rows, heads, dim))
        op, orow, oh = o.data_ptr(), heads * dim, dim
    else:
        op, orow, oh = _heads_at(o, q.dtype, rows, heads, dim, "o", here)
    code = lib().armor_kv_attend(ctx, cache.args, batch.args, armor_kv_attend_args(qp, op, rows, heads, qr, qh, orow, oh, window, max_chunk, scale, code),
                                 _stream())
    if code:
        _check(code, "armor_kv_attend")
    return o


def armor_kv_attend(ctx, cache: KvCache, batch: KvBatch, q, o, scale: float, window: int = 0, max_chunk: int = 0) -> None:
    """o [rows, heads, head_dim] = attention of q over the cache (see armor.h)."""
    if o is None:
        raise ValueError("o is missing")
    _kv_attend(ctx, _cuda_index(q, "q"), cache, batch, q, o, scale, window, max_chunk)


def armor_get_device_status(ctx, n: int = 16) -> list[int]:
    buf = (C.c_int32 * n)()
    _check(lib().armor_get_device_status(ctx, buf, n), "armor_get_device_status")
    return list(buf)


def armor_selftest_wait_timeout(ctx, limit_cycles: int, result: torch.Tensor) -> None:
    _check(lib().armor_selftest_wait_timeout(ctx, int(limit_cycles), _ptr(result, torch.int32, "result"), _stream()),
           "armor_selftest_wait_timeout")


def armor_launch_count(ctx) -> int:
    return int(lib().armor_launch_count(ctx))


def armor_normalize_noalloc(W: torch.Tensor, Wbar: torch.Tensor, r1: torch.Tensor, r2: torch.Tensor) -> None:
    """Normalisation without a context or a workspace, for callers that may not allocate device memory:
    the scratch is a fixed 4 MiB array inside the library (d_in <= 8192, d_out <= 65536).  All arguments are
    the caller's CUDA tensors; this wrapper allocates nothing either.  Calls that overlap on one GPU race."""
    f = torch.float32
    if W.dim() != 2:
        raise ValueError("W must be [d_out, d_in]")
    _check(lib().armor_normalize_noalloc(_ptr(W, f, "W"), W.shape[0], W.shape[1], _ptr(Wbar, f, "Wbar"),
                                         _ptr(r1, f, "r1"), _ptr(r2, f, "r2"), _stream()), "armor_normalize_noalloc")


def armor_block_product(ctx, side: int, transpose: bool, blocks, x, out, alpha=1.0, add=None, beta=0.0, path=-1) -> None:
    """out = alpha * (x . Q or Q . x) + beta * add with the block-diagonal Q (see armor.h)."""
    f = torch.float32
    _check(lib().armor_block_product(ctx, int(side), int(bool(transpose)), _ptr(blocks, f, "blocks"), _ptr(x, f, "x"),
                                     _ptr(out, f, "out"), x.shape[0], x.shape[1], float(alpha), _ptr(add, f, "add"),
                                     float(beta), int(path), _stream()), "armor_block_product")


def armor_block_product_two_sided(ctx, left, transpose_left: bool, x, right, transpose_right: bool, out, alpha=1.0,
                                  path=-1) -> None:
    """out = alpha * Lop . x . Rop with both block-diagonal wrappers (see armor.h)."""
    f = torch.float32
    _check(lib().armor_block_product_two_sided(ctx, _ptr(left, f, "left"), int(bool(transpose_left)), _ptr(x, f, "x"),
                                               _ptr(right, f, "right"), int(bool(transpose_right)), _ptr(out, f, "out"),
                                               float(alpha), int(path), _stream()), "armor_block_product_two_sided")


def armor_block_product_dual(ctx, blocks, x1, x2, out, path=-1) -> float:
    """out = Q . x2 per block row; returns <Q . x1, Q . x2> (see armor.h)."""
    f = torch.float32
    dot = torch.zeros(1, dtype=torch.float64, device=out.device)
    _check(lib().armor_block_product_dual(ctx, _ptr(blocks, f, "blocks"), _ptr(x1, f, "x1"), _ptr(x2, f, "x2"),
                                          _ptr(out, f, "out"), _ptr(dot, torch.float64, "dot"), int(path), _stream()),
           "armor_block_product_dual")
    return float(dot.item())


def armor_gemm_timing_enable(ctx, enable: bool) -> None:
    _check(lib().armor_gemm_timing_enable(ctx, int(bool(enable))), "armor_gemm_timing_enable")


KERNEL_CLASSES = ["gemm", "block_product", "block_gram", "cholesky", "axpy", "dot", "masked_copy", "mask_select",
                  "mask_guard", "operand_split", "gram_staging", "init", "small", "forward"]


def armor_fuse_grams(ctx, enable: bool) -> None:
    _check(lib().armor_fuse_grams(ctx, 1 if enable else 0), "armor_fuse_grams")


def armor_use_graphs(ctx, enable: bool) -> None:
    _check(lib().armor_use_graphs(ctx, 1 if enable else 0), "armor_use_graphs")


def armor_kernel_timing_enable(ctx, level: int) -> None:
    _check(lib().armor_kernel_timing_enable(ctx, int(level)), "armor_kernel_timing_enable")


def armor_kernel_timing(ctx) -> dict:
    """{class name: (launches, total ms, total work)} since the last read; clears the record."""
    n = len(KERNEL_CLASSES)
    cnt, ms, work = (C.c_int64 * n)(), (C.c_double * n)(), (C.c_double * n)()
    _check(lib().armor_kernel_timing(ctx, n, cnt, ms, work), "armor_kernel_timing")
    return {name: (int(cnt[k]), float(ms[k]), float(work[k])) for k, name in enumerate(KERNEL_CLASSES)}


def armor_gemm_timing(ctx) -> tuple[int, float, float]:
    """(timed launches, total milliseconds, total algorithmic flops) since the last call."""
    n, ms, fl = C.c_int64(0), C.c_double(0), C.c_double(0)
    _check(lib().armor_gemm_timing(ctx, C.byref(n), C.byref(ms), C.byref(fl)), "armor_gemm_timing")
    return int(n.value), float(ms.value), float(fl.value)


# ---------------------------------------------------------------- convenience wrapper
def _empty_rows(t: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of t's shape, type and device."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


@dataclass
class LayerState:
    Wbar: torch.Tensor
    A: torch.Tensor
    B: torch.Tensor
    S: torch.Tensor
    M: torch.Tensor
    r1: torch.Tensor | None = None
    r2: torch.Tensor | None = None


class ArmorContext:
    """A configuration plus its device workspace.  All methods enqueue on torch's current stream."""

    def __init__(self, d_out, d_in, d_block, device="cuda:0", **kw):
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("ArmorContext needs a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self._sizes = {}
        self.cfg = make_config(d_out, d_in, d_block, **kw)
        self.d_out, self.d_in, self.d_block = d_out, d_in, d_block
        nbytes = armor_workspace_bytes(self.cfg)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            off = (-self.workspace.data_ptr()) % 256
            self._ws_view = self.workspace[off: off + nbytes]
            self.ctx = armor_create(self.cfg, self._ws_view)

    def close(self):
        if getattr(self, "ctx", None) is not None:
            armor_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- calls
    def new_gram(self) -> torch.Tensor:
        return torch.zeros(self.d_in, self.d_in, dtype=torch.float32, device=self.device)

    def gram(self, X: torch.Tensor, H: torch.Tensor) -> torch.Tensor:
        armor_gram(self.ctx, X, H)
        return H

    def init(self, W: torch.Tensor, H: torch.Tensor) -> LayerState:
        dev, f = self.device, torch.float32
        nbo, nbi, db = self.d_out // self.d_block, self.d_in // self.d_block, self.d_block
        st = LayerState(
            Wbar=torch.empty_like(W),
            A=torch.empty(nbo, db, db, dtype=f, device=dev), B=torch.empty(nbi, db, db, dtype=f, device=dev),
            S=torch.empty_like(W), M=torch.empty(self.d_out, self.d_in // self.cfg.m_group, dtype=torch.uint8, device=dev))
        if self.cfg.normalize:
            st.r1 = torch.empty(self.d_in, dtype=f, device=dev)
            st.r2 = torch.empty(self.d_out, dtype=f, device=dev)
        armor_init(self.ctx, W, H, st.Wbar, st.r1, st.r2, st.A, st.B, st.S, st.M)
        return st

    def bcd_step(self, st: LayerState, H: torch.Tensor, t_first: int, n_iters: int, want_stats: bool = True):
        stats = None
        if want_stats:
            stats = torch.zeros(max(n_iters, 1) * STATS_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        armor_bcd_step(self.ctx, st.Wbar, H, st.A, st.B, st.S, st.M, t_first, n_iters, stats)
        return stats

    @staticmethod
    def read_stats(stats: torch.Tensor) -> np.ndarray:
        """Device->host copy of the per-iteration records (synchronises)."""
        return stats.cpu().numpy().view(STATS_DTYPE)

    def proxy_loss(self, st: LayerState, H: torch.Tensor) -> torch.Tensor:
        out = torch.zeros(1, dtype=torch.float64, device=self.device)
        armor_proxy_loss(self.ctx, st.Wbar, H, st.A, st.B, st.S, out)
        return out

    def apply(self, st: LayerState, x: torch.Tensor, denormalize: bool = False, sparse: bool = False) -> torch.Tensor:
        y = torch.empty(x.shape[0], self.d_out, dtype=x.dtype, device=self.device)
        r1, r2 = (st.r1, st.r2) if denormalize else (None, None)
        armor_apply(self.ctx, st.A, st.B, st.S, st.M, r1, r2, x, y, sparse)
        return y

    def pack_core(self, st: LayerState) -> torch.Tensor:
        """The 2:4 core in the sparse tensor cores' format (kept values, then positions), packed once."""
        packed = torch.empty(armor_packed_core_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        armor_pack_core(self.ctx, st.S, st.M, packed)
        return packed

    def apply_packed(self, st: LayerState, packed: torch.Tensor, x: torch.Tensor, denormalize: bool = False) -> torch.Tensor:
        self._packed(packed, armor_packed_core_bytes, "pack_core")
        y = torch.empty(x.shape[0], self.d_out, dtype=x.dtype, device=self.device)
        r1, r2 = (st.r1, st.r2) if denormalize else (None, None)
        armor_apply_packed(self.ctx, st.A, st.B, packed, r1, r2, x, y)
        return y

    def pack_layer(self, st: LayerState, denormalize: bool = False) -> torch.Tensor:
        """Core and wrappers packed for the all-bf16 forward (the normalisation's scales folded into the wrappers)."""
        packed = torch.empty(armor_packed_layer_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        r1, r2 = (st.r1, st.r2) if denormalize else (None, None)
        armor_pack_layer(self.ctx, st.A, st.B, st.S, st.M, r1, r2, packed)
        return packed

    def apply_layer(self, packed: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
        self._packed(packed, armor_packed_layer_bytes, "pack_layer")
        y = torch.empty(x.shape[0], self.d_out, dtype=x.dtype, device=self.device)
        armor_apply_layer(self.ctx, packed, x, y)
        return y

    # -- 8-bit products
    def _here(self, *tensors) -> None:
        """The context's device is the current one and holds every tensor given: the calls enqueue on its current stream."""
        here = self._index
        for t in tensors:
            if t is not None and t.get_device() != here:
                raise ValueError(f"the context is on {self.device}, a tensor on {t.device}")
        if torch._C._cuda_getDevice() != here:
            raise ValueError(f"{self.device} must be the current device")

    def _current(self) -> int:
        """The index of the context's device, which has to be the current one."""
        here = self._index
        if torch._C._cuda_getDevice() != here:
            raise ValueError(f"{self.device} must be the current device")
        return here

    def _packed(self, packed: torch.Tensor, size, made_by: str, exact: bool = False) -> None:
        """`packed` holds what `made_by` packs: the kinds differ in size alone, and a larger one's forward reads behind a smaller one's end."""
        want = self._size(size)
        if packed.dtype is not torch.uint8 or packed.numel() < want or (exact and packed.numel() != want):
            raise ValueError(f"packed must be what {made_by} made for this shape: {want} bytes, got {packed.numel()} elements of {packed.dtype}")

    def _size(self, size) -> int:
        if size not in self._sizes:
            self._sizes[size] = size(self.cfg)
        return self._sizes[size]

    def new_int8_rows(self, n: int, cols: int) -> torch.Tensor:
        """[n, cols] int8 whose rows start on 16-byte boundaries."""
        return torch.empty(n, (cols + 15) // 16 * 16, dtype=torch.int8, device=self.device)[:, :cols]

    def quantize_rows(self, x: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
        """The rows of x (tokens, or the output channels of a weight) as int8 with an fp32 scale each."""
        self._here(x)
        q = self.new_int8_rows(x.shape[0], x.shape[1])
        scale = torch.empty(x.shape[0], dtype=torch.float32, device=self.device)
        armor_quantize_rows(self.ctx, x, q, scale)
        return q, scale

    def linear_i8(self, x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, *, bias: torch.Tensor | None = None,
                  x_scale: torch.Tensor | None = None, out_dtype: torch.dtype | None = None) -> torch.Tensor:
        """y = x W^T (+ bias) in 8 bits with W = w_scale wq as quantize_rows gives it.  x: fp32, bf16 or fp16 (rounded to int8 here), or
        int8 with its x_scale; out_dtype: x's by default, bf16 for int8."""
        here = self._current()
        dt = x.dtype
        code = DTYPE_I8 if dt is torch.int8 else _row_dtype(x, "x")
        xp, ldx, n = _rows_at(x, dt, None, "x", here)
        n_in = x.size(1)
        wp, ldw, n_out = _rows_at(wq, torch.int8, n_in, "wq", here)
        if out_dtype is None:
            out_dtype = torch.bfloat16 if code == DTYPE_I8 else dt
        y = torch.empty(n, n_out, dtype=out_dtype, device=self.device)
        code = lib().armor_linear_i8(self.ctx, xp, code, ldx, None if x_scale is None else _vector_at(x_scale, n, "x_scale", here), wp, ldw,
                                     _vector_at(w_scale, n_out, "w_scale", here), None if bias is None else _vector_at(bias, n_out, "bias", here),
                                     y.data_ptr(), _row_dtype(y, "y"), n_out, n, n_out, n_in, _stream())
        if code:
            _check(code, "armor_linear_i8")
        return y

    def pack_layer_i8(self, st: LayerState, denormalize: bool = False) -> torch.Tensor:
        """Core in 8 bits (a scale for each row) and bf16 wrappers, packed for apply_layer_i8."""
        r1, r2 = (st.r1, st.r2) if denormalize else (None, None)
        self._here(st.A, st.B, st.S, st.M, r1, r2)
        packed = torch.empty(self._size(armor_packed_layer_i8_bytes), dtype=torch.uint8, device=self.device)
        armor_pack_layer_i8(self.ctx, st.A, st.B, st.S, st.M, r1, r2, packed)
        return packed

    def apply_layer_i8(self, packed: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
        here = self._current()
        bf16 = torch.bfloat16
        if x.dtype is not bf16:
            raise ValueError("the packed layer takes bf16 x and y")
        xp, ld, n = _rows_at(x, bf16, self.d_in, "x", here)
        if ld != self.d_in and n > 1:
            raise ValueError("x must be contiguous")
        self._packed(packed, armor_packed_layer_i8_bytes, "pack_layer_i8", exact=True)
        if packed.get_device() != here or not packed.is_contiguous():
            raise ValueError(f"packed must be contiguous and on {self.device}")
        y = torch.empty(n, self.d_out, dtype=bf16, device=self.device)
        code = lib().armor_apply_layer_i8(self.ctx, packed.data_ptr(), xp, y.data_ptr(), n, _stream())
        if code:
            _check(code, "armor_apply_layer_i8")
        return y

    # -- norms between two blocks
    def block_norm(self, x: torch.Tensor, y: torch.Tensor | None = None, *, gate: torch.Tensor | None = None, rows_per_gate: int = 0,
                   w_post: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, post: bool | None = None, pre: bool = True,
                   residual_scale: float = 1.0, eps: float = 1e-6) -> tuple[torch.Tensor, torch.Tensor]:
        """(h, n): the residual stream x plus a block's output y, normed, weighted and gated, and the normed stream that the next
        block reads.  gate: [d], or [n_gates, d] with rows_per_gate; post: a norm of y, None: with w_post."""
        here = self._current()
        h = _empty_rows(x)
        n = _empty_rows(x if y is None else y)
        _block_norm(self.ctx, here, x, y, h, n, None, None, True, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps)
        return h, n

    def block_norm_i8(self, x: torch.Tensor, y: torch.Tensor | None = None, *, gate: torch.Tensor | None = None, rows_per_gate: int = 0,
                      w_post: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, post: bool | None = None, pre: bool = True,
                      residual_scale: float = 1.0, eps: float = 1e-6) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(h, q, scale): as block_norm, the normed stream as int8 rows for linear_i8."""
        here = self._current()
        h = _empty_rows(x)
        q = self.new_int8_rows(x.shape[0], x.shape[1])
        scale = torch.empty(x.shape[0], dtype=torch.float32, device=self.device)
        _block_norm(self.ctx, here, x, y, h, None, q, scale, True, gate, rows_per_gate, w_post, w_pre, post, pre, residual_scale, eps)
        return h, q, scale

    def block_norm_backward(self, h: torch.Tensor, y: torch.Tensor | None, dh: torch.Tensor | None, dn: torch.Tensor | None, *,
                            gate: torch.Tensor | None = None, rows_per_gate: int = 0, w_post: torch.Tensor | None = None,
                            w_pre: torch.Tensor | None = None, post: bool | None = None, pre: bool = True, residual_scale: float = 1.0,
                            eps: float = 1e-6) -> dict[str, torch.Tensor]:
        """The gradients dx, dy (where there is a y) and those of the weights and the gate that are given (fp32), from the h that
        block_norm returned, y and the gradients of h and n."""
        here = self._current()
        out = {"dx": _empty_rows(h)}
        dx, dy = out["dx"], None
        if y is not None:
            out["dy"] = dy = _empty_rows(y)
        dw_pre = dw_post = dgate = None
        if w_pre is not None:
            out["dw_pre"] = dw_pre = torch.empty_like(w_pre)
        if w_post is not None:
            out["dw_post"] = dw_post = torch.empty_like(w_post)
        if gate is not None:
            out["dgate"] = dgate = _empty_rows(gate)
        _block_norm_backward(self.ctx, here, h, y, dh, dn, dx, dy, dw_post, dw_pre, dgate, True, gate, rows_per_gate, w_post, w_pre, post, pre,
                             residual_scale, eps)
        return out

    # -- a paged cache of keys and values, and the attention over it
    def new_kv_cache(self, n_pages: int, page_size: int, kv_heads: int, head_dim: int) -> KvCache:
        """An empty cache of int8 keys and values."""
        k, v = (torch.zeros(n_pages, kv_heads, page_size, head_dim, dtype=torch.int8, device=self.device) for _ in range(2))
        return KvCache(k, v, *(torch.zeros(n_pages, kv_heads, page_size, dtype=torch.float32, device=self.device) for _ in range(2)))

    def kv_write(self, cache: KvCache, batch: KvBatch, k: torch.Tensor, v: torch.Tensor) -> None:
        """Puts the new rows k and v [rows, kv_heads, head_dim] (fp32, bf16 or fp16) into the cache, rounded to int8 with a scale each."""
        _kv_write(self.ctx, self._current(), cache, batch, k, v)

    def kv_read(self, cache: KvCache, batch: KvBatch, rows: int, dtype: torch.dtype = torch.bfloat16, *,
                out: tuple[torch.Tensor, torch.Tensor] | None = None) -> tuple[torch.Tensor, torch.Tensor]:
        """(k, v) [rows, kv_heads, head_dim] of the batch's positions as the cache holds them.  Rows before the first sequence's
        and behind the last one's are left as they are (in new tensors: not set)."""
        here = self._current()
        if out is None:
            # one allocation for both
            _kv_here(cache, batch, here)
            heads, dim = cache.kv_heads, cache.head_dim
            both = cache.k.new_empty((2, rows, heads, dim), dtype=dtype)
            at, row = both.data_ptr(), heads * dim
            args = armor_kv_rows(at, at + rows * row * both.element_size(), rows, row, dim, row, dim, _row_dtype(both, "dtype"))
            _kv_read(self.ctx, cache, batch, args)
            return both.unbind(0)
        k, v = out
        if k.size(0) != rows or k.dtype is not dtype:
            raise ValueError(f"out must have {rows} rows of {dtype}, got {k.size(0)} of {k.dtype}")
        _kv_read(self.ctx, cache, batch, _kv_rows(cache, batch, k, v, here))
        return out

    def kv_attend(self, cache: KvCache, batch: KvBatch, q: torch.Tensor, *, scale: float | None = None, window: int = 0, max_chunk: int = 0,
                  out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of q [rows, heads, head_dim] (bf16 or fp16) over the cache, each row over the positions of its sequence up to its own, the
        last `window` of them if that is not 0; scale: head_dim ** -0.5.  The new rows' keys and values have been written.  Heads
        share keys in groups of heads / kv_heads.  max_chunk: the most rows of a sequence, where the caller knows it (a hint).  Rows
        before the first sequence's and behind the last one's are left as they are (in a new tensor: not set)."""
        return _kv_attend(self.ctx, self._current(), cache, batch, q, out, cache.head_dim ** -0.5 if scale is None else scale, window, max_chunk)

    def device_status(self) -> list[int]:
        torch.cuda.current_stream().synchronize()
        return armor_get_device_status(self.ctx)

    def launch_count(self) -> int:
        return armor_launch_count(self.ctx)

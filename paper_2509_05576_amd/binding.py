"""ctypes binding of include/fobq.h.  Argument marshalling only: torch supplies
device memory and the HIP stream; no arithmetic of the method happens here.
There is no CPU fallback: if libfobq.so is missing the import of the library
fails loudly."""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

OK, EINVAL, ENOMEM, EHIP, ENOTPD, ESTATE = 0, -1, -2, -3, -4, -5
ORDER_NATURAL, ORDER_SENSI_DESC, ORDER_CUSTOM = 0, 1, 2
ORDER_ERR_DESC, ORDER_W_DESC, ORDER_SENSI_ASC, ORDER_ERR_ASC, ORDER_W_ASC = 3, 4, 5, 6, 7
ORDER_SENSI_DYNAMIC = 8
STAGES = ("xxt", "finalize", "cholesky", "inverse", "order", "permute", "eliminate", "columns", "emit", "slice")
HESSIAN_FP64, HESSIAN_INT8_SLICES = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_HERE, "libfobq.so")


class FobqOpts(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("group", ctypes.c_int32),
                ("damp", ctypes.c_double), ("damp_abs", ctypes.c_double),
                ("order", ctypes.c_int32), ("block", ctypes.c_int32),
                ("stop_after", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("perm_in", ctypes.c_void_p)]


class FobqOut(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("zeros", ctypes.c_void_p),
                ("Q", ctypes.c_void_p), ("perm", ctypes.c_void_p), ("W_work", ctypes.c_void_p),
                ("Hinv_work", ctypes.c_void_p), ("loss", ctypes.c_void_p)]


# The structs of the calls that run a quantized network, as bytes with C's layout: fobq_fp8_matrix, fobq_kv4_cache, fobq_kv4_batch, fobq_kv4_query
# in the order of their fields.  (A ctypes structure takes four times as long to fill, and these calls are short.)
_fp8_matrix = struct.Struct("@PPqqqqii").pack
_kv4_cache = struct.Struct("@PPPPqiiii").pack
_kv4_batch = struct.Struct("@PPPqqii").pack
_kv4_query = struct.Struct("@PPPqqqqqiiiifi").pack
# and of a feed-forward part of experts: fobq_norm, fobq_router, fobq_routing, fobq_fp8_experts
_norm = struct.Struct("@PPPPPqqqqiifi").pack
_router = struct.Struct("@PPqqiiiiiiiifi").pack
_routing = struct.Struct("@PPPPP").pack
_fp8_experts = struct.Struct("@PPqqqqqqiiii").pack


class FobqLayer(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("d_row", ctypes.c_int64), ("d_col", ctypes.c_int64),
                ("H", ctypes.c_void_p), ("out", FobqOut)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libfobq.so (built by paper_2509_05576_amd/build.py).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not found: build it with `python -m paper_2509_05576_amd.build` "
                                "(there is no fallback implementation)")
    lib = ctypes.CDLL(path)
    vp, i64, i32, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_double
    lib.fobq_create.argtypes = [ctypes.POINTER(vp), i32, vp]
    lib.fobq_destroy.argtypes = [vp]
    lib.fobq_last_error.argtypes = [vp]
    lib.fobq_last_error.restype = ctypes.c_char_p
    lib.fobq_hessian_begin.argtypes = [vp, i64]
    lib.fobq_hessian_set_mode.argtypes = [vp, i32]
    lib.fobq_hessian_accumulate.argtypes = [vp, vp, i64, i64]
    lib.fobq_hessian_accumulate_conv.argtypes = [vp, vp, i64, i64, i64, i64, i32, i32, i32]
    lib.fobq_hessian_finalize.argtypes = [vp, vp]
    lib.fobq_quantize_layer.argtypes = [vp, vp, i64, i64, vp, ctypes.POINTER(FobqOpts), ctypes.POINTER(FobqOut)]
    lib.fobq_quantize_layer_enqueue.argtypes = lib.fobq_quantize_layer.argtypes
    lib.fobq_quantize_layers_batched.argtypes = [vp, i32, ctypes.POINTER(FobqLayer), ctypes.POINTER(FobqOpts)]
    lib.fobq_finish.argtypes = [vp]
    lib.fobq_spd_inverse.argtypes = [vp, vp, i64, vp]
    lib.fobq_sensitivity.argtypes = [vp, vp, i64, i64, vp, ctypes.POINTER(FobqOpts), vp, vp]
    lib.fobq_sensitivity_static.argtypes = lib.fobq_sensitivity.argtypes
    lib.fobq_debug_fail_after.argtypes = [vp, i32]
    lib.fobq_debug_wait_looks.argtypes = [vp, i32]
    lib.fobq_debug_plan.argtypes = [i32, ctypes.POINTER(i64), i32, ctypes.POINTER(i64), i32]
    lib.fobq_debug_offset_tables.argtypes = [i32, i32, i64, i64, ctypes.POINTER(i32), i64, ctypes.POINTER(i64)]
    lib.fobq_workspace_bytes.argtypes = [vp, ctypes.POINTER(i64)]
    lib.fobq_hessian_form.argtypes = [vp, ctypes.POINTER(i32)]
    lib.fobq_obq_rows.argtypes = [vp, vp, i64, i64, vp, ctypes.POINTER(FobqOpts), i64, i64, vp, vp, vp, vp]
    ptr = ctypes.POINTER
    lib.fobq_fp8_quantize.argtypes = [vp, vp, i32, i64, vp]
    lib.fobq_fp8_from_codes.argtypes = [vp, vp, vp, vp, i32, i32, vp]
    lib.fobq_fp8_matmul.argtypes = [vp, vp, vp, vp, i32, i64, vp, i64]
    lib.fobq_fp8_matmul_workspace.argtypes = [vp, i64, i64, i64, i32, ptr(i64)]
    lib.fobq_kv4_append.argtypes = [vp, vp, vp, i32, vp, i64, i64, vp, i64, i64]
    lib.fobq_kv4_read.argtypes = lib.fobq_kv4_append.argtypes
    lib.fobq_kv4_attention.argtypes = [vp, vp, vp, vp, vp, i64]
    lib.fobq_kv4_attention_workspace.argtypes = [vp, vp, vp, vp, ptr(i64)]
    lib.fobq_fp8_rms_norm.argtypes = [vp, vp, vp]
    lib.fobq_fp8_swiglu.argtypes = [vp, vp, i32, i64, vp]
    lib.fobq_route.argtypes = [vp, vp, vp, vp, i64]
    lib.fobq_route_workspace.argtypes = [vp, i64, i32, ptr(i64)]
    lib.fobq_fp8_expert_matmul.argtypes = [vp, vp, vp, vp, vp, i32, i64, vp, i32, i64]
    lib.fobq_expert_sum.argtypes = [vp, vp, i32, i64, i64, i64, vp, vp, i64, i32, vp, i64, vp, i64]
    lib.fobq_probe_int8_matrix_rate.argtypes = [vp, i32, ctypes.POINTER(dbl)]
    lib.fobq_profile_enable.argtypes = [vp, i32]
    lib.fobq_profile_get.argtypes = [vp, i32, ctypes.POINTER(dbl), ctypes.POINTER(i64)]
    lib.fobq_profile_reset.argtypes = [vp]
    for name in ("fobq_create", "fobq_destroy", "fobq_hessian_begin", "fobq_hessian_set_mode", "fobq_hessian_accumulate",
                 "fobq_hessian_accumulate_conv", "fobq_hessian_finalize", "fobq_quantize_layer",
                 "fobq_quantize_layer_enqueue", "fobq_quantize_layers_batched", "fobq_finish", "fobq_spd_inverse", "fobq_sensitivity",
                 "fobq_sensitivity_static", "fobq_debug_fail_after", "fobq_debug_wait_looks", "fobq_debug_plan", "fobq_debug_offset_tables", "fobq_workspace_bytes", "fobq_probe_int8_matrix_rate", "fobq_obq_rows", "fobq_hessian_form",
                 "fobq_fp8_quantize", "fobq_fp8_from_codes", "fobq_fp8_matmul", "fobq_fp8_matmul_workspace",
                 "fobq_kv4_append", "fobq_kv4_read", "fobq_kv4_attention", "fobq_kv4_attention_workspace",
                 "fobq_fp8_rms_norm", "fobq_fp8_swiglu", "fobq_route", "fobq_route_workspace", "fobq_fp8_expert_matmul", "fobq_expert_sum",
                 "fobq_profile_enable", "fobq_profile_get", "fobq_profile_reset"):
        getattr(lib, name).restype = i32
    _lib = lib
    return lib


# fobq_float and fobq_fp8 by torch's names
_FLOAT = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_FP8 = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}
_F32, _U8, _I32, _HALF = (torch.float32,), (torch.uint8,), (torch.int32,), (torch.bfloat16, torch.float16)


class FobqError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"fobq status {code}: {msg}")
        self.code = code


def _ptr(t: Optional[torch.Tensor], dtype: torch.dtype, what: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{what}: need a contiguous device tensor of {dtype}, got {t.dtype} on {t.device}")
    return t.data_ptr()


_streams = {}      # the device and the stream of every context made here


# ---- functions with the names of the C entry points -------------------------------------------
def fobq_create(device: int = 0, stream: Optional[int] = None) -> int:
    lib = load_library()
    h = ctypes.c_void_p()
    if stream is None:
        stream = torch.cuda.current_stream(device).cuda_stream
    rc = lib.fobq_create(ctypes.byref(h), device, ctypes.c_void_p(stream))
    if rc != OK:
        raise FobqError(rc, "fobq_create failed")
    _streams[h.value] = (device, stream)
    return h.value


def fobq_destroy(ctx: int) -> None:
    load_library().fobq_destroy(ctypes.c_void_p(ctx))
    _streams.pop(ctx, None)


def fobq_last_error(ctx: int) -> str:
    return load_library().fobq_last_error(ctypes.c_void_p(ctx)).decode()


def _check(ctx: int, rc: int) -> None:
    if rc != OK:
        raise FobqError(rc, fobq_last_error(ctx))


def fobq_hessian_begin(ctx: int, d_col: int) -> None:
    _check(ctx, load_library().fobq_hessian_begin(ctypes.c_void_p(ctx), d_col))


def fobq_hessian_set_mode(ctx: int, mode: int) -> None:
    _check(ctx, load_library().fobq_hessian_set_mode(ctypes.c_void_p(ctx), mode))


def fobq_hessian_accumulate(ctx: int, X: torch.Tensor) -> None:
    """X: device fp32, d_col x n, unit column stride (row stride = X.stride(0))."""
    if not X.is_cuda or X.dtype != torch.float32 or X.dim() != 2 or (X.shape[1] > 1 and X.stride(1) != 1):
        raise TypeError("X must be a 2-D device fp32 tensor with unit column stride")
    _check(ctx, load_library().fobq_hessian_accumulate(ctypes.c_void_p(ctx), ctypes.c_void_p(X.data_ptr()),
                                                       X.shape[1], X.stride(0)))


def fobq_hessian_accumulate_conv(ctx: int, maps: torch.Tensor, k: int, stride: int = 1, pad: int = 0) -> None:
    """maps: device fp32, images x h x w x channels, contiguous (channels innermost)."""
    if not maps.is_cuda or maps.dtype != torch.float32 or maps.dim() != 4 or not maps.is_contiguous():
        raise TypeError("maps must be a contiguous 4-D device fp32 tensor (images, h, w, channels)")
    n, h, w, c = maps.shape
    _check(ctx, load_library().fobq_hessian_accumulate_conv(ctypes.c_void_p(ctx), ctypes.c_void_p(maps.data_ptr()),
                                                            n, h, w, c, k, stride, pad))


def fobq_hessian_finalize(ctx: int, H_out: Optional[torch.Tensor] = None) -> None:
    _check(ctx, load_library().fobq_hessian_finalize(ctypes.c_void_p(ctx),
                                                     ctypes.c_void_p(_ptr(H_out, torch.float64, "H_out"))))


def _opts(bits, group, damp, damp_abs, order, block, stop_after, perm_in) -> FobqOpts:
    return FobqOpts(bits, group, damp, damp_abs, order, block, stop_after, 0,
                    _ptr(perm_in, torch.int32, "perm_in"))


@dataclass
class LayerOutput:
    codes: torch.Tensor
    scales: torch.Tensor
    zeros: torch.Tensor
    Q: torch.Tensor
    perm: torch.Tensor
    loss: torch.Tensor
    W_work: Optional[torch.Tensor] = None
    Hinv_work: Optional[torch.Tensor] = None


def fobq_quantize_layer(ctx: int, W: torch.Tensor, H: Optional[torch.Tensor] = None, *, bits: int = 4,
                        group: int = 0, damp: float = 0.01, damp_abs: float = 0.0,
                        order: int = ORDER_SENSI_DESC, block: int = 0, stop_after: int = -1,
                        perm_in: Optional[torch.Tensor] = None, debug: bool = False,
                        out: Optional[LayerOutput] = None, wait: bool = True) -> LayerOutput:
    """Allocates the outputs (unless `out` is given) and calls fobq_quantize_layer, or, with
    wait=False, fobq_quantize_layer_enqueue: the outputs are then valid after fobq_finish(ctx), and
    W, H, perm_in must be kept alive until then."""
    if W.dim() != 2:
        raise TypeError("W must be 2-D")
    r, d = W.shape
    dev = W.device
    g = d // group if group > 0 and d % group == 0 else 1
    if out is None:
        out = LayerOutput(
            codes=torch.empty((r, d), dtype=torch.uint8, device=dev),
            scales=torch.empty((r, g), dtype=torch.float32, device=dev),
            zeros=torch.empty((r, g), dtype=torch.float32, device=dev),
            Q=torch.empty((r, d), dtype=torch.float32, device=dev),
            perm=torch.empty((d,), dtype=torch.int32, device=dev),
            loss=torch.empty((1,), dtype=torch.float64, device=dev),
            W_work=torch.empty((r, d), dtype=torch.float64, device=dev) if debug else None,
            Hinv_work=torch.empty((d, d), dtype=torch.float64, device=dev) if debug else None)
    co = FobqOut(_ptr(out.codes, torch.uint8, "codes"), _ptr(out.scales, torch.float32, "scales"),
                 _ptr(out.zeros, torch.float32, "zeros"), _ptr(out.Q, torch.float32, "Q"),
                 _ptr(out.perm, torch.int32, "perm"), _ptr(out.W_work, torch.float64, "W_work"),
                 _ptr(out.Hinv_work, torch.float64, "Hinv_work"), _ptr(out.loss, torch.float64, "loss"))
    op = _opts(bits, group, damp, damp_abs, order, block, stop_after, perm_in)
    lib = load_library()
    fn = lib.fobq_quantize_layer if wait else lib.fobq_quantize_layer_enqueue
    rc = fn(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(W, torch.float32, "W")), r, d,
            ctypes.c_void_p(_ptr(H, torch.float64, "H")), ctypes.byref(op), ctypes.byref(co))
    _check(ctx, rc)
    return out


def _alloc_output(W: torch.Tensor, group: int) -> LayerOutput:
    r, d = W.shape
    g = d // group if group > 0 and d % group == 0 else 1
    dev = W.device
    return LayerOutput(codes=torch.empty((r, d), dtype=torch.uint8, device=dev),
                       scales=torch.empty((r, g), dtype=torch.float32, device=dev),
                       zeros=torch.empty((r, g), dtype=torch.float32, device=dev),
                       Q=torch.empty((r, d), dtype=torch.float32, device=dev),
                       perm=torch.empty((d,), dtype=torch.int32, device=dev),
                       loss=torch.empty((1,), dtype=torch.float64, device=dev))


def fobq_quantize_layers_batched(ctx: int, Ws, Hs, *, bits: int = 4, group: int = 0, damp: float = 0.01,
                                 damp_abs: float = 0.0, order: int = ORDER_SENSI_DESC, outs=None):
    """Ws, Hs: lists of device tensors (fp32 d_row x d_col, fp64 d_col x d_col).  Allocates the outputs unless
    `outs` (a list of LayerOutput) is given; returns the list of LayerOutput."""
    n = len(Ws)
    if outs is None:
        outs = [_alloc_output(W, group) for W in Ws]
    arr = (FobqLayer * max(n, 1))()
    for i, (W, H, out) in enumerate(zip(Ws, Hs, outs)):
        if W.dim() != 2:
            raise TypeError("W must be 2-D")
        co = FobqOut(_ptr(out.codes, torch.uint8, "codes"), _ptr(out.scales, torch.float32, "scales"),
                     _ptr(out.zeros, torch.float32, "zeros"), _ptr(out.Q, torch.float32, "Q"),
                     _ptr(out.perm, torch.int32, "perm"), None, None, _ptr(out.loss, torch.float64, "loss"))
        arr[i] = FobqLayer(_ptr(W, torch.float32, "W"), W.shape[0], W.shape[1], _ptr(H, torch.float64, "H"), co)
    op = _opts(bits, group, damp, damp_abs, order, 0, -1, None)
    _check(ctx, load_library().fobq_quantize_layers_batched(ctypes.c_void_p(ctx), n, arr, ctypes.byref(op)))
    return outs


def fobq_finish(ctx: int) -> None:
    _check(ctx, load_library().fobq_finish(ctypes.c_void_p(ctx)))


def fobq_spd_inverse(ctx: int, H: torch.Tensor) -> torch.Tensor:
    d = H.shape[0]
    Hinv = torch.empty((d, d), dtype=torch.float64, device=H.device)
    _check(ctx, load_library().fobq_spd_inverse(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(H, torch.float64, "H")),
                                                d, ctypes.c_void_p(Hinv.data_ptr())))
    return Hinv


def _sensitivity(fn, ctx, W, Hinv, bits, group, order, perm_in, S, perm):
    r, d = W.shape
    if S is None:
        S = torch.empty((d,), dtype=torch.float64, device=W.device)
    if perm is None:
        perm = torch.empty((d,), dtype=torch.int32, device=W.device)
    op = _opts(bits, group, 0.0, 0.0, order, 0, -1, perm_in)
    rc = fn(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(W, torch.float32, "W")), r, d,
            ctypes.c_void_p(_ptr(Hinv, torch.float64, "Hinv")), ctypes.byref(op),
            ctypes.c_void_p(_ptr(S, torch.float64, "S")), ctypes.c_void_p(_ptr(perm, torch.int32, "perm")))
    _check(ctx, rc)
    return S, perm


def fobq_sensitivity(ctx: int, W: torch.Tensor, Hinv: torch.Tensor, *, bits: int = 4, group: int = 0,
                     order: int = ORDER_SENSI_DESC, perm_in: Optional[torch.Tensor] = None,
                     S: Optional[torch.Tensor] = None, perm: Optional[torch.Tensor] = None):
    return _sensitivity(load_library().fobq_sensitivity, ctx, W, Hinv, bits, group, order, perm_in, S, perm)


def fobq_sensitivity_static(ctx: int, W: torch.Tensor, Hinv: torch.Tensor, *, bits: int = 4, group: int = 0,
                            order: int = ORDER_SENSI_DESC, perm_in: Optional[torch.Tensor] = None,
                            S: Optional[torch.Tensor] = None, perm: Optional[torch.Tensor] = None):
    """The entry point that allocates nothing; pass S and perm to keep torch from allocating either."""
    return _sensitivity(load_library().fobq_sensitivity_static, ctx, W, Hinv, bits, group, order, perm_in, S, perm)


def fobq_obq_rows(ctx: int, W: torch.Tensor, Hinv: torch.Tensor, *, bits: int = 4, group: int = 0,
                  rows: Optional[tuple] = None):
    """The per-row baseline (own inverse and own greedy order per row) on rows[0] .. rows[1] - 1 (default: all).
    Returns codes (uint8), Q (fp32), order (int32), lossrow (fp64); only the processed rows are written."""
    r, d = W.shape
    lo, hi = (0, r) if rows is None else rows
    codes = torch.zeros((r, d), dtype=torch.uint8, device=W.device)
    Q = torch.zeros((r, d), dtype=torch.float32, device=W.device)
    order = torch.zeros((r, d), dtype=torch.int32, device=W.device)
    lossrow = torch.zeros((r,), dtype=torch.float64, device=W.device)
    op = _opts(bits, group, 0.0, 0.0, ORDER_NATURAL, 0, -1, None)
    rc = load_library().fobq_obq_rows(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(W, torch.float32, "W")), r, d,
                                      ctypes.c_void_p(_ptr(Hinv, torch.float64, "Hinv")), ctypes.byref(op), lo, hi,
                                      ctypes.c_void_p(_ptr(codes, torch.uint8, "codes")), ctypes.c_void_p(_ptr(Q, torch.float32, "Q")),
                                      ctypes.c_void_p(_ptr(order, torch.int32, "order")),
                                      ctypes.c_void_p(_ptr(lossrow, torch.float64, "lossrow")))
    _check(ctx, rc)
    return codes, Q, order, lossrow


FORM_FP64, FORM_INT8_SLICES, FORM_INT8_TAP_OFFSETS = 0, 1, 2


def fobq_hessian_form(ctx: int) -> int:
    """The arithmetic the running (or last finalized) accumulation took: FORM_FP64 / _INT8_SLICES / _INT8_TAP_OFFSETS."""
    f = ctypes.c_int32(0)
    _check(ctx, load_library().fobq_hessian_form(ctypes.c_void_p(ctx), ctypes.byref(f)))
    return f.value


def fobq_workspace_bytes(ctx: int) -> int:
    b = ctypes.c_int64(0)
    _check(ctx, load_library().fobq_workspace_bytes(ctypes.c_void_p(ctx), ctypes.byref(b)))
    return b.value


PROBE_EQUAL_BYTES, PROBE_RANDOM_BYTES, PROBE_RELU_DIGITS = 0, 1, 2


def fobq_probe_int8_matrix_rate(ctx: int, operand_kind: int) -> float:
    """1e12 int8 operations per second of the X X^T kernel's inner loop with its operands fixed in LDS."""
    r = ctypes.c_double(0.0)
    _check(ctx, load_library().fobq_probe_int8_matrix_rate(ctypes.c_void_p(ctx), operand_kind, ctypes.byref(r)))
    return r.value


def fobq_debug_fail_after(ctx: int, n: int) -> None:
    _check(ctx, load_library().fobq_debug_fail_after(ctypes.c_void_p(ctx), n))


def fobq_debug_wait_looks(ctx: int, looks: int) -> None:
    _check(ctx, load_library().fobq_debug_wait_looks(ctypes.c_void_p(ctx), looks))


PLAN_PAD, PLAN_ELIMINATE, PLAN_HESSIAN, PLAN_SLABS = 0, 1, 2, 3
PLAN_FP8_MATMUL, PLAN_KV4_ATTENTION, PLAN_KV4_PLACE, PLAN_FP8_CHECK, PLAN_KV4_CHECK = 4, 5, 6, 7, 8
PLAN_ROUTE, PLAN_EXPERTS, PLAN_NORM_CHECK, PLAN_ROUTE_CHECK, PLAN_EXPERTS_CHECK, PLAN_SUM_CHECK = 9, 10, 11, 12, 13, 14


def fobq_debug_plan(what: int, args, n_out: int):
    """fobq_debug_plan: the list of its n_out words.  Host code only: no GPU, no context."""
    a, out = (ctypes.c_int64 * len(args))(*args), (ctypes.c_int64 * n_out)()
    rc = load_library().fobq_debug_plan(what, a, len(args), out, n_out)
    if rc != OK:
        raise FobqError(rc, "fobq_debug_plan: bad argument")
    return list(out)


def fobq_debug_offset_tables(k: int, pad: int, h: int, w: int):
    """fobq_debug_offset_tables: (jobs, pairs, terms) as lists of tuples, or None when the geometry does not fit
    the library's tables.  Host code only: no GPU, no context."""
    lib = load_library()
    cap = 3 + 6 * 128 + 4 * 81 + 2 * 384
    buf = (ctypes.c_int32 * cap)()
    used = ctypes.c_int64(0)
    rc = lib.fobq_debug_offset_tables(k, pad, h, w, buf, cap, ctypes.byref(used))
    if rc == ESTATE:
        return None
    if rc != OK:
        raise FobqError(rc, "fobq_debug_offset_tables: bad argument")
    v = list(buf[:used.value])
    nj, npair, nt = v[0], v[1], v[2]
    o = 3
    jobs = [tuple(v[o + 6 * i:o + 6 * i + 6]) for i in range(nj)]
    o += 6 * nj
    pairs = [tuple(v[o + 4 * i:o + 4 * i + 4]) for i in range(npair)]
    o += 4 * npair
    terms = [tuple(v[o + 2 * i:o + 2 * i + 2]) for i in range(nt)]
    return jobs, pairs, terms


# ---- running a quantized network ----------------------------------------------------------------
# Like the entry points they wrap, these calls enqueue on the context's stream and return.  What they allocate (outputs that are not
# given, scratch) belongs to that stream; inputs that another stream made, and outputs that another stream uses, are ordered by the
# caller, as between any two streams.  Under capture the context's stream has to be the captured one.
# They have no backward pass: tensors that require gradients are taken as they are, and results do not require any.
# The checks of a call are a few attribute reads each: a call takes the host 3 us to launch, and a step of generation makes hundreds.
_current_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)      # (the public call makes a stream object: 1.9 us against 0.1)


def _need(t: torch.Tensor, ctx: int, dtypes, dims: int, what: str) -> torch.Tensor:
    """A device tensor of one of these types whose last dimension is adjacent, on the context's device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or t.dim() != dims or (t.stride()[-1] != 1 and t.shape[-1] > 1):
        names = " or ".join(str(d) for d in dtypes)
        got = f"{tuple(t.shape)} {t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise TypeError(f"{what}: need a {dims}-D device tensor of {names} with adjacent last dimension, got {got}")
    home = _streams.get(ctx)
    if home is not None and t.get_device() != home[0]:
        raise TypeError(f"{what}: on {t.device}, but the context is on device {home[0]}")
    return t


def _empty(ctx: int, shape, dtype: torch.dtype, device) -> torch.Tensor:
    """Memory that belongs to the context's stream, which need not be the current one."""
    home = _streams.get(ctx)
    if home is None or _current_stream(device.index) == home[1]:
        return torch.empty(shape, dtype=dtype, device=device)
    # (the default stream has no handle: torch takes an external stream of 0 as one that is not given, and makes another)
    stream = torch.cuda.ExternalStream(home[1], device=device) if home[1] else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


@dataclass
class Fp8Matrix:
    """A matrix in 8-bit floating point: values (float8_e4m3fn or float8_e5m2, rows x cols, rows a multiple of 16 bytes apart) and the
    scales (fp32, ceil(cols / 128) x ceil(rows / rows_per_scale)) of its blocks of 128 columns and 1 or 128 rows."""
    values: torch.Tensor
    scales: torch.Tensor
    rows_per_scale: int = 1


def _fp8(ctx: int, m: Fp8Matrix, what: str):
    """What the library calls a matrix, its rows and columns."""
    v, s, per, home = m.values, m.scales, m.rows_per_scale, _streams.get(ctx)
    dev = home[0] if home is not None else None
    try:
        (ld, one), (ld_scales, one_scale), (rows, cols), (sc, sr) = v.stride(), s.stride(), v.shape, s.shape
        fine = (v.dtype in _FP8 and s.dtype is torch.float32 and v.get_device() == dev and s.get_device() == dev and (one == 1 or cols <= 1)
                and (one_scale == 1 or sr <= 1))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        # which of them it is
        _need(v, ctx, _FP8, 2, what + ".values")
        _need(s, ctx, _F32, 2, what + ".scales")
        (ld, _), (ld_scales, _), (rows, cols), (sc, sr) = v.stride(), s.stride(), v.shape, s.shape
    wide = (cols + 15) & -16
    if per not in (1, 128) or sc != (cols + 127) // 128 or sr != (rows + per - 1) // per:
        raise TypeError(f"{what}: rows_per_scale must be 1 or 128 and scales (ceil(cols / 128), ceil(rows / rows_per_scale)), "
                        f"got {per} and {(sc, sr)} for {rows} x {cols}")
    if rows <= 1 or not cols:
        ld = wide
    if wide != cols and rows and v.storage_offset() + (rows - 1) * ld + wide > v.untyped_storage().nbytes():
        raise TypeError(f"{what}: the last row must be readable to a multiple of 16 bytes")
    return _fp8_matrix(v.data_ptr(), s.data_ptr(), rows, cols, ld, ld_scales if sc > 1 else sr, per, _FP8[v.dtype]), rows, cols


def _new_fp8(ctx: int, rows: int, cols: int, format: torch.dtype, per: int, device):
    """A new matrix, and what the library calls it."""
    if format not in _FP8 or per not in (1, 128):
        raise TypeError(f"format must be float8_e4m3fn or float8_e5m2 and rows_per_scale 1 or 128, got {format} and {per}")
    wide, sr = (cols + 15) & -16, (rows + per - 1) // per
    values, scales = _empty(ctx, (rows, wide), format, device), _empty(ctx, ((cols + 127) // 128, sr), torch.float32, device)
    return (Fp8Matrix(values if wide == cols else values[:, :cols], scales, per),
            _fp8_matrix(values.data_ptr(), scales.data_ptr(), rows, cols, wide, sr, per, _FP8[format]))


def _out_fp8(ctx: int, out: Optional[Fp8Matrix], rows: int, cols: int, format: torch.dtype, per: int, device):
    if out is None:
        return _new_fp8(ctx, rows, cols, format, per, device)
    m, r, c = _fp8(ctx, out, "out")
    if r != rows or c != cols:
        raise TypeError(f"out is {r} x {c}, need {rows} x {cols}")
    return out, m


def fobq_fp8_quantize(ctx: int, X: torch.Tensor, format: torch.dtype = torch.float8_e4m3fn, rows_per_scale: int = 1,
                      out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
    """X: 2-D device tensor (fp32, bf16 or fp16) -> Fp8Matrix: rows_per_scale 1 for activations, 1 or 128 for weights.  No gradient passes it."""
    _need(X, ctx, _FLOAT, 2, "X")
    rows, cols = X.shape
    out, m = _out_fp8(ctx, out, rows, cols, format, rows_per_scale, X.device)
    _check(ctx, load_library().fobq_fp8_quantize(ctx, X.data_ptr(), _FLOAT[X.dtype], X.stride()[0] if rows > 1 else cols, m))
    return out


def fobq_fp8_from_codes(ctx: int, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, bits: int = 4,
                        out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
    """A layer quantized to up to 4 bits (LayerOutput's codes, scales, zeros; one grid per row, or groups of a multiple of 128 columns)
    as an Fp8Matrix that stands for its Q (but for the rounding of the returned scales to fp32)."""
    _need(codes, ctx, (torch.uint8,), 2, "codes")
    rows, cols = codes.shape
    for name, t in (("scales", scales), ("zeros", zeros)):
        _need(t, ctx, _F32, 2, name)
        if t.shape != scales.shape or t.shape[0] != rows or t.shape[1] < 1 or cols % t.shape[1] or not t.is_contiguous():
            raise TypeError(f"{name}: need contiguous rows x groups, got {tuple(t.shape)} for codes {rows} x {cols}")
    if not codes.is_contiguous():
        raise TypeError("codes: need a contiguous tensor")
    out, m = _out_fp8(ctx, out, rows, cols, torch.float8_e4m3fn, 1, codes.device)
    group = cols // scales.shape[1] if scales.shape[1] > 1 else 0
    _check(ctx, load_library().fobq_fp8_from_codes(ctx, codes.data_ptr(), scales.data_ptr(), zeros.data_ptr(), bits, group, m))
    return out


def _scratch(ctx: int, need: int, device) -> Optional[torch.Tensor]:
    return _empty(ctx, (need,), torch.uint8, device) if need else None


def fobq_fp8_matmul(ctx: int, A: Fp8Matrix, B: Fp8Matrix, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A (activations, m x k) times B (weights, n x k) transposed -> m x n of `dtype` (fp32, bf16 or fp16), or into `out`.  In 16 bits, rows beyond
    16 take the 8-bit matrix unit, whose sums of eight products keep 13 bits below the largest; up to 16 rows, and fp32, sum in fp32."""
    (a, m, k), (b, n, k2) = _fp8(ctx, A, "A"), _fp8(ctx, B, "B")
    if k != k2:
        raise TypeError(f"A has {k} columns, B {k2}")
    device = A.values.device
    if out is None:
        if dtype not in _FLOAT:
            raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
        out = _empty(ctx, (m, n), dtype, device)
    else:
        _need(out, ctx, _FLOAT, 2, "out")
        if tuple(out.shape) != (m, n):
            raise TypeError(f"out: need {m} x {n}, got {tuple(out.shape)}")
        dtype = out.dtype
    lib, need = load_library(), ctypes.c_int64(0)
    _check(ctx, lib.fobq_fp8_matmul_workspace(ctx, m, n, k, _FLOAT[dtype], ctypes.byref(need)))
    work = _scratch(ctx, need.value, device)
    _check(ctx, lib.fobq_fp8_matmul(ctx, a, b, out.data_ptr(), _FLOAT[dtype], out.stride()[0] if m > 1 else n,
                                    work.data_ptr() if work is not None else None, need.value))
    return out


@dataclass
class Kv4Cache:
    """A cache of keys and values in 4 bits: codes (uint8, pages x heads x page_size x head_dim / 2) and grid words (int32, pages x heads
    x page_size), contiguous."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_grids: torch.Tensor
    v_grids: torch.Tensor

    @staticmethod
    def empty(pages: int, heads: int, head_dim: int, page_size: int = 64, device="cuda") -> "Kv4Cache":
        codes = [torch.empty((pages, heads, page_size, head_dim // 2), dtype=torch.uint8, device=device) for _ in range(2)]
        return Kv4Cache(*codes, *[torch.empty((pages, heads, page_size), dtype=torch.int32, device=device) for _ in range(2)])


@dataclass
class Kv4Batch:
    """The sequences of a call: table (int32, n_seqs x max_pages: page numbers), lengths (int32, n_seqs: tokens held, new ones included)
    and starts (int32, n_seqs + 1: the sequences' packed rows; None: one row each)."""
    table: torch.Tensor
    lengths: torch.Tensor
    starts: Optional[torch.Tensor] = None


def _kv4(ctx: int, cache: Kv4Cache, batch: Kv4Batch, rows: int):
    """What the library calls a cache and a batch, and the cache's heads and channels."""
    k, v, kg, vg, table, lengths, starts = cache.k_codes, cache.v_codes, cache.k_grids, cache.v_grids, batch.table, batch.lengths, batch.starts
    home, u8, i32 = _streams.get(ctx), torch.uint8, torch.int32
    dev = home[0] if home is not None else None
    try:
        shape = k.shape
        n, width = table.shape
        pages, heads, page, half = shape
        grid = kg.shape
        fine = (k.dtype is u8 and v.dtype is u8 and kg.dtype is i32 and vg.dtype is i32 and table.dtype is i32 and lengths.dtype is i32
                and k.get_device() == dev and v.get_device() == dev and kg.get_device() == dev and vg.get_device() == dev
                and table.get_device() == dev and lengths.get_device() == dev and v.shape == shape and grid == shape[:3] and vg.shape == grid
                and k.is_contiguous() and v.is_contiguous() and kg.is_contiguous() and vg.is_contiguous()
                and ((strides := table.stride())[1] == 1 or width <= 1) and lengths.shape == (n,) and lengths.is_contiguous()
                and (starts is None or (starts.dtype is i32 and starts.get_device() == dev and starts.shape == (n + 1,) and starts.is_contiguous())))
    except (AttributeError, ValueError):
        fine = False
    if not fine:
        # which of them it is
        _need(k, ctx, _U8, 4, "k_codes")
        for name, t, dtypes, dims in (("v_codes", v, _U8, 4), ("k_grids", kg, _I32, 3), ("v_grids", vg, _I32, 3)):
            _need(t, ctx, dtypes, dims, name)
        if v.shape != k.shape or kg.shape != k.shape[:3] or vg.shape != k.shape[:3] or not all(t.is_contiguous() for t in (k, v, kg, vg)):
            raise TypeError(f"cache: need contiguous codes {tuple(k.shape)} and grids {tuple(k.shape[:3])}, got v_codes {tuple(v.shape)}, "
                            f"k_grids {tuple(kg.shape)}, v_grids {tuple(vg.shape)}")
        n = _need(table, ctx, _I32, 2, "table").shape[0]
        if _need(lengths, ctx, _I32, 1, "lengths").shape[0] != n:
            raise TypeError(f"lengths: need {n} entries, got {lengths.shape[0]}")
        if starts is not None and _need(starts, ctx, _I32, 1, "starts").shape[0] != n + 1:
            raise TypeError(f"starts: need {n + 1} entries, got {starts.shape[0]}")
        pages, heads, page, half = k.shape
        width, strides = table.shape[1], table.stride()
    return (_kv4_cache(k.data_ptr(), v.data_ptr(), kg.data_ptr(), vg.data_ptr(), pages, page, heads, 2 * half, 0),
            _kv4_batch(table.data_ptr(), lengths.data_ptr(), starts.data_ptr() if starts is not None else 0, rows,
                       strides[0] if n > 1 else width, n, width), heads, 2 * half)


def _kv_rows(ctx: int, heads: int, dim: int, k: torch.Tensor, v: torch.Tensor, rows: int, dtypes):
    home, shape = _streams.get(ctx), (rows, heads, dim)
    dev = home[0] if home is not None else None
    try:
        (k_row, k_head, one), (v_row, v_head, one_v), dtype = k.stride(), v.stride(), k.dtype
        fine = (dtype in dtypes and v.dtype is dtype and k.shape == shape and v.shape == shape and one == 1 and one_v == 1 and k.get_device() == dev
                and v.get_device() == dev)
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        # which of them it is
        _need(k, ctx, dtypes, 3, "k")
        _need(v, ctx, dtypes, 3, "v")
        if k.shape != shape or v.shape != shape or k.dtype != v.dtype:
            raise TypeError(f"k and v: need {shape} of one type, got {tuple(k.shape)} {k.dtype} and {tuple(v.shape)} {v.dtype}")
        (k_row, k_head, _), (v_row, v_head, _), dtype = k.stride(), v.stride(), k.dtype
    return (_FLOAT[dtype], k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head)


def fobq_kv4_append(ctx: int, cache: Kv4Cache, batch: Kv4Batch, k: torch.Tensor, v: torch.Tensor) -> None:
    """New keys and values (bf16 or fp16, rows x heads x head_dim, any row and head strides) into the sequences' last places."""
    rows = k.shape[0]
    c, b, heads, dim = _kv4(ctx, cache, batch, rows)
    _check(ctx, load_library().fobq_kv4_append(ctx, c, b, *_kv_rows(ctx, heads, dim, k, v, rows, _HALF)))


def fobq_kv4_read(ctx: int, cache: Kv4Cache, batch: Kv4Batch, rows: int, dtype: torch.dtype = torch.bfloat16, out=None):
    """What the packed rows' places in the cache stand for: (k, v), rows x heads x head_dim of `dtype`, or into out = (k, v)."""
    c, b, heads, dim = _kv4(ctx, cache, batch, rows)
    if out is None:
        if dtype not in _FLOAT:
            raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
        shape, device = (rows, heads, dim), cache.k_codes.device
        out = (_empty(ctx, shape, dtype, device), _empty(ctx, shape, dtype, device))
    k, v = out
    _check(ctx, load_library().fobq_kv4_read(ctx, c, b, *_kv_rows(ctx, heads, dim, k, v, rows, _FLOAT)))
    return k, v


def fobq_kv4_attention(ctx: int, cache: Kv4Cache, batch: Kv4Batch, q: torch.Tensor, *, scale: Optional[float] = None, causal: bool = True,
                       window: int = 0, max_length: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q (bf16 or fp16, rows x query heads x head_dim) over the sequences' tokens -> the same shape, or into `out`.  scale: head_dim^-0.5
    unless given.  max_length: the most tokens a sequence holds, if known (a hint).  lse (fp32, rows x query heads): filled.  No gradient passes
    it.  Rows of no sequence stay as they are, uninitialized in a new result."""
    _need(q, ctx, _HALF, 3, "q")
    rows, heads_q, dim = q.shape
    c, b, heads, channels = _kv4(ctx, cache, batch, rows)
    if dim != channels or heads < 1 or heads_q < 1 or heads_q % heads:
        raise TypeError(f"q: need rows x (a multiple of {heads}) x {channels}, got {tuple(q.shape)}")
    if out is None:
        out = _empty(ctx, (rows, heads_q, dim), q.dtype, q.device)
    elif _need(out, ctx, (q.dtype,), 3, "out").shape != q.shape:
        raise TypeError(f"out: need {tuple(q.shape)}, got {tuple(out.shape)}")
    if lse is not None and (tuple(_need(lse, ctx, _F32, 2, "lse").shape) != (rows, heads_q) or not lse.is_contiguous()):
        raise TypeError(f"lse: need a contiguous {(rows, heads_q)}, got {tuple(lse.shape)}")
    (q_row, q_head, _), (o_row, o_head, _) = q.stride(), out.stride()
    d = _kv4_query(q.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else 0, q_row, q_head, o_row, o_head, max_length, _FLOAT[q.dtype],
                   heads_q // heads, 1 if causal else 0, min(window, (1 << 31) - 1), dim ** -0.5 if scale is None else scale, 0)
    lib, need = load_library(), ctypes.c_int64(0)
    _check(ctx, lib.fobq_kv4_attention_workspace(ctx, c, b, d, ctypes.byref(need)))
    work = _scratch(ctx, need.value, q.device)
    _check(ctx, lib.fobq_kv4_attention(ctx, c, b, d, work.data_ptr() if work is not None else None, need.value))
    return out


# ---- a feed-forward part of experts ----------------------------------------------------------------
def _new(ctx: int, rows: int, cols: int, dtype: torch.dtype, device) -> torch.Tensor:
    """_empty for a matrix (with strides given torch takes 1.3 us for it instead of 1.6)."""
    home = _streams.get(ctx)
    if home is None or _current_stream(device.index) == home[1]:
        return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)
    return _empty(ctx, (rows, cols), dtype, device)


def _new_rows(ctx: int, rows: int, cols: int, format: torch.dtype, device):
    """_new_fp8 with a scale per row."""
    if format not in _FP8:
        raise TypeError(f"format must be float8_e4m3fn or float8_e5m2, got {format}")
    wide, blocks = (cols + 15) & -16, (cols + 127) // 128
    values, scales = _new(ctx, rows, wide, format, device), _new(ctx, blocks, rows, torch.float32, device)
    return (Fp8Matrix(values if wide == cols else values[:, :cols], scales, 1),
            _fp8_matrix(values.data_ptr(), scales.data_ptr(), rows, cols, wide, rows, 1, _FP8[format]))


def _like(t: torch.Tensor, dev: int, dtype: torch.dtype, shape):
    """The row stride of a matrix of this type and shape on the device, or None."""
    try:
        ld, one = t.stride()
        if t.dtype is dtype and t.shape == shape and t.get_device() == dev and (one == 1 or shape[1] <= 1):
            return ld if shape[0] > 1 else shape[1]
    except (AttributeError, TypeError, ValueError):
        pass
    return None


def fobq_fp8_rms_norm(ctx: int, x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
                      format: torch.dtype = torch.float8_e4m3fn, out: Optional[Fp8Matrix] = None, sum: Optional[torch.Tensor] = None,
                      norm: Optional[torch.Tensor] = None):
    """x (fp32, bf16 or fp16, rows x cols) + residual, and its root-mean-square norm times weight (cols, x's type or fp32) in 8-bit blocks: (Fp8Matrix, sum).  sum:
    x + residual, new, or into the tensor given (which may be x or residual); None without a residual if none is given.  norm: filled with the
    norm in x's type, if given.  No gradient passes it."""
    _need(x, ctx, _FLOAT, 2, "x")
    shape, dtype, device, wtype = x.shape, x.dtype, x.device, x.dtype
    rows, cols = shape
    dev = device.index
    if weight is not None:
        wtype = getattr(weight, "dtype", None)
        if (wtype is not dtype and wtype is not torch.float32) or weight.shape != (cols,) or weight.get_device() != dev or not weight.is_contiguous():
            _need(weight, ctx, (dtype, torch.float32), 1, "weight")
            raise TypeError(f"weight: need {cols} entries, got {weight.shape[0]}")
    if residual is not None and sum is None:
        sum = _new(ctx, rows, cols, dtype, device)
    lds = [cols, cols, cols]
    for i, t in enumerate((residual, sum, norm)):
        if t is not None:
            lds[i] = _like(t, dev, dtype, shape)
            if lds[i] is None:
                name = ("residual", "sum", "norm")[i]
                _need(t, ctx, (dtype,), 2, name)
                raise TypeError(f"{name}: need {rows} x {cols}, got {tuple(t.shape)}")
    out, m = _new_rows(ctx, rows, cols, format, device) if out is None else _out_fp8(ctx, out, rows, cols, format, 1, device)
    n = _norm(x.data_ptr(), residual.data_ptr() if residual is not None else 0, weight.data_ptr() if weight is not None else 0,
              sum.data_ptr() if sum is not None else 0, norm.data_ptr() if norm is not None else 0, x.stride()[0] if rows > 1 else cols, *lds,
              _FLOAT[dtype], _FLOAT[wtype], eps, 0)
    _check(ctx, load_library().fobq_fp8_rms_norm(ctx, n, m))
    return out, sum


def fobq_fp8_swiglu(ctx: int, x: torch.Tensor, format: torch.dtype = torch.float8_e4m3fn, out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
    """x (fp32, bf16 or fp16, rows x 2 cols: the gates, then the ups) -> silu(gate) * up, rows x cols, as an Fp8Matrix.  No gradient passes it."""
    _need(x, ctx, _FLOAT, 2, "x")
    rows, both = x.shape
    if both % 2:
        raise TypeError(f"x: need an even number of columns, got {both}")
    cols = both // 2
    out, m = _new_rows(ctx, rows, cols, format, x.device) if out is None else _out_fp8(ctx, out, rows, cols, format, 1, x.device)
    _check(ctx, load_library().fobq_fp8_swiglu(ctx, x.data_ptr(), _FLOAT[x.dtype], x.stride()[0] if rows > 1 else both, m))
    return out


@dataclass
class Routing:
    """Which experts each token goes to (chosen, int32, tokens x top_k; -1: none) with which weights (fp32), and where the rows of each lie: expert e has packed
    rows starts[e] .. starts[e + 1] - 1 (int32, experts + 1); pairs (int32, tokens * top_k): the pair token * top_k + slot of each packed row, -1 behind the
    last expert's; places (int32, tokens x top_k): the packed row of each pair, or -1."""
    chosen: torch.Tensor
    weights: torch.Tensor
    starts: torch.Tensor
    pairs: torch.Tensor
    places: torch.Tensor

    @staticmethod
    def empty(tokens: int, experts: int, top_k: int, device="cuda") -> "Routing":
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=device)  # noqa: E731
        return Routing(i32(tokens, top_k), torch.empty((tokens, top_k), device=device), i32(experts + 1), i32(tokens * top_k), i32(tokens, top_k))


_SCORES = {"softmax": 0, "sigmoid": 1}


def _dense(t: torch.Tensor, ctx: int, dtype: torch.dtype, shape, what: str) -> int:
    """The address of a contiguous device tensor of this type and shape."""
    home = _streams.get(ctx)
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous() and home is not None and t.get_device() == home[0]):
        got = f"{tuple(t.shape)} {t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise TypeError(f"{what}: need a contiguous {tuple(shape)} of {dtype} on the context's device, got {got}")
    return t.data_ptr()


def fobq_route(ctx: int, logits: torch.Tensor, top_k: int, *, score: str = "softmax", bias: Optional[torch.Tensor] = None, groups: int = 1, top_groups: int = 1,
               group_top: int = 2, renormalize: bool = True, scale: float = 1.0, out: Optional[Routing] = None) -> Routing:
    """logits (fp32, bf16 or fp16, tokens x experts) -> the top_k experts of each token and their weights.  score: "softmax" or "sigmoid"; bias (fp32, experts): added for
    the choice, not for the weights (-inf: never chosen, which is faster than other large negative values); groups: only the top_groups groups of neighbouring
    experts are chosen from, which count as the sum of their group_top (1 or 2) best; renormalize: the weights are relative to the sum of the chosen ones; scale: times the weights.  No gradient passes it."""
    _need(logits, ctx, _FLOAT, 2, "logits")
    tokens, experts = logits.shape
    if score not in _SCORES:
        raise TypeError(f"score must be softmax or sigmoid, got {score}")
    if not (isinstance(top_k, int) and 1 <= top_k <= min(32, experts)):
        raise TypeError(f"top_k must be in 1..{min(32, experts)}, got {top_k}")
    i32, f32, device = torch.int32, torch.float32, logits.device
    if out is None:
        # the whole numbers in one allocation: a view takes half of one's time
        size = tokens * top_k
        whole, weights = _new(ctx, 1, 3 * size + experts + 1, i32, device), _new(ctx, tokens, top_k, f32, device)
        two = (tokens, top_k), (top_k, 1)
        out = Routing(whole.as_strided(*two, 0), weights, whole.as_strided((experts + 1,), (1,), 3 * size), whole.as_strided((size,), (1,), size),
                      whole.as_strided(*two, 2 * size))
        to = _routing(out.chosen.data_ptr(), out.weights.data_ptr(), out.starts.data_ptr(), out.pairs.data_ptr(), out.places.data_ptr())
    else:
        to = _routing(_dense(out.chosen, ctx, i32, (tokens, top_k), "chosen"), _dense(out.weights, ctx, f32, (tokens, top_k), "weights"),
                      _dense(out.starts, ctx, i32, (experts + 1,), "starts"), _dense(out.pairs, ctx, i32, (tokens * top_k,), "pairs"),
                      _dense(out.places, ctx, i32, (tokens, top_k), "places"))
    r = _router(logits.data_ptr(), _dense(bias, ctx, f32, (experts,), "bias") if bias is not None else 0, tokens, logits.stride()[0] if tokens > 1 else experts,
                _FLOAT[logits.dtype], experts, top_k, _SCORES[score], groups, top_groups, group_top, 1 if renormalize else 0, scale, 0)
    lib, need = load_library(), ctypes.c_int64(0)
    _check(ctx, lib.fobq_route_workspace(ctx, tokens, experts, ctypes.byref(need)))
    work = _scratch(ctx, need.value, device)
    _check(ctx, lib.fobq_route(ctx, r, to, work.data_ptr() if work is not None else None, need.value))
    return out


@dataclass
class Fp8Experts:
    """The weights of all experts: values (float8_e4m3fn or float8_e5m2, experts x rows x cols, rows a multiple of 16 bytes apart) and scales (fp32, experts x
    ceil(cols / 128) x ceil(rows / rows_per_scale)).  expert(e) is one of them as an Fp8Matrix, for example for fp8_quantize's out."""
    values: torch.Tensor
    scales: torch.Tensor
    rows_per_scale: int = 1

    @staticmethod
    def empty(experts: int, rows: int, cols: int, format: torch.dtype = torch.float8_e4m3fn, rows_per_scale: int = 128, device="cuda") -> "Fp8Experts":
        values = torch.empty((experts, rows, (cols + 15) & -16), dtype=format, device=device)[:, :, :cols]
        return Fp8Experts(values, torch.empty((experts, (cols + 127) // 128, (rows + rows_per_scale - 1) // rows_per_scale), device=device), rows_per_scale)

    def expert(self, e: int) -> Fp8Matrix:
        return Fp8Matrix(self.values[e], self.scales[e], self.rows_per_scale)


def _experts(ctx: int, b: Fp8Experts):
    """What the library calls the weights of all experts, and how many there are, their rows and columns."""
    v, s, per = b.values, b.scales, b.rows_per_scale
    _need(v, ctx, _FP8, 3, "experts.values")
    _need(s, ctx, _F32, 3, "experts.scales")
    (count, rows, cols), (apart, ld, _), (scales_apart, ld_scales, _) = v.shape, v.stride(), s.stride()
    if per not in (1, 128) or s.shape != (count, (cols + 127) // 128, (rows + per - 1) // per):
        raise TypeError(f"experts: rows_per_scale must be 1 or 128 and scales (experts, ceil(cols / 128), ceil(rows / rows_per_scale)), got {per} and "
                        f"{tuple(s.shape)} for {tuple(v.shape)}")
    wide, sr = (cols + 15) & -16, s.shape[2]
    if rows <= 1 or not cols:
        ld = wide
    if count <= 1 or not rows or not cols:
        apart, scales_apart = 0, 0
    if wide != cols and count and rows and v.storage_offset() + (count - 1) * apart + (rows - 1) * ld + wide > v.untyped_storage().nbytes():
        raise TypeError("experts: the last row must be readable to a multiple of 16 bytes")
    return (_fp8_experts(v.data_ptr(), s.data_ptr(), rows, cols, ld, ld_scales if s.shape[1] > 1 else sr, apart, scales_apart, count, per, _FP8[v.dtype], 0),
            count, rows, cols)


def fobq_fp8_expert_matmul(ctx: int, A: Fp8Matrix, experts: Fp8Experts, routing: Routing, dtype: torch.dtype = torch.bfloat16, *, packed: bool = False,
                           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The packed rows of a routing times their experts' weights transposed -> packed rows x rows of an expert, of `dtype` (fp32, bf16 or fp16), or into `out`.  A:
    the tokens' rows, or (packed) the packed rows themselves.  Packed rows of no expert are not written (uninitialized in a new result).  Precision as
    fp8_matmul's for more than 16 rows, or better.  No gradient passes it."""
    a, m, k = _fp8(ctx, A, "A")
    b, count, n, k2 = _experts(ctx, experts)
    if k != k2:
        raise TypeError(f"A has {k} columns, the experts {k2}")
    pairs, places = _need(routing.pairs, ctx, _I32, 1, "pairs"), _need(routing.places, ctx, _I32, 2, "places")
    if places.numel() != pairs.shape[0]:
        raise TypeError(f"routing: need places tokens x top_k and as many pairs, got {tuple(places.shape)} and {tuple(pairs.shape)}")
    (tokens, top_k), rows = places.shape, pairs.shape[0]
    if m != (rows if packed else tokens):
        raise TypeError(f"A has {m} rows, need {rows if packed else tokens}: the {'packed' if packed else 'tokens'}' rows")
    starts, device = _dense(routing.starts, ctx, torch.int32, (count + 1,), "starts"), A.values.device
    if out is None:
        if dtype not in _FLOAT:
            raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
        out = _new(ctx, rows, n, dtype, device)
    else:
        _need(out, ctx, _FLOAT, 2, "out")
        if tuple(out.shape) != (rows, n):
            raise TypeError(f"out: need {rows} x {n}, got {tuple(out.shape)}")
        dtype = out.dtype
    _check(ctx, load_library().fobq_fp8_expert_matmul(ctx, a, b, starts, None if packed else _dense(pairs, ctx, torch.int32, (rows,), "pairs"), max(1, top_k), rows,
                                                      out.data_ptr(), _FLOAT[dtype], out.stride()[0] if rows > 1 else n))
    return out


def fobq_expert_sum(ctx: int, y: torch.Tensor, routing: Routing, base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y (fp32, bf16 or fp16, packed rows x cols) -> for each token base (tokens x cols, if given) + the sum over its slots of weight times row, in slot order, of y's type;
    or into `out`, which may be base.  No gradient passes it."""
    _need(y, ctx, _FLOAT, 2, "y")
    (rows, cols), dtype = y.shape, y.dtype
    shape, device = _need(routing.places, ctx, _I32, 2, "places").shape, y.device
    tokens, top_k = shape
    places, weights = _dense(routing.places, ctx, torch.int32, shape, "places"), _dense(routing.weights, ctx, torch.float32, shape, "weights")
    if out is None:
        out = _new(ctx, tokens, cols, dtype, device)
    lds = [cols, cols]
    for i, t in enumerate((out, base)):
        if t is not None:
            lds[i] = _like(t, device.index, dtype, (tokens, cols))
            if lds[i] is None:
                name = ("out", "base")[i]
                _need(t, ctx, (dtype,), 2, name)
                raise TypeError(f"{name}: need {tokens} x {cols}, got {tuple(t.shape)}")
    _check(ctx, load_library().fobq_expert_sum(ctx, y.data_ptr(), _FLOAT[dtype], rows, cols, y.stride()[0] if rows > 1 else cols, weights, places, tokens, top_k,
                                               base.data_ptr() if base is not None else None, lds[1], out.data_ptr(), lds[0]))
    return out


def FOBQ_PROFILE_STAGE(stage: int) -> int:
    return 2 << stage


def fobq_profile_enable(ctx: int, on) -> None:
    """on: False / True (every stage), or a sum of FOBQ_PROFILE_STAGE(s)."""
    _check(ctx, load_library().fobq_profile_enable(ctypes.c_void_p(ctx), int(on)))


def fobq_profile_get(ctx: int, stage: int):
    ms, n = ctypes.c_double(0.0), ctypes.c_int64(0)
    _check(ctx, load_library().fobq_profile_get(ctypes.c_void_p(ctx), stage, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def fobq_profile_reset(ctx: int) -> None:
    _check(ctx, load_library().fobq_profile_reset(ctypes.c_void_p(ctx)))


class Ctx:
    """Context manager around a fobq context bound to torch's current stream."""

    def __init__(self, device: int = 0, stream: Optional[int] = None):
        self.handle = fobq_create(device, stream)

    def close(self) -> None:
        if self.handle:
            fobq_destroy(self.handle)
            self.handle = 0

    def __enter__(self) -> "Ctx":
        return self

    def __exit__(self, *exc) -> None:
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_hessian_mode(self, mode: int) -> None:
        fobq_hessian_set_mode(self.handle, mode)

    def hessian(self, X: torch.Tensor, chunk: Optional[int] = None, H_out: Optional[torch.Tensor] = None) -> None:
        """begin / accumulate (optionally in column chunks) / finalize."""
        fobq_hessian_begin(self.handle, X.shape[0])
        n = X.shape[1]
        step = n if not chunk else chunk
        for lo in range(0, n, step):
            fobq_hessian_accumulate(self.handle, X[:, lo:lo + step])
        fobq_hessian_finalize(self.handle, H_out)

    def hessian_conv(self, maps: torch.Tensor, k: int, stride: int = 1, pad: int = 0,
                     images_per_call: Optional[int] = None, H_out: Optional[torch.Tensor] = None) -> None:
        """begin / accumulate_conv (optionally a few images per call) / finalize for a k x k convolution."""
        fobq_hessian_begin(self.handle, maps.shape[3] * k * k)
        n = maps.shape[0]
        step = n if not images_per_call else images_per_call
        for lo in range(0, n, step):
            fobq_hessian_accumulate_conv(self.handle, maps[lo:lo + step], k, stride, pad)
        fobq_hessian_finalize(self.handle, H_out)

    def quantize_layer(self, W: torch.Tensor, H: Optional[torch.Tensor] = None, **kw) -> LayerOutput:
        return fobq_quantize_layer(self.handle, W, H, **kw)

    def quantize_layers_batched(self, Ws, Hs, **kw):
        return fobq_quantize_layers_batched(self.handle, Ws, Hs, **kw)

    def finish(self) -> None:
        fobq_finish(self.handle)

    def fp8_quantize(self, X: torch.Tensor, format: torch.dtype = torch.float8_e4m3fn, rows_per_scale: int = 1, out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
        return fobq_fp8_quantize(self.handle, X, format, rows_per_scale, out)

    def fp8_from_codes(self, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, bits: int = 4, out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
        return fobq_fp8_from_codes(self.handle, codes, scales, zeros, bits, out)

    def fp8_matmul(self, A: Fp8Matrix, B: Fp8Matrix, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        return fobq_fp8_matmul(self.handle, A, B, dtype, out)

    def kv4_append(self, cache: Kv4Cache, batch: Kv4Batch, k: torch.Tensor, v: torch.Tensor) -> None:
        fobq_kv4_append(self.handle, cache, batch, k, v)

    def kv4_read(self, cache: Kv4Cache, batch: Kv4Batch, rows: int, dtype: torch.dtype = torch.bfloat16, out=None):
        return fobq_kv4_read(self.handle, cache, batch, rows, dtype, out)

    def kv4_attention(self, cache: Kv4Cache, batch: Kv4Batch, q: torch.Tensor, **kw) -> torch.Tensor:
        return fobq_kv4_attention(self.handle, cache, batch, q, **kw)

    def fp8_rms_norm(self, x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, **kw):
        return fobq_fp8_rms_norm(self.handle, x, weight, residual, **kw)

    def fp8_swiglu(self, x: torch.Tensor, format: torch.dtype = torch.float8_e4m3fn, out: Optional[Fp8Matrix] = None) -> Fp8Matrix:
        return fobq_fp8_swiglu(self.handle, x, format, out)

    def route(self, logits: torch.Tensor, top_k: int, **kw) -> Routing:
        return fobq_route(self.handle, logits, top_k, **kw)

    def fp8_expert_matmul(self, A: Fp8Matrix, experts: Fp8Experts, routing: Routing, dtype: torch.dtype = torch.bfloat16, **kw) -> torch.Tensor:
        return fobq_fp8_expert_matmul(self.handle, A, experts, routing, dtype, **kw)

    def expert_sum(self, y: torch.Tensor, routing: Routing, base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        return fobq_expert_sum(self.handle, y, routing, base, out)

    def workspace_bytes(self) -> int:
        return fobq_workspace_bytes(self.handle)

    def hessian_form(self) -> int:
        return fobq_hessian_form(self.handle)

    def obq_rows(self, W, Hinv, **kw):
        return fobq_obq_rows(self.handle, W, Hinv, **kw)

    def probe_int8_matrix_rate(self, operand_kind: int) -> float:
        return fobq_probe_int8_matrix_rate(self.handle, operand_kind)

    def stage_ms(self):
        return {name: fobq_profile_get(self.handle, i) for i, name in enumerate(STAGES)}

"""Thin Python binding of the C-ABI library (include/permuquant.h).

Argument marshalling only: every step of the path runs inside the library's HIP kernels.
torch tensors provide device memory and the current stream; nothing is computed here and
there is no CPU fallback -- if the library cannot be loaded the first call raises.  Importing this module loads the
library where it is built (host code only: the GPU is not touched).
Functions carry the names of the C entry points.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os
import warnings
from dataclasses import dataclass
from typing import List, NamedTuple, Optional, Sequence

import torch

FMT_NVFP4, FMT_INT4, FMT_INT3 = 0, 1, 2
FMT_BF16 = 3            # of a key-value cache only
FMT_MXFP4 = 4           # of the quantizers, the packed products and the products grouped by expert
LOGITS_F32, LOGITS_BF16 = 0, 1
OP_CALIB_MOMENTS, OP_SELECT_PERM, OP_QUANTIZE_WEIGHTS, OP_QUANTIZE_ACT, OP_QGEMM, OP_QUANT_ERROR, \
    OP_SELECT_PERM_OUTPUT, OP_CHANNEL_STATS, OP_ORDER = range(9)
CRIT_VARIANCE, CRIT_ABSMAX = 0, 1
MAX_ALPHAS = 15
DEFAULT_ALPHAS = (0.0, 0.2, 0.4, 0.6, 0.8, 1.0)

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libpermuquant.so")
_lib = None


class PQError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("permuquant error %d: %s" % (code, msg))
        self.code = code


class _Report(C.Structure):
    _fields_ = [("accepted", C.c_int), ("alpha_index", C.c_int), ("e_orig", C.c_double),
                ("e_best", C.c_double), ("e_cand", C.c_double * MAX_ALPHAS),
                ("sum_x2", C.c_double), ("sum_w2", C.c_double)]


class NormParams(C.Structure):
    """pq_norm_params of the header."""
    _fields_ = [("kind", C.c_int), ("perm", C.c_void_p), ("gamma", C.c_void_p), ("mod_scale", C.c_void_p),
                ("mod_shift", C.c_void_p), ("rows_per_mod", C.c_int64), ("eps", C.c_float)]


class OutputPlan(C.Structure):
    """pq_output_plan of the header."""
    _fields_ = [(n, C.c_int) for n in ("batches", "orders", "tile_m", "tile_n", "tile_waves")]


class _KVCacheStruct(C.Structure):
    """pq_kv_cache of the header."""
    _fields_ = [("fmt", C.c_int), ("group", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int), ("page", C.c_int),
                ("pages", C.c_int64), ("data", C.c_void_p), ("k_tensor_scale", C.c_void_p), ("v_tensor_scale", C.c_void_p)]


NORM_RMS, NORM_ADALN = 0, 1


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load libpermuquant.so (built in-tree by paper_2605_09503_amd.build). Raises if it is missing or another version's."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise PQError(-100, "library not built: %s (run python -m paper_2605_09503_amd.build)" % _LIB_PATH)
    try:
        lib = C.CDLL(_LIB_PATH)
        _declare(lib)
    except (OSError, AttributeError) as e:
        raise PQError(-100, "library not usable: %s (run python -m paper_2605_09503_amd.build)" % e) from e
    _lib = lib
    _bind_calls()
    return lib


def _declare(lib):
    vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
    lib.pq_last_error.restype = C.c_char_p
    lib.pq_last_error.argtypes = []
    lib.pq_version.restype = i32
    lib.pq_workspace_bytes.restype = sz
    lib.pq_workspace_bytes.argtypes = [i32, i32, i32, i64, i64, i64, i32]
    lib.pq_calib_moments.argtypes = [vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.pq_calib_moments_static.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    lib.pq_calib_moments_batched.argtypes = [C.POINTER(vp), i32, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.pq_tensor_scale.argtypes = [vp, vp, vp]
    lib.pq_tensor_scale.restype = i32
    lib.pq_select_perm.argtypes = [i32, i32, vp, vp, i64, C.POINTER(vp), i32, i64, vp, i64,
                                   C.c_float, C.c_float, C.POINTER(C.c_double), i32, C.c_double,
                                   vp, C.POINTER(_Report), vp, sz, vp]
    lib.pq_select_perm_output_error.argtypes = lib.pq_select_perm.argtypes
    lib.pq_select_perm_device_scales.argtypes = [i32, i32, vp, vp, i64, C.POINTER(vp), i32, i64, vp, i64,
                                                 vp, vp, C.POINTER(C.c_double), i32, C.c_double,
                                                 vp, C.POINTER(_Report), vp, sz, vp]
    lib.pq_quant_error.argtypes = [i32, i32, vp, i64, i64, vp, C.c_float, vp, vp, sz, vp]
    lib.pq_quantize_weights.argtypes = [i32, i32, vp, i64, i64, vp, vp, vp, vp, vp]
    lib.pq_quantize_act.argtypes = [i32, i32, vp, i64, i64, i64, vp, vp, vp, vp, vp]
    gemm_args = [i32, i32, vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, i64, vp, sz, vp]
    lib.pq_qgemm.argtypes = gemm_args
    lib.pq_qgemm_f32.argtypes = gemm_args
    lib.pq_qgemm_run.argtypes = gemm_args
    lib.pq_qgemm_prep.argtypes = [i32, i32, vp, vp, i64, i64, i64, vp, sz, vp]
    lib.pq_qgemm_tile.argtypes = [i32, i32, i64, i64, i64, C.POINTER(i32), C.POINTER(i32)]
    lib.pq_select_output_plan.argtypes = [i32, i32, i64, i64, i64, i32, i32, sz, C.POINTER(OutputPlan)]
    lib.pq_operand_bytes.restype = sz
    lib.pq_operand_bytes.argtypes = [i32, i32, i64, i64]
    lib.pq_pack_operand.argtypes = [i32, i32, vp, vp, i64, i64, vp, sz, vp]
    lib.pq_quantize_act_packed.argtypes = [i32, i32, vp, i64, i64, i64, vp, vp, sz, vp, vp, vp]
    lib.pq_int3_dense_bytes.restype = sz
    lib.pq_int3_dense_bytes.argtypes = [i64, i64]
    lib.pq_int3_pack.argtypes = [vp, i64, i64, vp, vp]
    lib.pq_int3_unpack.argtypes = [vp, i64, i64, vp, vp]
    lib.pq_pack_operand_int3.argtypes = [i32, vp, vp, i64, i64, vp, sz, vp]
    packed_args = [i32, i32, vp, vp, vp, vp, i64, i64, i64, vp, i64, vp]
    lib.pq_qgemm_packed.argtypes = packed_args
    lib.pq_qgemm_packed_f32.argtypes = packed_args
    lib.pq_qgemm_packed_bias.argtypes = [i32, i32, vp, vp, vp, vp, i64, i64, i64, vp, vp, i64, vp]
    lib.pq_calib_channel_stats.argtypes = [vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.pq_channel_statistic.argtypes = [i32, vp, vp, vp, i64, i64, vp, vp]
    lib.pq_order_by_score.argtypes = [vp, vp, i64, C.c_double, vp, vp, sz, vp]
    lib.pq_order_round_robin.argtypes = [vp, i64, i32, vp, vp]
    lib.pq_order_random.argtypes = [C.c_uint64, i64, vp, vp, sz, vp]
    lib.pq_hadamard_reorder.argtypes = [vp, vp, i64, i64, i64, vp, i64, vp]
    lib.pq_hadamard_quantize_act_packed.argtypes = [vp, i32, i32, vp, i64, i64, i64, vp, vp, sz, vp, i64, vp]
    lib.pq_dynamic_tensor_scale.argtypes = [vp, i64, i64, i64, vp, vp]
    lib.pq_norm_reorder.argtypes = [C.POINTER(NormParams), vp, i64, i64, i64, vp, i64, vp]
    lib.pq_norm_quantize_act_packed.argtypes = [C.POINTER(NormParams), i32, i32, vp, i64, i64, i64, vp, vp, sz,
                                                vp, i64, vp]
    lib.pq_kv_cache_bytes.restype = sz
    lib.pq_kv_cache_bytes.argtypes = [i32, i32, i32, i32, i32, i64]
    lib.pq_kv_write.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp, i64, vp]
    lib.pq_kv_read.argtypes = [vp, vp, i64, vp, i64, i64, vp, i64, i64, vp]
    lib.pq_attn_decode_workspace_bytes.restype = sz
    lib.pq_attn_decode_workspace_bytes.argtypes = [vp, i64, i32, i64, i64]
    lib.pq_attn_decode.argtypes = [vp, vp, i64, i64, vp, i64, vp, i64, i32, i64, i64, C.c_float, vp, i64, i64, vp, vp, sz, vp]
    lib.pq_dequantize.argtypes = [i32, i32, vp, vp, vp, i64, i64, vp, i64, vp]
    lib.pq_qgemm_grouped.argtypes = [i32, i32, vp, i64, vp, i32, vp, vp, i64, i64, i64, vp, vp, i64, vp]
    lib.pq_qgemm_grouped_tile.argtypes = [i32, i32, i32, i64, i64, i64, C.POINTER(i32), C.POINTER(i32)]
    lib.pq_moe_route_workspace_bytes.restype = sz
    lib.pq_moe_route_workspace_bytes.argtypes = [i64, i32, i32]
    lib.pq_moe_route.argtypes = [i32, vp, i64, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pq_moe_combine.argtypes = [vp, i64, i64, vp, vp, i64, i32, i64, vp, i64, vp, i64, vp]
    lib.pq_probe_stream.argtypes = [vp, sz, vp, sz, vp]
    lib.pq_qgemm_check_int_scales.argtypes = [i32, i32, vp, i64, i64, C.POINTER(C.c_int64), vp, sz, vp]
    lib.pq_probe_mfma.argtypes = [i32, vp, C.POINTER(C.c_double), vp]
    lib.pq_probe_mfma_operands.argtypes = [i32, i32, vp, vp, i64, i64, i64, i32, vp, C.POINTER(C.c_double), vp]
    for name in ("pq_calib_moments", "pq_calib_moments_batched", "pq_select_perm", "pq_quant_error", "pq_quantize_weights",
                 "pq_quantize_act", "pq_qgemm", "pq_qgemm_f32", "pq_qgemm_run", "pq_qgemm_prep", "pq_probe_stream",
                 "pq_probe_mfma", "pq_pack_operand", "pq_qgemm_packed", "pq_qgemm_packed_f32",
                 "pq_quantize_act_packed"):
        getattr(lib, name).restype = i32


def _check(rc: int):
    if rc != 0:
        _raise(rc)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The current stream's handle without the Stream object around it: building that object takes 3.0 us, this 0.2,
# where a launch takes 3 and a whole call 5.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


# ------------------------------------------------------------------------ the calls of a forward pass
# A wrapper here and ctypes cost 2 us of the 5 that a call takes, so these are marshalled by the module _pq_calls
# (csrc/pq_calls.cpp): it takes the place of the functions of these names below, which do the same and serve where the module
# is not built (it needs a host compiler and the interpreter's headers) or was built for another torch.
_CALLS = ("pq_quantize_act", "pq_quantize_act_packed", "pq_norm_quantize_act_packed", "pq_hadamard_quantize_act_packed",
          "pq_qgemm", "pq_qgemm_packed", "pq_qgemm_packed_f32", "pq_qgemm_packed_bias", "pq_calib_moments", "pq_kv_write",
          "pq_kv_read", "pq_attn_decode", "pq_dequantize", "pq_qgemm_grouped", "pq_moe_route", "pq_moe_combine")
_CALLS_PATH = os.path.join(os.path.dirname(_LIB_PATH), "_pq_calls.so")
_calls = None           # the module, or False where it cannot be had


def _raise(rc: int):
    raise PQError(rc, load().pq_last_error().decode())


def _refuse(msg: str):
    raise PQError(-2, msg)


def _new_operand(fmt: int, group: int, rows: int, K: int, like: torch.Tensor) -> torch.Tensor:
    return torch.empty(max(pq_operand_bytes(fmt, group, rows, K), 16), dtype=torch.uint8, device=like.device)


def _new_attn_workspace(cache, seqs: int, q_heads: int, max_len: int, window: int) -> torch.Tensor:
    return pq_attn_decode_workspace(cache, seqs, q_heads, max_len, window)


def _new_route_workspace(tokens: int, experts: int, k: int, like: torch.Tensor) -> torch.Tensor:
    return pq_moe_route_workspace(tokens, experts, k, like.device)


def _new_route(tokens: int, experts: int, k: int, like: torch.Tensor):
    return alloc_route(tokens, experts, k, like.device)


def _new_workspace(op: int, fmt: int, group: int, M: int, N: int, K: int, n_batches: int, like: torch.Tensor):
    return _workspace(pq_workspace_bytes(op, fmt, group, M, N, K, n_batches), like.device)


def _bind_calls():
    """Puts _pq_calls in place of the functions of its names, once; without it they stay and a warning says so."""
    global _calls
    if _calls is not None:
        return
    _calls = False
    try:
        if not os.path.exists(_CALLS_PATH):
            raise ImportError("not built: " + _CALLS_PATH)
        loader = importlib.machinery.ExtensionFileLoader("_pq_calls", _CALLS_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_pq_calls", loader))
        loader.exec_module(module)
        module.bind(_raise, _new_operand, _new_workspace, _refuse, _new_attn_workspace, _new_route_workspace, _new_route)
        bound = {name: getattr(module, name) for name in _CALLS}
    except (ImportError, AttributeError, OSError) as e:
        warnings.warn("the native binding of the hot calls cannot be used, ctypes takes 2 us more a call (%s); build it with "
                      "python -m paper_2605_09503_amd.build" % e, RuntimeWarning)
        return
    _calls = module
    globals().update(bound)


def pq_last_error() -> str:
    return load().pq_last_error().decode()


def pq_version() -> int:
    return load().pq_version()


def pq_workspace_bytes(op: int, fmt: int, group: int, M: int, N: int, K: int, n_batches: int = 0) -> int:
    return int(load().pq_workspace_bytes(op, fmt, group, M, N, K, n_batches))


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def pq_calib_moments(x: torch.Tensor, sumsq: torch.Tensor, absmax: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, rows: Optional[int] = None,
                     K: Optional[int] = None, ld: Optional[int] = None) -> None:
    """sumsq[K] (float64, in/out) += column sums of squares of bf16 x[rows, ld]."""
    rows = x.shape[0] if rows is None else rows
    K = x.shape[1] if K is None else K
    ld = x.stride(0) if ld is None else ld
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(OP_CALIB_MOMENTS, 0, 0, rows, 0, K, 1), x.device)
    _check(load().pq_calib_moments(_ptr(x), rows, K, ld, _ptr(sumsq), _ptr(absmax), _ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream()))


STATIC_SCRATCH_BYTES = 3 << 20      # PQ_STATIC_SCRATCH_BYTES of the header


def pq_calib_moments_static(x: torch.Tensor, sumsq: torch.Tensor, absmax: Optional[torch.Tensor] = None,
                            rows: Optional[int] = None, K: Optional[int] = None,
                            ld: Optional[int] = None) -> None:
    """pq_calib_moments with the partial sums in scratch memory the library holds itself: the call
    takes no workspace and allocates nothing."""
    rows = x.shape[0] if rows is None else rows
    K = x.shape[1] if K is None else K
    ld = x.stride(0) if ld is None else ld
    _check(load().pq_calib_moments_static(_ptr(x), rows, K, ld, _ptr(sumsq), _ptr(absmax), _stream()))


def pq_calib_moments_batched(xs: Sequence[torch.Tensor], sumsq: torch.Tensor,
                             absmax: Optional[torch.Tensor] = None,
                             workspace: Optional[torch.Tensor] = None) -> None:
    """sumsq[K] += column sums of squares over all batches (equal shapes), one launch."""
    rows, K = xs[0].shape
    ld = xs[0].stride(0)
    nb = len(xs)
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(OP_CALIB_MOMENTS, 0, 0, rows, 0, K, nb), xs[0].device)
    ptrs = (C.c_void_p * nb)(*[x.data_ptr() for x in xs])
    _check(load().pq_calib_moments_batched(ptrs, nb, rows, K, ld, _ptr(sumsq), _ptr(absmax), _ptr(workspace),
                                           0 if workspace is None else workspace.numel(), _stream()))


def pq_tensor_scale(absmax: torch.Tensor, tensor_scale_out: torch.Tensor) -> None:
    """NVFP4 per-tensor scale T = fl32(absmax / 2688), computed on the device."""
    _check(load().pq_tensor_scale(_ptr(absmax), _ptr(tensor_scale_out), _stream()))


@dataclass
class SelectReport:
    accepted: bool
    alpha_index: int
    e_orig: float
    e_best: float
    e_cand: List[float]
    sum_x2: float
    sum_w2: float


def _select(entry: str, op: int, fmt, group, act_sumsq, w_sumsq, x_calib, w, act_tensor_scale, w_tensor_scale,
            perm_out, alphas, tau, workspace) -> SelectReport:
    M, K = x_calib[0].shape
    N = w.shape[0]
    nb = len(x_calib)
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(op, fmt, group, M, N, K, nb), w.device)
    ptrs = (C.c_void_p * nb)(*[xb.data_ptr() for xb in x_calib])
    al = (C.c_double * len(alphas))(*[float(a) for a in alphas])
    rep = _Report()
    if entry == "pq_select_perm_device_scales":
        ta, tw = _ptr(act_tensor_scale), _ptr(w_tensor_scale)
    else:
        ta, tw = float(act_tensor_scale), float(w_tensor_scale)
    _check(getattr(load(), entry)(fmt, group, _ptr(act_sumsq), _ptr(w_sumsq), K, ptrs, nb, M, _ptr(w), N,
                                  ta, tw, al, len(alphas),
                                  float(tau), _ptr(perm_out), C.byref(rep), _ptr(workspace),
                                  0 if workspace is None else workspace.numel(), _stream()))
    return SelectReport(bool(rep.accepted), rep.alpha_index, rep.e_orig, rep.e_best,
                        [rep.e_cand[j] for j in range(len(alphas))], rep.sum_x2, rep.sum_w2)


def pq_select_perm(fmt: int, group: int, act_sumsq: torch.Tensor, w_sumsq: torch.Tensor,
                   x_calib: Sequence[torch.Tensor], w: torch.Tensor, act_tensor_scale: float,
                   w_tensor_scale: float, perm_out: torch.Tensor,
                   alphas: Sequence[float] = DEFAULT_ALPHAS, tau: float = 0.0,
                   workspace: Optional[torch.Tensor] = None) -> SelectReport:
    return _select("pq_select_perm", OP_SELECT_PERM, fmt, group, act_sumsq, w_sumsq, x_calib, w,
                   act_tensor_scale, w_tensor_scale, perm_out, alphas, tau, workspace)


def pq_select_perm_device_scales(fmt: int, group: int, act_sumsq: torch.Tensor, w_sumsq: torch.Tensor,
                                 x_calib: Sequence[torch.Tensor], w: torch.Tensor,
                                 act_tensor_scale: Optional[torch.Tensor], w_tensor_scale: Optional[torch.Tensor],
                                 perm_out: torch.Tensor, alphas: Sequence[float] = DEFAULT_ALPHAS, tau: float = 0.0,
                                 workspace: Optional[torch.Tensor] = None) -> SelectReport:
    """pq_select_perm with the NVFP4 tensor scales as device floats (no host copy needed before the call)."""
    return _select("pq_select_perm_device_scales", OP_SELECT_PERM, fmt, group, act_sumsq, w_sumsq, x_calib, w,
                   act_tensor_scale, w_tensor_scale, perm_out, alphas, tau, workspace)


def pq_select_perm_output_error(fmt: int, group: int, act_sumsq: torch.Tensor, w_sumsq: torch.Tensor,
                                x_calib: Sequence[torch.Tensor], w: torch.Tensor, act_tensor_scale: float,
                                w_tensor_scale: float, perm_out: torch.Tensor,
                                alphas: Sequence[float] = DEFAULT_ALPHAS, tau: float = 0.0,
                                workspace: Optional[torch.Tensor] = None) -> SelectReport:
    """The selection with the relative error of the layer's output as the metric."""
    return _select("pq_select_perm_output_error", OP_SELECT_PERM_OUTPUT, fmt, group, act_sumsq, w_sumsq, x_calib, w,
                   act_tensor_scale, w_tensor_scale, perm_out, alphas, tau, workspace)


def pq_select_output_plan(fmt: int, group: int, M: int, N: int, K: int, n_batches: int, n_alpha: int,
                          workspace_bytes: Optional[int] = None) -> OutputPlan:
    """The launches of pq_select_perm_output_error with a workspace of that size (default: what pq_workspace_bytes says)."""
    if workspace_bytes is None:
        workspace_bytes = pq_workspace_bytes(OP_SELECT_PERM_OUTPUT, fmt, group, M, N, K, n_batches)
    plan = OutputPlan()
    _check(load().pq_select_output_plan(fmt, group, M, N, K, n_batches, n_alpha, workspace_bytes, C.byref(plan)))
    return plan


def pq_quant_error(fmt: int, group: int, x: torch.Tensor, perm: Optional[torch.Tensor],
                   tensor_scale: float, err_out: torch.Tensor,
                   workspace: Optional[torch.Tensor] = None) -> None:
    rows, K = x.shape
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(OP_QUANT_ERROR, fmt, group, rows, 0, K), x.device)
    _check(load().pq_quant_error(fmt, group, _ptr(x), rows, K, _ptr(perm), float(tensor_scale),
                                 _ptr(err_out), _ptr(workspace),
                                 0 if workspace is None else workspace.numel(), _stream()))


def pq_quantize_weights(fmt: int, group: int, w: torch.Tensor, perm: Optional[torch.Tensor],
                        codes: torch.Tensor, scales: torch.Tensor, tensor_scale_out: torch.Tensor) -> None:
    N, K = w.shape
    _check(load().pq_quantize_weights(fmt, group, _ptr(w), N, K, _ptr(perm), _ptr(codes), _ptr(scales),
                                      _ptr(tensor_scale_out), _stream()))


def pq_quantize_act(fmt: int, group: int, x: torch.Tensor, perm: Optional[torch.Tensor],
                    tensor_scale: Optional[torch.Tensor], codes: torch.Tensor, scales: torch.Tensor,
                    M: Optional[int] = None, K: Optional[int] = None, ld: Optional[int] = None) -> None:
    M = x.shape[0] if M is None else M
    K = x.shape[1] if K is None else K
    ld = x.stride(0) if ld is None else ld
    _check(load().pq_quantize_act(fmt, group, _ptr(x), M, K, ld, _ptr(perm), _ptr(tensor_scale),
                                  _ptr(codes), _ptr(scales), _stream()))


def _gemm(fn, fmt, group, a_codes, a_scales, a_ts, w_codes, w_scales, w_ts, y, workspace, M, N, K, ldy):
    M = a_codes.shape[0] if M is None else M
    K = a_codes.shape[1] * 2 if K is None else K
    N = w_codes.shape[0] if N is None else N
    ldy = y.stride(0) if ldy is None else ldy
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(OP_QGEMM, fmt, group, M, N, K), a_codes.device)
    _check(fn(fmt, group, _ptr(a_codes), _ptr(a_scales), _ptr(a_ts), _ptr(w_codes), _ptr(w_scales),
              _ptr(w_ts), M, N, K, _ptr(y), ldy, _ptr(workspace),
              0 if workspace is None else workspace.numel(), _stream()))


def pq_qgemm(fmt: int, group: int, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
             w_tensor_scale, y: torch.Tensor, workspace: Optional[torch.Tensor] = None,
             M=None, N=None, K=None, ldy=None) -> None:
    """y[M, N] (bf16) = dequant(A) @ dequant(W)^T."""
    _gemm(load().pq_qgemm, fmt, group, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
          w_tensor_scale, y, workspace, M, N, K, ldy)


def pq_qgemm_prep(fmt: int, group: int, a_scales, w_scales, M: int, N: int, K: int,
                  workspace: Optional[torch.Tensor]) -> None:
    """Scale preparation half of pq_qgemm (INT formats; no-op for NVFP4)."""
    _check(load().pq_qgemm_prep(fmt, group, _ptr(a_scales), _ptr(w_scales), M, N, K, _ptr(workspace),
                                0 if workspace is None else workspace.numel(), _stream()))


def pq_qgemm_run(fmt: int, group: int, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
                 w_tensor_scale, y: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                 M=None, N=None, K=None, ldy=None) -> None:
    """Product half of pq_qgemm: the workspace must have been filled by pq_qgemm_prep or left by pq_qgemm."""
    _gemm(load().pq_qgemm_run, fmt, group, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
          w_tensor_scale, y, workspace, M, N, K, ldy)


def pq_qgemm_f32(fmt: int, group: int, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
                 w_tensor_scale, y: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                 M=None, N=None, K=None, ldy=None) -> None:
    """Same product, fp32 output (accumulator before the bf16 rounding)."""
    _gemm(load().pq_qgemm_f32, fmt, group, a_codes, a_scales, a_tensor_scale, w_codes, w_scales,
          w_tensor_scale, y, workspace, M, N, K, ldy)


def pq_qgemm_tile(fmt: int, group: int, M: int, N: int, K: int):
    """(rows, columns) of the output tile that a product of this shape takes."""
    m, n = C.c_int(), C.c_int()
    _check(load().pq_qgemm_tile(fmt, group, M, N, K, C.byref(m), C.byref(n)))
    return m.value, n.value


def pq_operand_bytes(fmt: int, group: int, rows: int, K: int) -> int:
    return int(load().pq_operand_bytes(fmt, group, rows, K))


def pq_pack_operand(fmt: int, group: int, codes: torch.Tensor, scales: torch.Tensor,
                    operand: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Stored quantizer output -> the GEMM's panel layout (allocates the buffer unless given)."""
    rows, K = codes.shape[0], codes.shape[1] * 2
    if operand is None:
        operand = torch.empty(max(pq_operand_bytes(fmt, group, rows, K), 16), dtype=torch.uint8, device=codes.device)
    _check(load().pq_pack_operand(fmt, group, _ptr(codes), _ptr(scales), rows, K, _ptr(operand),
                                  operand.numel(), _stream()))
    return operand


def pq_int3_dense_bytes(rows: int, K: int) -> int:
    return int(load().pq_int3_dense_bytes(rows, K))


def pq_int3_pack(codes: torch.Tensor, dense: Optional[torch.Tensor] = None) -> torch.Tensor:
    """INT3 codes in nibbles [rows, K/2] -> dense 3-bit storage [rows, 3K/8] (allocates unless given)."""
    rows, K = codes.shape[0], codes.shape[1] * 2
    if dense is None:
        dense = torch.empty((rows, K // 8 * 3), dtype=torch.uint8, device=codes.device)
    _check(load().pq_int3_pack(_ptr(codes), rows, K, _ptr(dense), _stream()))
    return dense


def pq_int3_unpack(dense: torch.Tensor, K: int, codes: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Dense 3-bit storage [rows, 3K/8] -> nibbles [rows, K/2] (allocates unless given)."""
    rows = dense.shape[0]
    if codes is None:
        codes = torch.empty((rows, K // 2), dtype=torch.uint8, device=dense.device)
    _check(load().pq_int3_unpack(_ptr(dense), rows, K, _ptr(codes), _stream()))
    return codes


def pq_pack_operand_int3(group: int, dense: torch.Tensor, scales: torch.Tensor, K: int,
                         operand: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Dense 3-bit codes + scales -> the GEMM's panel layout (allocates the buffer unless given)."""
    rows = dense.shape[0]
    if operand is None:
        operand = torch.empty(max(pq_operand_bytes(FMT_INT3, group, rows, K), 16), dtype=torch.uint8,
                              device=dense.device)
    _check(load().pq_pack_operand_int3(group, _ptr(dense), _ptr(scales), rows, K, _ptr(operand),
                                       operand.numel(), _stream()))
    return operand


def pq_quantize_act_packed(fmt: int, group: int, x: torch.Tensor, tensor_scale: Optional[torch.Tensor],
                           operand: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
                           scales: Optional[torch.Tensor] = None, K: Optional[int] = None) -> torch.Tensor:
    """Dynamic activation quantization straight into the GEMM's panel layout."""
    M = x.shape[0]
    K = x.shape[1] if K is None else K
    if operand is None:
        operand = _new_operand(fmt, group, M, K, x)
    _check(load().pq_quantize_act_packed(fmt, group, _ptr(x), M, K, x.stride(0), _ptr(tensor_scale),
                                         _ptr(operand), operand.numel(), _ptr(codes), _ptr(scales), _stream()))
    return operand


def pq_calib_channel_stats(x: torch.Tensor, total: Optional[torch.Tensor], absmax: Optional[torch.Tensor],
                           K: Optional[int] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Per channel: sum (fp64, accumulated into `total`) and largest magnitude (fp32, max into `absmax`)."""
    rows = x.shape[0]
    K = x.shape[1] if K is None else K
    if workspace is None:
        workspace = _workspace(pq_workspace_bytes(OP_CHANNEL_STATS, 0, 0, rows, 0, K), x.device)
    _check(load().pq_calib_channel_stats(_ptr(x), rows, K, x.stride(0), _ptr(total), _ptr(absmax), _ptr(workspace),
                                         workspace.numel(), _stream()))


def pq_channel_statistic(kind: int, total, sumsq, absmax, n_rows: int, out: torch.Tensor) -> torch.Tensor:
    _check(load().pq_channel_statistic(kind, _ptr(total), _ptr(sumsq), _ptr(absmax), n_rows, out.numel(), _ptr(out),
                                       _stream()))
    return out


def _order_ws(K: int, device, workspace):
    return workspace if workspace is not None else _workspace(pq_workspace_bytes(OP_ORDER, 0, 0, 0, 0, K), device)


def pq_order_by_score(act_stat: torch.Tensor, w_stat: torch.Tensor, alpha: float, perm_out: torch.Tensor,
                      workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    K = act_stat.numel()
    ws = _order_ws(K, act_stat.device, workspace)
    _check(load().pq_order_by_score(_ptr(act_stat), _ptr(w_stat), K, float(alpha), _ptr(perm_out), _ptr(ws),
                                    ws.numel(), _stream()))
    return perm_out


def pq_order_round_robin(order: torch.Tensor, group: int, perm_out: torch.Tensor) -> torch.Tensor:
    _check(load().pq_order_round_robin(_ptr(order), order.numel(), group, _ptr(perm_out), _stream()))
    return perm_out


def pq_order_random(seed: int, perm_out: torch.Tensor, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    K = perm_out.numel()
    ws = _order_ws(K, perm_out.device, workspace)
    _check(load().pq_order_random(int(seed), K, _ptr(perm_out), _ptr(ws), ws.numel(), _stream()))
    return perm_out


def pq_dynamic_tensor_scale(x: torch.Tensor, tensor_scale_out: Optional[torch.Tensor] = None,
                            K: Optional[int] = None) -> torch.Tensor:
    """T = max|x| / 2688 of the live tensor, left on the device (first pass of a dynamic NVFP4 scale)."""
    if tensor_scale_out is None:
        tensor_scale_out = torch.empty(1, dtype=torch.float32, device=x.device)
    _check(load().pq_dynamic_tensor_scale(_ptr(x), x.shape[0], x.shape[1] if K is None else K, x.stride(0),
                                          _ptr(tensor_scale_out), _stream()))
    return tensor_scale_out


def _norm_params(kind, perm, gamma, mod_scale, mod_shift, rows_per_mod, eps) -> "NormParams":
    raw = [None if t is None else t.data_ptr() for t in (perm, gamma, mod_scale, mod_shift)]
    return NormParams(int(kind), raw[0], raw[1], raw[2], raw[3], int(rows_per_mod), float(eps))


def pq_norm_reorder(kind: int, x: torch.Tensor, eps: float, perm: Optional[torch.Tensor] = None,
                    gamma: Optional[torch.Tensor] = None, mod_scale: Optional[torch.Tensor] = None,
                    mod_shift: Optional[torch.Tensor] = None, rows_per_mod: int = 0,
                    y: Optional[torch.Tensor] = None, K: Optional[int] = None) -> torch.Tensor:
    """RMSNorm / modulated LayerNorm whose output comes out in the channel order `perm` (bf16 [M, K])."""
    M = x.shape[0]
    K = x.shape[1] if K is None else K
    if y is None:
        y = torch.empty((M, K), dtype=torch.bfloat16, device=x.device)
    p = _norm_params(kind, perm, gamma, mod_scale, mod_shift, rows_per_mod, eps)
    _check(load().pq_norm_reorder(C.byref(p), _ptr(x), M, K, x.stride(0), _ptr(y), y.stride(0), _stream()))
    return y


def pq_norm_quantize_act_packed(kind: int, fmt: int, group: int, x: torch.Tensor, eps: float,
                                tensor_scale: Optional[torch.Tensor], perm: Optional[torch.Tensor] = None,
                                gamma: Optional[torch.Tensor] = None, mod_scale: Optional[torch.Tensor] = None,
                                mod_shift: Optional[torch.Tensor] = None, rows_per_mod: int = 0,
                                operand: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                                K: Optional[int] = None) -> torch.Tensor:
    """pq_norm_reorder feeding the activation quantizer directly: returns the GEMM operand."""
    M = x.shape[0]
    K = x.shape[1] if K is None else K
    if operand is None:
        operand = _new_operand(fmt, group, M, K, x)
    p = _norm_params(kind, perm, gamma, mod_scale, mod_shift, rows_per_mod, eps)
    _check(load().pq_norm_quantize_act_packed(C.byref(p), fmt, group, _ptr(x), M, K, x.stride(0),
                                              _ptr(tensor_scale), _ptr(operand), operand.numel(), _ptr(y),
                                              0 if y is None else y.stride(0), _stream()))
    return operand


def pq_hadamard_reorder(x: torch.Tensor, perm: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                        K: Optional[int] = None) -> torch.Tensor:
    """x H with the columns of the result in the order `perm` (bf16 [M, K])."""
    M = x.shape[0]
    K = x.shape[1] if K is None else K
    if y is None:
        y = torch.empty((M, K), dtype=torch.bfloat16, device=x.device)
    _check(load().pq_hadamard_reorder(_ptr(perm), _ptr(x), M, K, x.stride(0), _ptr(y), y.stride(0), _stream()))
    return y


def pq_hadamard_quantize_act_packed(fmt: int, group: int, x: torch.Tensor, tensor_scale: Optional[torch.Tensor],
                                    perm: Optional[torch.Tensor] = None, operand: Optional[torch.Tensor] = None,
                                    y: Optional[torch.Tensor] = None, K: Optional[int] = None) -> torch.Tensor:
    """The rotation feeding the activation quantizer directly: returns the GEMM operand."""
    M = x.shape[0]
    K = x.shape[1] if K is None else K
    if operand is None:
        operand = _new_operand(fmt, group, M, K, x)
    _check(load().pq_hadamard_quantize_act_packed(_ptr(perm), fmt, group, _ptr(x), M, K, x.stride(0),
                                                  _ptr(tensor_scale), _ptr(operand), operand.numel(), _ptr(y),
                                                  0 if y is None else y.stride(0), _stream()))
    return operand


def _gemm_packed(fn, fmt, group, a_operand, a_ts, w_operand, w_ts, y, M, N, K, ldy):
    _check(fn(fmt, group, _ptr(a_operand), _ptr(a_ts), _ptr(w_operand), _ptr(w_ts), M, N, K, _ptr(y),
              y.stride(0) if ldy is None else ldy, _stream()))


def pq_qgemm_packed(fmt: int, group: int, a_operand, a_tensor_scale, w_operand, w_tensor_scale,
                    y: torch.Tensor, M: int, N: int, K: int, ldy=None) -> None:
    """y[M, N] (bf16) = the product of two packed operands."""
    _gemm_packed(load().pq_qgemm_packed, fmt, group, a_operand, a_tensor_scale, w_operand, w_tensor_scale,
                 y, M, N, K, ldy)


def pq_qgemm_packed_bias(fmt: int, group: int, a_operand, a_tensor_scale, w_operand, w_tensor_scale,
                         bias: torch.Tensor, y: torch.Tensor, M: int, N: int, K: int, ldy=None) -> None:
    """The packed product plus the layer's bias (bf16 [N]), added before the rounding to bf16."""
    _check(load().pq_qgemm_packed_bias(fmt, group, _ptr(a_operand), _ptr(a_tensor_scale), _ptr(w_operand),
                                       _ptr(w_tensor_scale), M, N, K, _ptr(bias), _ptr(y),
                                       y.stride(0) if ldy is None else ldy, _stream()))


def pq_qgemm_packed_f32(fmt: int, group: int, a_operand, a_tensor_scale, w_operand, w_tensor_scale,
                        y: torch.Tensor, M: int, N: int, K: int, ldy=None) -> None:
    """The packed product in fp32, before the rounding to bf16."""
    _gemm_packed(load().pq_qgemm_packed_f32, fmt, group, a_operand, a_tensor_scale, w_operand,
                 w_tensor_scale, y, M, N, K, ldy)


def pq_probe_stream(src: torch.Tensor, read_bytes: int, dst: torch.Tensor, write_bytes: int) -> None:
    """Plain streaming kernel: reads read_bytes of src, writes write_bytes of dst."""
    _check(load().pq_probe_stream(_ptr(src), read_bytes, _ptr(dst), write_bytes, _stream()))


def pq_probe_mfma(iters: int, sink: torch.Tensor) -> float:
    """Matrix-pipe-only loop on every compute unit; returns the floating-point operations issued."""
    flops = C.c_double(0.0)
    _check(load().pq_probe_mfma(iters, _ptr(sink), C.byref(flops), _stream()))
    return flops.value


def pq_qgemm_check_int_scales(fmt: int, group: int, scales: torch.Tensor, rows: int, K: int) -> int:
    """Number of INT group scales the product kernel would not reproduce exactly (synchronises)."""
    ws = torch.empty(256, dtype=torch.uint8, device=scales.device)
    bad = C.c_int64(-1)
    _check(load().pq_qgemm_check_int_scales(fmt, group, _ptr(scales), rows, K, C.byref(bad), _ptr(ws), ws.numel(),
                                            _stream()))
    return bad.value


def pq_probe_mfma_operands(fmt: int, group: int, a_operand: torch.Tensor, w_operand: torch.Tensor, M: int, N: int,
                           K: int, iters: int, sink: torch.Tensor) -> float:
    """Matrix-pipe-only loop on fragments of the two packed operands; returns the operations issued."""
    flops = C.c_double(0.0)
    _check(load().pq_probe_mfma_operands(fmt, group, _ptr(a_operand), _ptr(w_operand), M, N, K, iters, _ptr(sink),
                                         C.byref(flops), _stream()))
    return flops.value


# ------------------------------------------------------------------------ key-value cache and the attention over it
@dataclass(frozen=True)
class KVCache:
    """A key-value cache (pq_kv_cache of the header): `data` holds pages * page tokens of kv_heads heads."""
    fmt: int
    group: int
    kv_heads: int
    head_dim: int
    page: int
    pages: int
    data: torch.Tensor
    k_tensor_scale: Optional[torch.Tensor] = None
    v_tensor_scale: Optional[torch.Tensor] = None

    def __post_init__(self):
        need = pq_kv_cache_bytes(self.fmt, self.group, self.kv_heads, self.head_dim, self.page, self.pages)
        if need == 0:
            raise PQError(-2, pq_last_error())
        if self.data.dtype != torch.uint8 or not self.data.is_contiguous() or self.data.numel() < need:
            _refuse("a cache of %d contiguous bytes is needed" % need)
        for t in (self.k_tensor_scale, self.v_tensor_scale):
            if self.fmt == FMT_NVFP4 and (t is None or t.dtype != torch.float32 or t.numel() != 1 or t.device != self.data.device):
                _refuse("NVFP4 needs the tensor scales of keys and values, one float32 each, on the cache's device")
        struct = _KVCacheStruct(self.fmt, self.group, self.kv_heads, self.head_dim, self.page, self.pages, self.data.data_ptr(),
                                _ptr(self.k_tensor_scale), _ptr(self.v_tensor_scale))
        object.__setattr__(self, "_struct", struct)
        object.__setattr__(self, "_address", C.addressof(struct))


def pq_kv_cache_bytes(fmt: int, group: int, kv_heads: int, head_dim: int, page: int, pages: int) -> int:
    return int(load().pq_kv_cache_bytes(fmt, group, kv_heads, head_dim, page, pages))


def alloc_kv_cache(fmt: int, group: int, kv_heads: int, head_dim: int, page: int, pages: int,
                   k_tensor_scale: Optional[torch.Tensor] = None, v_tensor_scale: Optional[torch.Tensor] = None,
                   device="cuda") -> KVCache:
    """A cache of `pages` pages of `page` tokens; the tensor scales (float32 [1]) are NVFP4's."""
    need = pq_kv_cache_bytes(fmt, group, kv_heads, head_dim, page, pages)
    if need == 0:
        raise PQError(-2, pq_last_error())
    return KVCache(fmt, group, kv_heads, head_dim, page, pages, torch.empty(need, dtype=torch.uint8, device=device),
                   k_tensor_scale, v_tensor_scale)


def _head_rows(cache: KVCache, name: str, t: torch.Tensor, rows: int, heads: int):
    """(pointer, stride of a row, stride of a head) of bf16 [rows, heads, head_dim]; strides of one row or head do not matter."""
    if t.dtype != torch.bfloat16 or tuple(t.shape) != (rows, heads, cache.head_dim) or t.stride(2) != 1 or t.device != cache.data.device:
        _refuse("%s must be bfloat16 [%d, %d, %d] with adjacent channels, on the cache's device" % (name, rows, heads, cache.head_dim))
    return t.data_ptr(), t.stride(0) if rows > 1 else 0, t.stride(1) if heads > 1 else 0


def _indices(cache: KVCache, name: str, t: torch.Tensor, dtype, dims: int):
    if t.dtype != dtype or t.dim() != dims or (t.numel() > 1 and t.stride(-1) != 1) or t.device != cache.data.device:
        _refuse("%s must be %s with %d dimension%s, the last one contiguous, on the cache's device" % (name, dtype, dims, "s" * (dims > 1)))
    return t.data_ptr()


def _stream_of(cache: KVCache):
    if not cache.data.is_cuda:
        _refuse("the cache must lie in GPU memory")
    return _stream()


def pq_kv_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Quantizes keys and values, bf16 [n, kv_heads, head_dim] (slices of a fused projection's rows are), into the slots (int64 [n])."""
    s = _indices(cache, "slots", slots, torch.int64, 1)
    n = slots.shape[0]
    kr, vr = (_head_rows(cache, name, t, n, cache.kv_heads) for name, t in (("k", k), ("v", v)))
    _check(load().pq_kv_write(cache._address, *kr, *vr, s, n, _stream_of(cache)))


def pq_kv_read(cache: KVCache, slots: torch.Tensor, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
    """(k, v) of the slots as bf16 [n, kv_heads, head_dim] (allocated unless given)."""
    s = _indices(cache, "slots", slots, torch.int64, 1)
    n = slots.shape[0]
    k, v = (torch.empty((n, cache.kv_heads, cache.head_dim), dtype=torch.bfloat16, device=cache.data.device) if t is None else t
            for t in (k, v))
    kr, vr = (_head_rows(cache, name, t, n, cache.kv_heads) for name, t in (("k", k), ("v", v)))
    _check(load().pq_kv_read(cache._address, s, n, *kr, *vr, _stream_of(cache)))
    return k, v


ATTN_DECODE_ZERO_BYTES = 4096       # PQ_ATTN_DECODE_ZERO_BYTES of the header


def pq_attn_decode_workspace_bytes(cache: KVCache, seqs: int, q_heads: int, max_len: int, window: int = 0) -> int:
    return int(load().pq_attn_decode_workspace_bytes(cache._address, seqs, q_heads, max_len, window))


def pq_attn_decode_workspace(cache: KVCache, seqs: int, q_heads: int, max_len: int, window: int = 0) -> torch.Tensor:
    """A workspace for pq_attn_decode with these arguments, or smaller ones: for one stream, call after call."""
    need = pq_attn_decode_workspace_bytes(cache, seqs, q_heads, max_len, window)
    if need == 0:
        raise PQError(-2, pq_last_error())
    ws = torch.empty(need, dtype=torch.uint8, device=cache.data.device)
    ws[:ATTN_DECODE_ZERO_BYTES].zero_()
    return ws


def pq_attn_decode(cache: KVCache, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, max_len: int, scale: float,
                   out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, window: int = 0,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of one new token a sequence, q bf16 [seqs, q_heads, head_dim], over the lengths[b] (int32) tokens whose pages
    table[b] (int32) names; out like q (allocated unless given), lse float32 [seqs, q_heads].  max_len: no sequence is longer."""
    if q.dim() != 3:
        _refuse("q must be bfloat16 [seqs, q_heads, head_dim]")
    seqs, q_heads = q.shape[0], q.shape[1]
    qr = _head_rows(cache, "q", q, seqs, q_heads)
    tab, n = _indices(cache, "table", table, torch.int32, 2), _indices(cache, "lengths", lengths, torch.int32, 1)
    if table.shape[0] != seqs or lengths.shape[0] != seqs or table.shape[1] * cache.page < max_len:
        _refuse("table and lengths must have a row for each of %d sequences, and table the pages of %d tokens" % (seqs, max_len))
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (seqs, q_heads) or not lse.is_contiguous()
                            or lse.device != cache.data.device):
        _refuse("lse must be contiguous float32 [%d, %d] on the cache's device" % (seqs, q_heads))
    if out is None:
        out = torch.empty((seqs, q_heads, cache.head_dim), dtype=torch.bfloat16, device=cache.data.device)
    outr = _head_rows(cache, "out", out, seqs, q_heads)
    if workspace is None:
        workspace = pq_attn_decode_workspace(cache, seqs, q_heads, max_len, window)
    if not workspace.is_contiguous() or workspace.device != cache.data.device:
        _refuse("workspace must be contiguous, on the cache's device")
    _check(load().pq_attn_decode(cache._address, *qr, tab, table.stride(0) if seqs > 1 else table.shape[1], n, seqs, q_heads, max_len, window,
                                 float(scale), *outr, _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream_of(cache)))
    return out


# ------------------------------------------------------------------------ reading back, products by expert, routing
def pq_dequantize(fmt: int, group: int, codes: torch.Tensor, scales: torch.Tensor, tensor_scale: Optional[torch.Tensor] = None,
                  y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that stored codes [rows, K/2] and scales stand for, bf16 [rows, K] (allocated unless given)."""
    if codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_contiguous():
        _refuse("codes must be contiguous uint8 [rows, K/2]")
    rows, K = codes.shape[0], codes.shape[1] * 2
    _on_current_device("codes", codes)
    if scales.dtype != scale_dtype(fmt) or not scales.is_contiguous() or scales.numel() * group != rows * K:
        _refuse("scales must be contiguous, one for every %d channels" % group)
    _on_current_device("scales", scales, codes)
    if tensor_scale is not None:
        if tensor_scale.dtype != torch.float32 or tensor_scale.numel() < 1:
            _refuse("tensor_scale must be float32")
        _on_current_device("tensor_scale", tensor_scale, codes)
    if y is None:
        y = torch.empty((rows, K), dtype=torch.bfloat16, device=codes.device)
    yp, ldy = _rows2("y", y, rows, K, codes)
    _check(load().pq_dequantize(fmt, group, _ptr(codes), _ptr(scales), _ptr(tensor_scale), rows, K, yp, ldy, _stream()))
    return y


def pack_experts(codes: torch.Tensor, scales: torch.Tensor, experts: int) -> torch.Tensor:
    """MXFP4 weights of all experts, codes [experts * N, K/2] and scales [experts * N, K/32], as the operands of pq_qgemm_grouped:
    uint8 [experts, pq_operand_bytes(FMT_MXFP4, 32, N, K)]."""
    if codes.dim() != 2 or scales.dim() != 2 or experts <= 0 or codes.shape[0] % experts or scales.shape[0] != codes.shape[0]:
        _refuse("codes and scales must have the same rows, a multiple of %d" % experts)
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or scales.shape[1] * 16 != codes.shape[1]:
        _refuse("codes must be uint8 [rows, K/2] and scales uint8 [rows, K/32]")
    _on_current_device("codes", codes)
    _on_current_device("scales", scales, codes)
    N, K = codes.shape[0] // experts, codes.shape[1] * 2
    need = pq_operand_bytes(FMT_MXFP4, 32, N, K)
    if need == 0:
        raise PQError(-2, pq_last_error())
    out = torch.empty((experts, need), dtype=torch.uint8, device=codes.device)
    for e in range(experts):
        # rows of K/32 bytes: an expert's may begin at an address that is not the call's 16-byte alignment
        pq_pack_operand(FMT_MXFP4, 32, _aligned(codes[e * N:(e + 1) * N]), _aligned(scales[e * N:(e + 1) * N]), out[e])
    return out


def _aligned(t: torch.Tensor) -> torch.Tensor:
    return t if t.data_ptr() % 16 == 0 and t.is_contiguous() else t.contiguous().clone()


def _on_current_device(name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None):
    """The stream of a call on t: its device has to be the current one, or that of the call's other tensors."""
    if not t.is_cuda or (t.device != like.device if like is not None else t.device.index != torch.cuda.current_device()):
        _refuse("%s must lie in the memory of the current GPU, with the call's other tensors" % name)


def _array(name: str, t: torch.Tensor, dtype, shape, like: torch.Tensor) -> int:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        _refuse("%s must be contiguous %s %s" % (name, dtype, list(shape)))
    _on_current_device(name, t, like)
    return t.data_ptr()


def _rows2(name: str, t: torch.Tensor, rows: int, width: int, like: Optional[torch.Tensor]):
    """(pointer, row stride) of bf16 [rows, width] with adjacent columns; the stride of a single row does not matter."""
    if t.dtype != torch.bfloat16 or tuple(t.shape) != (rows, width) or (width > 1 and t.stride(1) != 1):
        _refuse("%s must be bfloat16 [%d, %d] with adjacent columns" % (name, rows, width))
    _on_current_device(name, t, like)
    return t.data_ptr(), t.stride(0) if rows > 1 else (width + 7) // 8 * 8


def pq_qgemm_grouped(fmt: int, group: int, a_operand: torch.Tensor, a_rows: int, w_operands: torch.Tensor, offsets: torch.Tensor,
                     y: torch.Tensor, N: int, K: int, rows: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> None:
    """y[i] (bf16 [M, N]) = row rows[i] (int32 [M], or i) of A times the weights of the expert whose rows offsets (int32 [experts + 1])
    places i in, plus bias[expert] (bf16 [experts, N]).  w_operands: uint8 [experts, pq_operand_bytes(fmt, group, N, K)]."""
    if w_operands.dim() != 2 or w_operands.dtype != torch.uint8 or not w_operands.is_contiguous():
        _refuse("w_operands must be contiguous uint8 [experts, bytes of an operand]")
    experts, M = w_operands.shape[0], y.shape[0]
    need = pq_operand_bytes(fmt, group, N, K)
    if need and w_operands.shape[1] != need:
        _refuse("w_operands must hold %d bytes an expert" % need)
    yp, ldy = _rows2("y", y, M, N, None)
    _on_current_device("w_operands", w_operands, y)
    _on_current_device("a_operand", a_operand, y)
    if a_operand.dtype != torch.uint8 or not a_operand.is_contiguous() or a_operand.numel() < pq_operand_bytes(fmt, group, a_rows, K):
        _refuse("a_operand must be contiguous uint8 and hold an operand of %d rows" % a_rows)
    op = _array("offsets", offsets, torch.int32, (experts + 1,), y)
    rp = None if rows is None else _array("rows", rows, torch.int32, (M,), y)
    bp = None if bias is None else _array("bias", bias, torch.bfloat16, (experts, N), y)
    _check(load().pq_qgemm_grouped(fmt, group, _ptr(a_operand), a_rows, _ptr(w_operands), experts, op, rp, M, N, K, bp, yp, ldy, _stream()))


def pq_qgemm_grouped_tile(fmt: int, group: int, experts: int, M: int, N: int, K: int):
    """(rows, columns) of the output tile that pq_qgemm_grouped takes for these sizes."""
    m, n = C.c_int(), C.c_int()
    _check(load().pq_qgemm_grouped_tile(fmt, group, experts, M, N, K, C.byref(m), C.byref(n)))
    return m.value, n.value


class Route(NamedTuple):
    """What pq_moe_route leaves: see pq_moe_route of the header."""
    ids: torch.Tensor           # int32 [tokens, k]
    weights: torch.Tensor       # float32 [tokens, k]
    offsets: torch.Tensor       # int32 [experts + 1]
    rows: torch.Tensor          # int32 [tokens * k]
    positions: torch.Tensor     # int32 [tokens, k]


def alloc_route(tokens: int, experts: int, k: int, device="cuda") -> Route:
    ints = lambda *shape: torch.empty(shape, dtype=torch.int32, device=device)
    return Route(ints(tokens, k), torch.empty((tokens, k), dtype=torch.float32, device=device), ints(experts + 1), ints(tokens * k),
                 ints(tokens, k))


def pq_moe_route_workspace_bytes(tokens: int, experts: int, k: int) -> int:
    return int(load().pq_moe_route_workspace_bytes(tokens, experts, k))


def pq_moe_route_workspace(tokens: int, experts: int, k: int, device="cuda") -> torch.Tensor:
    """A workspace for pq_moe_route with these arguments, or fewer tokens: for one stream, call after call."""
    need = pq_moe_route_workspace_bytes(tokens, experts, k)
    if need == 0:
        raise PQError(-2, pq_last_error())
    return torch.empty(need, dtype=torch.uint8, device=device)


def pq_moe_route(logits: torch.Tensor, k: int, renormalize: bool = True, out: Optional[Route] = None,
                 workspace: Optional[torch.Tensor] = None) -> Route:
    """The k largest of every row of logits (float32 or bf16 [tokens, experts]), their softmax weights, and the order of the rows by
    expert (allocated unless given)."""
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or (logits.shape[1] > 1 and logits.stride(1) != 1):
        _refuse("logits must be float32 or bfloat16 [tokens, experts] with adjacent experts")
    tokens, experts = logits.shape
    _on_current_device("logits", logits)
    if workspace is None:
        workspace = pq_moe_route_workspace(tokens, experts, k, logits.device)
    if not workspace.is_contiguous():
        _refuse("workspace must be contiguous")
    _on_current_device("workspace", workspace, logits)
    if out is None:
        out = alloc_route(tokens, experts, k, logits.device)
    shapes = ((tokens, k), (tokens, k), (experts + 1,), (tokens * k,), (tokens, k))
    ptrs = [_array(name, t, torch.float32 if name == "weights" else torch.int32, shape, logits)
            for name, t, shape in zip(Route._fields, out, shapes)]
    _check(load().pq_moe_route(LOGITS_BF16 if logits.dtype == torch.bfloat16 else LOGITS_F32, _ptr(logits), tokens, experts,
                               logits.stride(0) if tokens > 1 else experts, k, int(renormalize), *ptrs, _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream()))
    return out


def pq_moe_combine(y: torch.Tensor, positions: torch.Tensor, weights: torch.Tensor, addend: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[t] = addend[t] + sum_j weights[t, j] * y[positions[t, j]], bf16 [tokens, N] (allocated unless given); y bf16 [rows, N],
    positions int32 and weights float32 [tokens, k]."""
    if y.dim() != 2 or positions.dim() != 2:
        _refuse("y must be bfloat16 [rows, N], positions int32 [tokens, k]")
    (rows, N), (tokens, k) = y.shape, positions.shape
    yp, y_ld = _rows2("y", y, rows, N, None)
    pp = _array("positions", positions, torch.int32, (tokens, k), y)
    wp = _array("weights", weights, torch.float32, (tokens, k), y)
    ap, a_ld = (None, 0) if addend is None else _rows2("addend", addend, tokens, N, y)
    if out is None:
        out = torch.empty((tokens, (N + 7) // 8 * 8), dtype=torch.bfloat16, device=y.device)[:, :N]
    outp, o_ld = _rows2("out", out, tokens, N, y)
    _check(load().pq_moe_combine(yp, rows, y_ld, pp, wp, tokens, k, N, ap, a_ld, outp, o_ld, _stream()))
    return out


# ------------------------------------------------------------------------ allocation helpers
def scale_dtype(fmt: int):
    return torch.uint8 if fmt in (FMT_NVFP4, FMT_MXFP4) else torch.float32


def alloc_quantized(fmt: int, group: int, rows: int, K: int, device="cuda"):
    """(codes, scales) buffers in the stored layout."""
    codes = torch.empty((rows, K // 2), dtype=torch.uint8, device=device)
    scales = torch.empty((rows, K // group), dtype=scale_dtype(fmt), device=device)
    return codes, scales


def bf16_from_bits(bits_u16, device="cuda") -> torch.Tensor:
    """numpy uint16 bit patterns -> bf16 tensor on the device (no value conversion)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits_u16).view(np.int16))
    return t.to(device).view(torch.bfloat16)


# at import, so that names imported from here are the native ones; a library that cannot be loaded raises where it is used
if os.path.exists(_LIB_PATH):
    try:
        load()
    except PQError:
        pass

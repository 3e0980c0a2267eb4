"""Thin Python binding of the C-ABI library declared in include/snip.h.

Argument marshalling only: every function takes torch CUDA tensors (used here purely as device
memory) and forwards raw pointers and sizes to the entry point of the same name.  All work runs
in the library's CUDA kernels on torch's current stream.  There is no fallback: if the shared
library is missing or fails to load, importing this module raises.
"""
from __future__ import annotations

import bisect
import ctypes
import functools
import os
import struct

import torch

FMT_BF16, FMT_FP8_E4M3, FMT_FP4_E2M1 = 0, 1, 2
BLOCK_ROW, BLOCK_COL, BLOCK_BLK = 0, 1, 2
BLOCK_ROW32, BLOCK_COL32 = 3, 4   # 32-long tiles, power-of-two scales only
BLOCK_ROW16, BLOCK_COL16 = 5, 6   # 16-long tiles of the two-level option
OUT_BF16, OUT_FP32 = 0, 1
OP_FWD, OP_DGRAD, OP_WGRAD = 0, 1, 2
Q_TRANSPOSED, Q_STATS, Q_NO_CODES = 1, 2, 4
OK = 0
ERR_ARG, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(1, 8)

LIB_PATH = os.environ.get("SNIP_B200_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsnip_b200.so")

EXPORTS = (
    "snip_version", "snip_status_string", "snip_last_cuda_error", "snip_quantize_sizes",
    "snip_quantize", "snip_quantize_noalloc", "snip_quantize_mx_sizes", "snip_quantize_mx", "snip_quantize_dual_workspace", "snip_quantize_dual", "snip_quantize_sr", "snip_workspace_size", "snip_gemm_quantized", "snip_gemm_mx", "snip_quantize_nvfp4_sizes", "snip_quantize_nvfp4_dual", "snip_gemm_nvfp4", "snip_linear_fwd_bwd_nvfp4_workspace", "snip_linear_fwd_bwd_nvfp4", "snip_linear_fwd",
    "snip_linear_dgrad", "snip_linear_wgrad", "snip_linear_mx", "snip_linear_mx_workspace", "snip_linear_fwd_bwd_workspace", "snip_linear_fwd_bwd", "snip_layer_stats", "snip_layer_stats_workspace", "snip_adamw_sensitivity_workspace", "snip_adamw_sensitivity",
    "snip_rmsnorm_fwd", "snip_rmsnorm_bwd_workspace", "snip_rmsnorm_bwd", "snip_adamw_state_sizes", "snip_adamw_step", "snip_loss_divergence", "snip_weight_divergence", "snip_select_scheme",
    "snip_poll_status", "snip_debug_set", "snip_debug_last_gemm",
)


class SnipError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        name = _lib.snip_status_string(status).decode()
        detail = _lib.snip_last_cuda_error().decode() if status == ERR_CUDA else ""
        super().__init__(f"{fn} failed: {name} {detail}".strip())


class QTensor(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("fmt", ctypes.c_int32), ("block", ctypes.c_int32),
                ("transposed", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class QOut(ctypes.Structure):
    _fields_ = [("fmt", ctypes.c_int32), ("rounding", ctypes.c_int32), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("sf", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("seed", ctypes.c_uint64)]


DUAL_ROW_COLT, DUAL_BLK_BLKT, DUAL_ROW32_COL32T = 0, 1, 2
ROUND_NEAREST_EVEN, ROUND_STOCHASTIC = 0, 1
DEBUG_WAIT_LIMIT_NS, DEBUG_TX_SKEW_BYTES, DEBUG_GEMM_KERNEL, DEBUG_GEMM_SLICING = 0, 1, 2, 3
GEMM_KERNEL_AUTO, GEMM_KERNEL_SINGLE, GEMM_KERNEL_PAIR, GEMM_KERNEL_NARROW = 0, 1, 2, 3


class LayerTensors(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("X", "W", "Y", "dY", "dX", "dW")] + \
               [(n, ctypes.c_int64) for n in ("M", "N", "K")]


class RmsNorm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "gain", "h", "y", "rstd", "codes", "scales", "codes_t", "scales_t")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "ld_x", "ld_residual", "ld_h", "ld_y")] + \
               [("eps", ctypes.c_float), ("gain_dtype", ctypes.c_int32), ("fmt", ctypes.c_int32), ("fmt_t", ctypes.c_int32)]


class RmsNormBwd(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dy", "h", "gain", "rstd", "dresidual", "dx", "dgain")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "ld_dy", "ld_h", "ld_dresidual", "ld_dx")] + \
               [("gain_dtype", ctypes.c_int32), ("accumulate", ctypes.c_int32)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "param_bf16")] + \
               [("n", ctypes.c_int64), ("weight_decay", ctypes.c_float), ("reserved", ctypes.c_int32)]


class Adamw(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps")] + [("step", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("step_device", "lr_device", "grad_scale")] + [("seed", ctypes.c_uint64)] + \
               [(n, ctypes.c_int32) for n in ("param_dtype", "grad_dtype", "state_bits", "rounding")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2602_01410_b200.build`")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, u32, vp, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_size_t
    psz = ctypes.POINTER(sz)
    lib.snip_version.restype = i32
    lib.snip_status_string.restype = ctypes.c_char_p
    lib.snip_status_string.argtypes = [i32]
    lib.snip_last_cuda_error.restype = ctypes.c_char_p
    lib.snip_quantize_sizes.argtypes = [i64, i64, i32, i32, u32, psz, psz, psz]
    lib.snip_quantize.argtypes = [vp, i64, i64, i64, i32, i32, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.snip_quantize_noalloc.argtypes = [vp, i64, i64, i64, i32, i32, u32, vp, vp, vp, vp]
    lib.snip_quantize_mx_sizes.argtypes = [i64, i64, psz]
    lib.snip_quantize_mx.argtypes = [vp, i64, i64, i64, i32, i32, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.snip_quantize_dual_workspace.argtypes = [i64, i64, psz]
    lib.snip_quantize_dual.argtypes = [vp, i64, i64, i64, i32, i32, ctypes.POINTER(QOut), ctypes.POINTER(QOut), vp, sz, vp]
    lib.snip_quantize_sr.argtypes = [vp, i64, i64, i64, i32, u32, ctypes.c_uint64, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.snip_workspace_size.argtypes = [i32, i64, i64, i64, i32, i32, psz, psz]
    lib.snip_gemm_quantized.argtypes = [i32, ctypes.POINTER(QTensor), ctypes.POINTER(QTensor), vp, i32, i32, vp, sz, vp]
    lib.snip_gemm_mx.argtypes = [i32, ctypes.POINTER(QTensor), vp, ctypes.POINTER(QTensor), vp, vp, i32, vp, sz, vp]
    lib.snip_quantize_nvfp4_sizes.argtypes = [i64, i64, psz, psz]
    lib.snip_quantize_nvfp4_dual.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, i32, ctypes.c_uint64, vp, sz, vp]
    lib.snip_gemm_nvfp4.argtypes = [i32, ctypes.POINTER(QTensor), vp, vp, ctypes.POINTER(QTensor), vp, vp, vp, i32, vp, sz, vp]
    lib.snip_linear_fwd_bwd_nvfp4_workspace.argtypes = [i64, i64, i64, psz]
    lib.snip_linear_fwd_bwd_nvfp4.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, i32, ctypes.c_uint64, vp, vp, sz, vp]
    lin = [vp, vp, vp, i64, i64, i64, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.snip_linear_fwd.argtypes = lin
    lib.snip_linear_dgrad.argtypes = lin
    lib.snip_linear_wgrad.argtypes = [vp, vp, vp, i64, i64, i64, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.snip_linear_mx.argtypes = [i32, vp, vp, vp, i64, i64, i64, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.snip_linear_mx_workspace.argtypes = [i32, i64, i64, i64, i32, i32, psz]
    lib.snip_linear_fwd_bwd_workspace.argtypes = [i64, i64, i64, i32, i32, i32, i32, psz]
    lib.snip_linear_fwd_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, i32, i32, i32, i32, ctypes.c_uint64, vp, vp, sz, vp]
    lib.snip_layer_stats.argtypes = [ctypes.POINTER(LayerTensors), u32, vp, vp, sz, vp]
    lib.snip_layer_stats_workspace.argtypes = [i64, i64, i64, psz]
    lib.snip_adamw_sensitivity_workspace.argtypes = [i64, psz]
    lib.snip_adamw_sensitivity.argtypes = [vp, vp, vp, i32, i64, ctypes.c_float, ctypes.c_float, ctypes.c_float, vp, vp, sz, vp]
    # (a RmsNorm, RmsNormBwd or Adamw by reference, or its bytes)
    lib.snip_rmsnorm_fwd.argtypes = [vp, vp]
    lib.snip_rmsnorm_bwd_workspace.argtypes = [i64, i64, psz]
    lib.snip_rmsnorm_bwd.argtypes = [vp, vp, sz, vp]
    lib.snip_adamw_state_sizes.argtypes = [i64, i32, psz, psz]
    lib.snip_adamw_step.argtypes = [ctypes.POINTER(AdamwTensor), i64, vp, vp]
    dbl = ctypes.c_double
    lib.snip_loss_divergence.restype = dbl
    lib.snip_loss_divergence.argtypes = [dbl, dbl, i64, i64, dbl, dbl, i64, dbl]
    lib.snip_weight_divergence.restype = dbl
    lib.snip_weight_divergence.argtypes = [dbl, dbl, i64, i64, dbl, dbl, dbl, i64, dbl, i64]
    lib.snip_select_scheme.argtypes = [i32, i32, vp, vp, i64, i32, vp, vp, vp]
    lib.snip_poll_status.argtypes = [vp, ctypes.POINTER(i32)]
    lib.snip_debug_set.argtypes = [i32, ctypes.c_longlong]
    lib.snip_debug_last_gemm.argtypes = [ctypes.POINTER(i32)]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is ctypes.c_int and name not in ("snip_version",):
            fn.restype = i32
    return lib


_lib = _load()


def _check(fn, status):
    if status != OK:
        raise SnipError(fn, status)


def _p(t):
    return None if t is None else t.data_ptr()


# Handle of the current device's current stream.  The small calls of this library are bound by what the host does per call:
# building a torch.cuda.Stream object for the handle took 3.5 of a call's 10-24 us, so torch's own shortcut is used where it exists
# (it is not part of torch's public interface).
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is not None and _device is not None:
    def _stream():
        return _raw_stream(_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def snip_version() -> int:
    return int(_lib.snip_version())


def snip_status_string(status: int) -> str:
    return _lib.snip_status_string(status).decode()


def snip_quantize_sizes(rows, cols, fmt, block, flags=0):
    cb, sb, wb = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check("snip_quantize_sizes", _lib.snip_quantize_sizes(rows, cols, fmt, block, flags, ctypes.byref(cb),
                                                            ctypes.byref(sb), ctypes.byref(wb)))
    return cb.value, sb.value, wb.value


def stats_to_host(stats: torch.Tensor) -> dict:
    """Decode a snip_stats_t held in a 24-byte uint8 tensor (synchronizes)."""
    raw = stats.cpu().numpy().tobytes()
    import struct
    sx, se, am, _ = struct.unpack("<ddfI", raw[:24])
    return {"sumsq_x": sx, "sumsq_err": se, "amax": am}


def snip_quantize(x: torch.Tensor, fmt: int, block: int, flags: int = 0, *, codes=None, scales=None,
                  stats=None, row_stats=None, ws=None, want_row_stats=False):
    """x: bf16 CUDA tensor [rows, cols] (row stride = x.stride(0)).  Allocates any output not
    supplied, through torch, and returns (codes, scales, stats, row_stats) as uint8 / float32 /
    uint8[24] / float64[rows,2] tensors (None where not produced)."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    if codes is None or scales is None or ws is None:
        cb, sb, wb = snip_quantize_sizes(rows, cols, fmt, block, flags)
        dev = x.device
        if cb and codes is None:
            codes = torch.empty(cb, dtype=torch.uint8, device=dev)
        if sb and scales is None:
            scales = torch.empty(sb // 4, dtype=torch.float32, device=dev)
        if ws is None and ((flags & Q_STATS) or row_stats is not None or want_row_stats):
            ws = torch.empty(wb, dtype=torch.uint8, device=dev)
    if (flags & Q_STATS) and stats is None:
        stats = torch.empty(24, dtype=torch.uint8, device=x.device)
    if want_row_stats and row_stats is None:
        row_stats = torch.empty((rows, 2), dtype=torch.float64, device=x.device)
    _check("snip_quantize", _lib.snip_quantize(_p(x), rows, cols, x.stride(0), fmt, block, flags, _p(codes), _p(scales),
                                               _p(stats), _p(row_stats), _p(ws), 0 if ws is None else ws.numel(), _stream()))
    return codes, scales, stats, row_stats


def snip_quantize_noalloc(x: torch.Tensor, fmt: int, block: int, flags: int, codes, scales, stats):
    """Same work as snip_quantize with the statistics scratch taken from the array built into the
    library, for hosts that cannot give it any.  The caller passes every output buffer: this wrapper,
    like the entry point, allocates nothing."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    _check("snip_quantize_noalloc", _lib.snip_quantize_noalloc(_p(x), rows, cols, x.stride(0), fmt, block, flags, _p(codes),
                                                               _p(scales), _p(stats), _stream()))


def snip_quantize_mx(x: torch.Tensor, fmt: int, block: int, flags: int = 0, *, want_sf=True):
    """Power-of-two scale option.  Returns (codes, scales, sf, stats): uint8, float32, uint8 (UE8M0
    atoms, None unless want_sf) and a 32-byte stats buffer (None unless Q_STATS)."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    cb, sb, wb = snip_quantize_sizes(rows, cols, fmt, block, flags)
    dev = x.device
    codes = torch.empty(cb, dtype=torch.uint8, device=dev)
    scales = torch.empty(sb // 4, dtype=torch.float32, device=dev)
    sf = None
    if want_sf:
        n = ctypes.c_size_t()
        _check("snip_quantize_mx_sizes", _lib.snip_quantize_mx_sizes(rows, cols, ctypes.byref(n)))
        sf = torch.empty(n.value, dtype=torch.uint8, device=dev)
    stats = torch.empty(32, dtype=torch.uint8, device=dev) if (flags & Q_STATS) else None
    ws = torch.empty(wb, dtype=torch.uint8, device=dev) if (flags & Q_STATS) else None
    _check("snip_quantize_mx", _lib.snip_quantize_mx(_p(x), rows, cols, x.stride(0), fmt, block, flags, _p(codes), _p(scales), _p(sf),
                                                     _p(stats), _p(ws), 0 if ws is None else ws.numel(), _stream()))
    return codes, scales, sf, stats


def snip_quantize_dual_workspace(rows, cols):
    n = ctypes.c_size_t()
    _check("snip_quantize_dual_workspace", _lib.snip_quantize_dual_workspace(rows, cols, ctypes.byref(n)))
    return n.value


def snip_quantize_sr(x: torch.Tensor, block: int, flags: int, seed: int, *, pow2_scale=False, want_sf=False):
    """FP4 codes with stochastic rounding.  Returns (codes, scales, sf, stats) like snip_quantize_mx."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    cb, sb, wb = snip_quantize_sizes(rows, cols, FMT_FP4_E2M1, block, flags)
    dev = x.device
    codes = torch.empty(cb, dtype=torch.uint8, device=dev)
    scales = torch.empty(sb // 4, dtype=torch.float32, device=dev)
    sf = None
    if want_sf:
        n = ctypes.c_size_t()
        _check("snip_quantize_mx_sizes", _lib.snip_quantize_mx_sizes(rows, cols, ctypes.byref(n)))
        sf = torch.empty(n.value, dtype=torch.uint8, device=dev)
    stats = torch.empty(32, dtype=torch.uint8, device=dev) if (flags & Q_STATS) else None
    ws = torch.empty(wb, dtype=torch.uint8, device=dev) if (flags & Q_STATS) else None
    _check("snip_quantize_sr", _lib.snip_quantize_sr(_p(x), rows, cols, x.stride(0), block, flags, seed, int(pow2_scale), _p(codes), _p(scales),
                                                     _p(sf), _p(stats), _p(ws), 0 if ws is None else ws.numel(), _stream()))
    return codes, scales, sf, stats


def snip_quantize_dual(x: torch.Tensor, kind: int, fmt_stored: int, fmt_transposed: int, *, pow2_scale=False, want_stats=True,
                       want_sf=False, bufs=None, ws=None, sr_seeds=(None, None)):
    """One read, two outputs.  Returns two dicts (as stored, transposed) with codes / scales / sf / stats
    tensors (sf, stats None unless asked for).  bufs = (dict, dict) reuses buffers of an earlier call."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    dev = x.device
    blocks = {DUAL_ROW_COLT: (BLOCK_ROW, BLOCK_COL), DUAL_BLK_BLKT: (BLOCK_BLK, BLOCK_BLK), DUAL_ROW32_COL32T: (BLOCK_ROW32, BLOCK_COL32)}[kind]
    outs, structs = [], []
    for i, fmt in enumerate((fmt_stored, fmt_transposed)):
        if bufs is not None:
            o = bufs[i]
        else:
            cb, sb, _ = snip_quantize_sizes(rows, cols, fmt, blocks[i], Q_TRANSPOSED if i else 0)
            o = {"codes": torch.empty(cb, dtype=torch.uint8, device=dev), "scales": torch.empty(sb // 4, dtype=torch.float32, device=dev),
                 "sf": None, "stats": torch.empty(32, dtype=torch.uint8, device=dev) if want_stats else None}
            if want_sf:
                n = ctypes.c_size_t()
                _check("snip_quantize_mx_sizes", _lib.snip_quantize_mx_sizes(rows, cols, ctypes.byref(n)))
                o["sf"] = torch.empty(n.value, dtype=torch.uint8, device=dev)
        outs.append(o)
        seed = sr_seeds[i]
        structs.append(QOut(fmt, ROUND_NEAREST_EVEN if seed is None else ROUND_STOCHASTIC, _p(o["codes"]), _p(o["scales"]), _p(o["sf"]),
                            _p(o["stats"]), 0 if seed is None else seed))
    if ws is None and outs[0]["stats"] is not None:
        ws = torch.empty(snip_quantize_dual_workspace(rows, cols), dtype=torch.uint8, device=dev)
    _check("snip_quantize_dual", _lib.snip_quantize_dual(_p(x), rows, cols, x.stride(0), kind, int(pow2_scale), ctypes.byref(structs[0]),
                                                         ctypes.byref(structs[1]), _p(ws), 0 if ws is None else ws.numel(), _stream()))
    return outs[0], outs[1]


def snip_workspace_size(op, M, N, K, fmt_a, fmt_b):
    g, l = ctypes.c_size_t(), ctypes.c_size_t()
    _check("snip_workspace_size", _lib.snip_workspace_size(op, M, N, K, fmt_a, fmt_b, ctypes.byref(g), ctypes.byref(l)))
    return g.value, l.value


def make_qtensor(codes, scales, rows, cols, fmt, block, transposed=False) -> QTensor:
    return QTensor(codes.data_ptr(), 0 if scales is None else scales.data_ptr(), rows, cols, fmt, block,
                   int(transposed), 0)


def _out(shape, out_dtype, device, out):
    if out is not None:
        return out
    return torch.empty(shape, dtype=torch.bfloat16 if out_dtype == OUT_BF16 else torch.float32, device=device)


def snip_gemm_quantized(op, a: QTensor, b: QTensor, out_shape, out_dtype=OUT_BF16, accumulate=False, *, out=None,
                        ws=None, device="cuda"):
    out = _out(out_shape, out_dtype, device, out)
    if ws is None:
        M, N = out_shape
        g, _ = snip_workspace_size(op, *_mnk(op, a, b), a.fmt, b.fmt)
        ws = torch.empty(g, dtype=torch.uint8, device=out.device)
    _check("snip_gemm_quantized", _lib.snip_gemm_quantized(op, ctypes.byref(a), ctypes.byref(b), _p(out), out_dtype,
                                                           int(accumulate), _p(ws), ws.numel(), _stream()))
    return out


def snip_gemm_mx(op, a: QTensor, sf_a, b: QTensor, sf_b, out_shape, out_dtype=OUT_BF16, *, out=None, ws=None, device="cuda"):
    out = _out(out_shape, out_dtype, device, out)
    if ws is None:
        ws = torch.empty(256, dtype=torch.uint8, device=out.device)
    _check("snip_gemm_mx", _lib.snip_gemm_mx(op, ctypes.byref(a), _p(sf_a), ctypes.byref(b), _p(sf_b), _p(out), out_dtype, _p(ws),
                                             ws.numel(), _stream()))
    return out


def snip_quantize_nvfp4_sizes(rows, cols):
    cb, sb = ctypes.c_size_t(), ctypes.c_size_t()
    _check("snip_quantize_nvfp4_sizes", _lib.snip_quantize_nvfp4_sizes(rows, cols, ctypes.byref(cb), ctypes.byref(sb)))
    return cb.value, sb.value


def snip_quantize_nvfp4_dual(x: torch.Tensor, tensor_amax: torch.Tensor, *, want_stats=True, bufs=None, ws=None, sr_seed=None):
    """Two-level option, both copies from one read.  tensor_amax: float32 CUDA tensor with one element (the bound of |x|).
    Returns two dicts (as stored, transposed) with codes / sf / stats tensors."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    assert tensor_amax.is_cuda and tensor_amax.dtype == torch.float32
    rows, cols = x.shape
    dev = x.device
    if bufs is None:
        cb, sb = snip_quantize_nvfp4_sizes(rows, cols)
        bufs = tuple({"codes": torch.empty(cb, dtype=torch.uint8, device=dev), "sf": torch.empty(sb, dtype=torch.uint8, device=dev),
                      "stats": torch.empty(32, dtype=torch.uint8, device=dev) if want_stats else None} for _ in range(2))
    if ws is None and bufs[0]["stats"] is not None:
        ws = torch.empty(snip_quantize_dual_workspace(rows, cols), dtype=torch.uint8, device=dev)
    a, b = bufs
    _check("snip_quantize_nvfp4_dual", _lib.snip_quantize_nvfp4_dual(_p(x), rows, cols, x.stride(0), _p(tensor_amax), _p(a["codes"]), _p(a["sf"]),
                                                                     _p(a["stats"]), _p(b["codes"]), _p(b["sf"]), _p(b["stats"]),
                                                                     ROUND_NEAREST_EVEN if sr_seed is None else ROUND_STOCHASTIC, 0 if sr_seed is None else sr_seed,
                                                                     _p(ws), 0 if ws is None else ws.numel(), _stream()))
    return a, b


def snip_gemm_nvfp4(op, a: QTensor, sf_a, amax_a, b: QTensor, sf_b, amax_b, out_shape, out_dtype=OUT_BF16, *, out=None, ws=None, device="cuda"):
    out = _out(out_shape, out_dtype, device, out)
    if ws is None:
        ws = torch.empty(256, dtype=torch.uint8, device=out.device)
    _check("snip_gemm_nvfp4", _lib.snip_gemm_nvfp4(op, ctypes.byref(a), _p(sf_a), _p(amax_a), ctypes.byref(b), _p(sf_b), _p(amax_b), _p(out), out_dtype,
                                                   _p(ws), ws.numel(), _stream()))
    return out


def _mnk(op, a: QTensor, b: QTensor):
    if op == OP_FWD:      # a = X[M,K], b = W[N,K]
        return a.rows, b.rows, a.cols
    if op == OP_DGRAD:    # a = dY[M,N], b = W[N,K]
        return a.rows, a.cols, b.cols
    return a.rows, a.cols, b.cols  # wgrad: a = dY[M,N], b = X[M,K]


def _linear(fn_name, A, B, out_shape, M, N, K, fmt_a, fmt_b, out_dtype, op, out, ws, want_stats, extra=()):
    out = _out(out_shape, out_dtype, A.device, out)
    if ws is None:
        _, l = snip_workspace_size(op, M, N, K, fmt_a, fmt_b)
        ws = torch.empty(l, dtype=torch.uint8, device=A.device)
    sa = torch.empty(24, dtype=torch.uint8, device=A.device) if want_stats else None
    sb = torch.empty(24, dtype=torch.uint8, device=A.device) if want_stats else None
    fn = getattr(_lib, fn_name)
    _check(fn_name, fn(_p(A), _p(B), _p(out), M, N, K, fmt_a, fmt_b, out_dtype, *extra, _p(sa), _p(sb), _p(ws),
                       ws.numel(), _stream()))
    return out, sa, sb


def snip_linear_fwd(X, W, fmt_x, fmt_w, out_dtype=OUT_BF16, *, out=None, ws=None, want_stats=False):
    M, K = X.shape
    N = W.shape[0]
    return _linear("snip_linear_fwd", X, W, (M, N), M, N, K, fmt_x, fmt_w, out_dtype, OP_FWD, out, ws, want_stats)


def snip_linear_dgrad(dY, W, fmt_dy, fmt_w, out_dtype=OUT_BF16, *, out=None, ws=None, want_stats=False):
    M, N = dY.shape
    K = W.shape[1]
    return _linear("snip_linear_dgrad", dY, W, (M, K), M, N, K, fmt_dy, fmt_w, out_dtype, OP_DGRAD, out, ws, want_stats)


def snip_linear_wgrad(dY, X, fmt_dy, fmt_x, out_dtype=OUT_BF16, accumulate=False, *, out=None, ws=None,
                      want_stats=False):
    M, N = dY.shape
    K = X.shape[1]
    return _linear("snip_linear_wgrad", dY, X, (N, K), M, N, K, fmt_dy, fmt_x, out_dtype, OP_WGRAD, out, ws,
                   want_stats, extra=(int(accumulate),))


def snip_linear_mx_workspace(op, M, N, K, fmt_a, fmt_b):
    w = ctypes.c_size_t()
    _check("snip_linear_mx_workspace", _lib.snip_linear_mx_workspace(op, M, N, K, fmt_a, fmt_b, ctypes.byref(w)))
    return w.value


def snip_linear_mx(op, A, B, fmt_a, fmt_b, out_dtype=OUT_BF16, *, out=None, ws=None, want_stats=False):
    """Power-of-two scale option.  op FWD: (X, W) -> Y; DGRAD: (dY, W) -> dX; WGRAD: (dY, X) -> dW."""
    if op == OP_FWD:
        (M, K), N = A.shape, B.shape[0]
        shape = (M, N)
    elif op == OP_DGRAD:
        (M, N), K = A.shape, B.shape[1]
        shape = (M, K)
    else:
        (M, N), K = A.shape, B.shape[1]
        shape = (N, K)
    out = _out(shape, out_dtype, A.device, out)
    if ws is None:
        ws = torch.empty(snip_linear_mx_workspace(op, M, N, K, fmt_a, fmt_b), dtype=torch.uint8, device=A.device)
    sa = torch.empty(32, dtype=torch.uint8, device=A.device) if want_stats else None
    sb = torch.empty(32, dtype=torch.uint8, device=A.device) if want_stats else None
    _check("snip_linear_mx", _lib.snip_linear_mx(op, _p(A), _p(B), _p(out), M, N, K, fmt_a, fmt_b, out_dtype, _p(sa), _p(sb), _p(ws),
                                                 ws.numel(), _stream()))
    return out, sa, sb


def snip_linear_fwd_bwd_workspace(M, N, K, fmt_fwd, fmt_dgrad, fmt_wgrad, pow2_scale=False):
    n = ctypes.c_size_t()
    _check("snip_linear_fwd_bwd_workspace", _lib.snip_linear_fwd_bwd_workspace(M, N, K, fmt_fwd, fmt_dgrad, fmt_wgrad, int(pow2_scale),
                                                                               ctypes.byref(n)))
    return n.value


def snip_linear_fwd_bwd(x, w, dy, fmt_fwd, fmt_dgrad, fmt_wgrad, out_dtype=OUT_BF16, *, pow2_scale=False, dy_sr_seed=None, y=None,
                        dx=None, dw=None, stats=None, ws=None):
    """Forward and both gradients of one linear layer, each tensor read once.  Returns (y, dx, dw, stats)
    with stats a uint8 tensor holding six 24-byte snip_stats_t."""
    M, K = x.shape
    N = w.shape[0]
    dev = x.device
    y, dx, dw = _out((M, N), out_dtype, dev, y), _out((M, K), out_dtype, dev, dx), _out((N, K), out_dtype, dev, dw)
    if stats is None:
        stats = torch.zeros(6 * 24, dtype=torch.uint8, device=dev)
    if ws is None:
        ws = torch.empty(snip_linear_fwd_bwd_workspace(M, N, K, fmt_fwd, fmt_dgrad, fmt_wgrad, pow2_scale), dtype=torch.uint8, device=dev)
    _check("snip_linear_fwd_bwd", _lib.snip_linear_fwd_bwd(_p(x), _p(w), _p(dy), _p(y), _p(dx), _p(dw), M, N, K, fmt_fwd, fmt_dgrad, fmt_wgrad,
                                                           out_dtype, int(pow2_scale), ROUND_NEAREST_EVEN if dy_sr_seed is None else ROUND_STOCHASTIC,
                                                           0 if dy_sr_seed is None else dy_sr_seed, _p(stats), _p(ws), ws.numel(), _stream()))
    return y, dx, dw, stats


def snip_linear_fwd_bwd_nvfp4(x, w, dy, bounds3, out_dtype=OUT_BF16, *, dy_sr_seed=None, stats=None, ws=None):
    """Forward and both gradients under the two-level option.  bounds3: float32 CUDA tensor [3] (bounds of |X|, |W|, |dY|).
    Returns (y, dx, dw, stats) with stats a uint8 tensor holding six 24-byte snip_stats_t."""
    M, K = x.shape
    N = w.shape[0]
    dev = x.device
    y, dx, dw = _out((M, N), out_dtype, dev, None), _out((M, K), out_dtype, dev, None), _out((N, K), out_dtype, dev, None)
    if stats is None:
        stats = torch.zeros(6 * 24, dtype=torch.uint8, device=dev)
    if ws is None:
        n = ctypes.c_size_t()
        _check("snip_linear_fwd_bwd_nvfp4_workspace", _lib.snip_linear_fwd_bwd_nvfp4_workspace(M, N, K, ctypes.byref(n)))
        ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
    _check("snip_linear_fwd_bwd_nvfp4", _lib.snip_linear_fwd_bwd_nvfp4(_p(x), _p(w), _p(dy), _p(y), _p(dx), _p(dw), M, N, K, out_dtype, _p(bounds3),
                                                                       ROUND_NEAREST_EVEN if dy_sr_seed is None else ROUND_STOCHASTIC,
                                                                       0 if dy_sr_seed is None else dy_sr_seed, _p(stats), _p(ws), ws.numel(), _stream()))
    return y, dx, dw, stats


def snip_layer_stats_workspace(M, N, K):
    w = ctypes.c_size_t()
    _check("snip_layer_stats_workspace", _lib.snip_layer_stats_workspace(M, N, K, ctypes.byref(w)))
    return w.value


def snip_layer_stats(X=None, W=None, Y=None, dY=None, dX=None, dW=None, *, M, N, K, fmt_mask=0b110, out=None, ws=None):
    """Returns a float64 CUDA tensor of 24 values: sumsq[6] then sumsq_err[3][2][3]."""
    dev = next(t for t in (X, W, Y, dY, dX, dW) if t is not None).device
    lt = LayerTensors(*[0 if t is None else t.data_ptr() for t in (X, W, Y, dY, dX, dW)], M, N, K)
    if out is None:
        out = torch.zeros(24, dtype=torch.float64, device=dev)
    if ws is None:
        ws = torch.empty(snip_layer_stats_workspace(M, N, K), dtype=torch.uint8, device=dev)
    _check("snip_layer_stats", _lib.snip_layer_stats(ctypes.byref(lt), fmt_mask, _p(out), _p(ws), ws.numel(), _stream()))
    return out


def snip_adamw_sensitivity(m: torch.Tensor, v: torch.Tensor, g: torch.Tensor, beta1: float, beta2: float, eps: float, *, out=None, ws=None):
    """Sum of T^2 (AdamW sensitivity term) over a parameter tensor; returns a 1-element float64 CUDA tensor."""
    assert m.dtype == torch.float32 and v.dtype == torch.float32 and g.dtype in (torch.bfloat16, torch.float32)
    assert m.is_contiguous() and v.is_contiguous() and g.is_contiguous() and m.numel() == v.numel() == g.numel()
    n = m.numel()
    if out is None:
        out = torch.zeros(1, dtype=torch.float64, device=m.device)
    if ws is None:
        w = ctypes.c_size_t()
        _check("snip_adamw_sensitivity_workspace", _lib.snip_adamw_sensitivity_workspace(n, ctypes.byref(w)))
        ws = torch.empty(w.value, dtype=torch.uint8, device=m.device)
    _check("snip_adamw_sensitivity", _lib.snip_adamw_sensitivity(_p(m), _p(v), _p(g), OUT_BF16 if g.dtype == torch.bfloat16 else OUT_FP32, n, beta1, beta2,
                                                                 eps, _p(out), _p(ws), ws.numel(), _stream()))
    return out


def _require(ok, what):
    if not ok:
        raise ValueError(what)


if _device is None:
    def _device():
        return torch.cuda.current_device()


def _call_on(dev, fn, call, args):
    """The library's `call(*args, stream)` on the current stream of device `dev`, with `dev` current meanwhile."""
    if dev == _device():
        _check(fn, call(*args, _stream()))
    else:
        with torch.cuda.device(dev):
            _check(fn, call(*args, _stream()))


# The calls below are short on the device, and their checks are what the host does most of: each asks a tensor for no more than it has to.
_BF16, _F32, _U8 = torch.bfloat16, torch.float32, torch.uint8


def _rows_apart(t, shape, name):
    """Row stride of a bf16 matrix of `shape`."""
    if t.dtype is not _BF16:
        raise ValueError(f"{name}: a bf16 tensor is wanted")
    ld, step = t.stride()
    if step != 1 and shape[1] != 1:
        raise ValueError(f"{name}: the elements of a row have to be adjacent")
    return ld if shape[0] > 1 else shape[1]   # a single row's stride says nothing


def _matrix(t, shape, dev, name):
    """Checks a bf16 matrix of `shape` on device `dev`; its row stride."""
    if t.shape != shape or t.get_device() != dev:
        raise ValueError(f"{name}: a bf16 tensor of shape {tuple(shape)} on CUDA device {dev} is wanted")
    return _rows_apart(t, shape, name)


def _vector(t, n, dtype, dev, name):
    if t.dtype is not dtype or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous elements of {dtype} on CUDA device {dev} are wanted")
    return t.data_ptr()


def _gain(t, cols, dev):
    dtype = t.dtype
    if dtype is not _BF16 and dtype is not _F32 or t.dim() != 1:
        raise ValueError("gain: a bf16 or float32 vector is wanted")
    return _vector(t, cols, dtype, dev, "gain"), OUT_BF16 if dtype is _BF16 else OUT_FP32


def _cuda_device(t, name):
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name}: a tensor on a CUDA device is wanted")
    return dev


# a call's structure, as its bytes (filling a ctypes structure field by field takes three times as long)
_RMSNORM_ARGS = struct.Struct("=10Q6qf3i").pack        # RmsNorm
_RMSNORM_BWD_ARGS = struct.Struct("=7Q6q2i").pack      # RmsNormBwd
_ADAMW_ARGS = struct.Struct("=4dq4Q4i").pack            # Adamw
_RMSNORM_OUTPUTS = frozenset(("h", "y", "rstd", "codes", "scales", "codes_t", "scales_t"))
_QUANT = (FMT_FP8_E4M3, FMT_FP4_E2M1)


def _code_bytes(rows, cols, fmt):
    """As snip_quantize_sizes, for any number of rows and a multiple of 8 columns."""
    return rows * cols if fmt == FMT_FP8_E4M3 else rows * cols // 2 + (64 if rows % 128 or cols % 128 else 0)


def _copy_of(codes, scales, fmt, lines, along, dev, name):
    """Checks one quantized copy; the two addresses."""
    if fmt not in _QUANT:
        raise ValueError(f"{name}: codes are FMT_FP8_E4M3 or FMT_FP4_E2M1")
    if codes.dtype is not _U8 or codes.numel() < _code_bytes(lines, along, fmt) or codes.get_device() != dev or not codes.is_contiguous():
        raise ValueError(f"{name}: {_code_bytes(lines, along, fmt)} contiguous bytes on CUDA device {dev} are wanted")
    return codes.data_ptr(), _vector(scales, -(-along // 128) * lines, _F32, dev, "scales of " + name)


def snip_rmsnorm_fwd(x: torch.Tensor, gain: torch.Tensor, eps: float, *, residual=None, fmt=None, fmt_t=None, want_y=None, out=None):
    """RMS norm of x + residual and its quantized copies.  Returns a dict: h (bf16, the sum; x itself without a residual), rstd (float32 [rows]),
    y (bf16), codes / scales (row tiles, uint8 / float32), codes_t / scales_t (column tiles, stored transposed); None where not produced.
    x, residual: bf16 [rows, cols], any row stride that is a multiple of 8.
    Without `out`, buffers are allocated: codes if fmt is FMT_FP8_E4M3 or FMT_FP4_E2M1, codes_t if fmt_t is, y if want_y (default: no codes asked
    for).  With `out`, a dict of such buffers, exactly those that it names are written (out["h"] may be residual or x: the sum in place)."""
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("x: a matrix is wanted")
    rows, cols = shape
    dev = _cuda_device(x, "x")
    if out is None:
        def empty(n, dtype):
            return torch.empty(n, dtype=dtype, device=x.device)

        _require(fmt in (None, FMT_BF16) + _QUANT and fmt_t in (None, FMT_BF16) + _QUANT, "fmt, fmt_t: FMT_FP8_E4M3, FMT_FP4_E2M1 or None")
        out = {"h": None if residual is None else empty((rows, cols), _BF16), "rstd": empty(rows, _F32)}
        if want_y or (want_y is None and fmt not in _QUANT and fmt_t not in _QUANT):
            out["y"] = empty((rows, cols), _BF16)
        if fmt in _QUANT:
            out["codes"], out["scales"] = empty(_code_bytes(rows, cols, fmt), _U8), empty(-(-cols // 128) * rows, _F32)
        if fmt_t in _QUANT:
            out["codes_t"], out["scales_t"] = empty(_code_bytes(rows, cols, fmt_t), _U8), empty(-(-rows // 128) * cols, _F32)
    else:
        _require(want_y is None, "want_y: `out` says what is produced")
        if not _RMSNORM_OUTPUTS.issuperset(out):
            raise ValueError(f"out: unknown outputs {sorted(set(out) - _RMSNORM_OUTPUTS)}")
    get = out.get
    h, y, rstd, codes, scales, codes_t, scales_t = get("h"), get("y"), get("rstd"), get("codes"), get("scales"), get("codes_t"), get("scales_t")
    if residual is None and h is x:
        h = None   # what an earlier call returned for h
    ld_x, (p_gain, gain_dtype) = _rows_apart(x, shape, "x"), _gain(gain, cols, dev)
    p_res = ld_res = p_h = ld_h = p_y = ld_y = p_rstd = p_codes = p_scales = p_codes_t = p_scales_t = 0
    if residual is not None:
        if h is None:
            raise ValueError("out: the sum with a residual needs h")
        ld_res, p_res = _matrix(residual, shape, dev, "residual"), residual.data_ptr()
        ld_h, p_h = _matrix(h, shape, dev, "h"), h.data_ptr()
    elif h is not None:
        raise ValueError("out: h goes with a residual")
    if y is not None:
        ld_y, p_y = _matrix(y, shape, dev, "y"), y.data_ptr()
    if rstd is not None:
        p_rstd = _vector(rstd, rows, _F32, dev, "rstd")
    if (codes is None) != (scales is None) or (codes_t is None) != (scales_t is None):
        raise ValueError("out: codes and scales go together")
    if codes is not None:
        p_codes, p_scales = _copy_of(codes, scales, fmt, rows, cols, dev, "codes")
    if codes_t is not None:
        p_codes_t, p_scales_t = _copy_of(codes_t, scales_t, fmt_t, cols, rows, dev, "codes_t")
    a = _RMSNORM_ARGS(x.data_ptr(), p_res, p_gain, p_h, p_y, p_rstd, p_codes, p_scales, p_codes_t, p_scales_t, rows, cols, ld_x, ld_res, ld_h, ld_y, eps,
                      gain_dtype, fmt or 0, fmt_t or 0)
    _call_on(dev, "snip_rmsnorm_fwd", _lib.snip_rmsnorm_fwd, (a,))
    return {"h": x if h is None else h, "y": y, "rstd": rstd, "codes": codes, "scales": scales, "codes_t": codes_t, "scales_t": scales_t}


@functools.lru_cache(maxsize=256)   # of the sizes alone
def snip_rmsnorm_bwd_workspace(rows, cols):
    n = ctypes.c_size_t()
    _check("snip_rmsnorm_bwd_workspace", _lib.snip_rmsnorm_bwd_workspace(rows, cols, ctypes.byref(n)))
    return n.value


def snip_rmsnorm_bwd(dy: torch.Tensor, h: torch.Tensor, gain: torch.Tensor, rstd: torch.Tensor, *, dresidual=None, dx=None, dgain=None, want_dgain=True,
                     accumulate=False, ws=None):
    """Gradients of the norm: (dx, dgain).  dy, h, dresidual: bf16 [rows, cols]; h, rstd: of the forward call.  dx (bf16) may be dy or dresidual;
    dgain: float32 [cols] (None with want_dgain=False), added to with accumulate."""
    shape = dy.shape
    if len(shape) != 2:
        raise ValueError("dy: a matrix is wanted")
    rows, cols = shape
    dev = _cuda_device(dy, "dy")
    if dx is None:
        dx = torch.empty((rows, cols), dtype=_BF16, device=dy.device)
    if dgain is None and want_dgain:
        _require(not accumulate, "accumulate: needs the dgain to add to")
        dgain = torch.empty(cols, dtype=_F32, device=dy.device)
    ld_dy, ld_h, ld_dx = _rows_apart(dy, shape, "dy"), _matrix(h, shape, dev, "h"), _matrix(dx, shape, dev, "dx")
    p_res = ld_res = p_dgain = at = size = 0
    if dresidual is not None:
        ld_res, p_res = _matrix(dresidual, shape, dev, "dresidual"), dresidual.data_ptr()
    p_gain, gain_dtype = _gain(gain, cols, dev)
    p_rstd = _vector(rstd, rows, _F32, dev, "rstd")
    if dgain is not None:
        p_dgain = _vector(dgain, cols, _F32, dev, "dgain")
        if ws is None:
            size = snip_rmsnorm_bwd_workspace(rows, cols)
            ws = torch.empty(size, dtype=_U8, device=dy.device)
            at = ws.data_ptr()
        else:
            size = ws.numel() * ws.element_size()
            at = _vector(ws, ws.numel(), ws.dtype, dev, "ws")
    a = _RMSNORM_BWD_ARGS(dy.data_ptr(), h.data_ptr(), p_gain, p_rstd, p_res, dx.data_ptr(), p_dgain, rows, cols, ld_dy, ld_h, ld_res, ld_dx, gain_dtype, 1 if accumulate else 0)
    _call_on(dev, "snip_rmsnorm_bwd", _lib.snip_rmsnorm_bwd, (a, at, size))
    return dx, dgain


def snip_adamw_state_sizes(n, state_bits):
    """Bytes of one state tensor (m or v) of n elements, and of its scales."""
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check("snip_adamw_state_sizes", _lib.snip_adamw_state_sizes(n, state_bits, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


class AdamwTensors:
    """The tensors of one AdamW step, checked and laid out for the library (make_adamw_tensors).  Holds the tensors."""

    def __init__(self, table, count, device, param_dtype, grad_dtype, state_bits, keep):
        self.table, self.count, self.device, self.param_dtype, self.grad_dtype, self.state_bits, self._keep = table, count, device, param_dtype, grad_dtype, state_bits, keep


def make_adamw_tensors(params, grads, m, v, *, m_scales=None, v_scales=None, copies=None, weight_decay=0.0) -> AdamwTensors:
    """Lists of contiguous CUDA tensors of one device, one entry per parameter.  params: float32 or bf16; grads: float32 or bf16; m, v: float32, or
    uint8 (8-bit states) with m_scales, v_scales: float32, one value per 128 elements; copies: None, or a list of bf16 tensors (or None) that receive
    the new float32 params; weight_decay: one number, or one per tensor.  Made once, used for as long as the tensors stay where they are (it holds them)."""
    count = len(params)
    lists = {"params": params, "grads": grads, "m": m, "v": v, "m_scales": m_scales, "v_scales": v_scales, "copies": copies}
    decay = [weight_decay] * count if isinstance(weight_decay, (int, float)) else list(weight_decay)
    for name, ts in lists.items():
        _require(ts is None or len(ts) == count, f"{name}: one entry per parameter is wanted")
    _require(len(decay) == count, "weight_decay: a number, or one per parameter")
    lists = {name: [None] * count if ts is None else list(ts) for name, ts in lists.items()}
    device = next((_cuda_device(t, "params") for t in lists["params"]), None)
    first = {name: next((t.dtype for t in ts if t is not None), None) for name, ts in lists.items()}
    _require(first["params"] in (None, torch.float32, torch.bfloat16) and first["grads"] in (None, torch.float32, torch.bfloat16), "params, grads: float32 or bf16")
    bits = 8 if first["m"] == torch.uint8 else 32
    state = torch.uint8 if bits == 8 else torch.float32
    written = []
    table = (AdamwTensor * max(count, 1))()
    for i in range(count):
        n = lists["params"][i].numel()
        wanted = {"params": (n, first["params"]), "grads": (n, first["grads"]), "m": (n, state), "v": (n, state)}
        if bits == 8:
            wanted |= {"m_scales": (-(-n // 128), torch.float32), "v_scales": (-(-n // 128), torch.float32)}
        if lists["copies"][i] is not None:
            _require(first["params"] == torch.float32, "copies: of float32 params")
            wanted["copies"] = (n, torch.bfloat16)
        row = {}
        for name, ts in lists.items():
            t = ts[i]
            _require((t is not None) == (name in wanted), f"{name}[{i}]: {'missing' if t is None else 'not wanted'}")
            if t is not None:
                row[name] = _vector(t, *wanted[name], device, f"{name}[{i}]")
                if t.numel() and name != "grads":
                    written.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
        table[i] = AdamwTensor(row["params"], row["grads"], row["m"], row["v"], row.get("m_scales"), row.get("v_scales"), row.get("copies"), n, decay[i], 0)
    read = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in lists["grads"] if t.numel()]
    written.sort()
    _require(all(a[1] <= b[0] for a, b in zip(written, written[1:])), "tensors overlap: each may be given once")
    starts = [w[0] for w in written]
    for lo, hi in read:
        k = bisect.bisect_left(starts, hi)
        _require(k == 0 or written[k - 1][1] <= lo, "a gradient overlaps what the step writes")
    return AdamwTensors(table, count, device, OUT_BF16 if first["params"] == torch.bfloat16 else OUT_FP32,
                        OUT_BF16 if first["grads"] == torch.bfloat16 else OUT_FP32, bits, lists)


def snip_adamw_step(tensors: AdamwTensors, lr, beta1: float, beta2: float, eps: float, step, *, rounding=ROUND_NEAREST_EVEN, seed=0, grad_scale=None):
    """One AdamW step over `tensors` in place.  lr: a number, or a float32 CUDA tensor with one element; step: a whole number from 1, or an int64 CUDA
    tensor with one element (both are then read when the step runs, also by each replay of a captured graph).  grad_scale: None, or a float32 CUDA tensor with one
    element by which every gradient is multiplied."""
    lr_dev, step_dev = lr if isinstance(lr, torch.Tensor) else None, step if isinstance(step, torch.Tensor) else None
    if tensors.count == 0:
        return
    for t, dtype, name in ((lr_dev, _F32, "lr"), (step_dev, torch.int64, "step"), (grad_scale, _F32, "grad_scale")):
        if t is not None:
            _vector(t, 1, dtype, tensors.device, name)
    _require(0 <= seed < 1 << 64, "seed: 64 bits")
    a = _ADAMW_ARGS(0.0 if lr_dev is not None else lr, beta1, beta2, eps, 0 if step_dev is not None else step, _p(step_dev) or 0, _p(lr_dev) or 0,
                    _p(grad_scale) or 0, seed, tensors.param_dtype, tensors.grad_dtype, tensors.state_bits, rounding)
    _call_on(tensors.device, "snip_adamw_step", _lib.snip_adamw_step, (tensors.table, tensors.count, a))


def snip_loss_divergence(grad_x_norm, err_x_norm, M, K, grad_w_norm, err_w_norm, N, loss) -> float:
    return float(_lib.snip_loss_divergence(grad_x_norm, err_x_norm, M, K, grad_w_norm, err_w_norm, N, loss))


def snip_weight_divergence(sens_norm, grad_err_norm, N, K, lr, beta1, beta2, step, weight_norm, num_layers) -> float:
    return float(_lib.snip_weight_divergence(sens_norm, grad_err_norm, N, K, lr, beta1, beta2, step, weight_norm, num_layers))


def snip_select_scheme(q, w, target: int, num_groups: int = 1):
    """q: m x n floats, w: m x n ints.  Returns (choice list, total loss, total work)."""
    import numpy as np
    qa = np.ascontiguousarray(np.asarray(q, dtype=np.float64))
    wa = np.ascontiguousarray(np.asarray(w, dtype=np.int64))
    m, n = qa.shape
    assert wa.shape == (m, n)
    choice = np.zeros(m, dtype=np.int32)
    qt, wt = ctypes.c_double(), ctypes.c_int64()
    _check("snip_select_scheme", _lib.snip_select_scheme(m, n, qa.ctypes.data_as(ctypes.c_void_p), wa.ctypes.data_as(ctypes.c_void_p), int(target),
                                                         num_groups, choice.ctypes.data_as(ctypes.c_void_p), ctypes.byref(qt), ctypes.byref(wt)))
    return [int(c) for c in choice], qt.value, wt.value


def snip_debug_set(key: int, value: int) -> None:
    """Testing hooks of the library (process-wide, off by default): see include/snip.h."""
    _check("snip_debug_set", _lib.snip_debug_set(key, value))


def snip_debug_last_gemm() -> tuple:
    """(columns of a tile, CTAs per tile, slices, CTAs of a cluster) of this thread's last quantized GEMM under the paper's rule."""
    plan = (ctypes.c_int * 4)()
    _check("snip_debug_last_gemm", _lib.snip_debug_last_gemm(plan))
    return tuple(plan)


def snip_poll_status(ws: torch.Tensor) -> int:
    st = ctypes.c_int(0)
    _check("snip_poll_status", _lib.snip_poll_status(_p(ws), ctypes.byref(st)))
    return st.value

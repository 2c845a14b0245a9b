"""B200-native SDQ decomposed linear layer: thin Python binding over the C-ABI in include/sdq.h.

Argument marshalling only -- every step of the path (weight decomposition + packing, activation
quantization, the fused sparse GEMM) runs in the CUDA kernels of libsdq_b200.so.  PyTorch supplies
device memory and streams.  The calls made for every batch of activations are marshalled by a small native
module (csrc/sdq_python.cpp), everything else by ctypes.  There is no CPU fallback: importing works without a GPU (so the build can
be checked), but every compute call needs the CUDA library and a CUDA tensor.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from dataclasses import dataclass, field

import torch

from .build import BINDING, LIB, build

GRAN_PAIR, GRAN_ELEM, GRAN_DENSE = 0, 1, 2
GRAN_3OF4 = 9      # S-Vectors of 4: 3:4 = 1:4 outliers (out_n = 2 per 8, or 0) + 2:4 inliers, stored and run like the dense pattern


def gran_keep(n: int) -> int:
    """SDQ_GRAN_KEEP(n): Stage 1 keeps the n most significant of every 8 (out_n outliers + n - out_n inliers at any
    positions); stored and executed like the dense pattern.  gran_keep(8) == GRAN_DENSE."""
    assert 2 <= n <= 8
    return 2 + (8 - n)
SCALE_OCP_FLOOR, SCALE_CEIL_NOSAT, SCALE_UE4M3 = 0, 1, 2
ORDER_LARGE, ORDER_SMALL = 0, 1
OUT_E4M3, OUT_INT8 = 0, 1
ROUTE_SOFTMAX, ROUTE_SIGMOID = 0, 1
FMT_MXFP4, FMT_NVFP4 = 0, 1                 # plain microscaled formats: E8M0 scale per 32, E4M3 scale per 16 under a row factor

STATUS = ["ok", "invalid_arg", "shape", "alignment", "unsupported", "buffer_too_small", "nonfinite", "cuda", "timeout"]


class SdqError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (where, STATUS[code] if 0 <= code < len(STATUS) else "?", code))


class Config(ctypes.Structure):
    """`pattern, formats` of the decomposition (sdq_config_t)."""
    _fields_ = [("out_n", ctypes.c_int32), ("in_gran", ctypes.c_int32), ("in_block", ctypes.c_int32),
                ("scale_rule", ctypes.c_int32), ("out_order", ctypes.c_int32), ("out_fmt", ctypes.c_int32)]

    def __init__(self, out_n=1, in_gran=GRAN_PAIR, in_block=64, scale_rule=SCALE_OCP_FLOOR, out_order=0, out_fmt=0):
        super().__init__(out_n, in_gran, in_block, scale_rule, out_order, out_fmt)


class _Packed(ctypes.Structure):
    _fields_ = [("dev", ctypes.c_void_p), ("bytes", ctypes.c_size_t), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("cfg", Config), ("off", ctypes.c_size_t * 8)]


class _Act(ctypes.Structure):
    _fields_ = [("dev", ctypes.c_void_p), ("bytes", ctypes.c_size_t), ("M", ctypes.c_int64), ("K", ctypes.c_int64),
                ("cfg", Config), ("off", ctypes.c_size_t * 6)]


class _Canon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("in_code", "in_meta", "in_scale", "out_code", "out_idx", "out_sexp", "in_texp")]


class _ActCanon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("xq4_code", "xq4_scale", "xq8_code", "xq8_sexp")]


class _Mx4(ctypes.Structure):
    _fields_ = [("dev", ctypes.c_void_p), ("bytes", ctypes.c_size_t), ("E", ctypes.c_int64), ("R", ctypes.c_int64), ("K", ctypes.c_int64),
                ("fmt", ctypes.c_int32), ("reserved", ctypes.c_int32), ("factors", ctypes.c_size_t)]


EXPORTS = ["sdq_packed_size", "sdq_decompose", "sdq_decompose_metric", "sdq_channel_norm", "sdq_packed_export", "sdq_packed_attach", "sdq_packed_compact_size", "sdq_packed_compact", "sdq_act_size", "sdq_quantize_act", "sdq_act_export",
           "sdq_linear", "sdq_linear_f32", "sdq_workspace_size", "sdq_workspace_init", "sdq_linear_ws", "sdq_linear_f32_ws", "sdq_linear_noalloc",
           "sdq_linear_group", "sdq_linear_group_f32", "sdq_linear_group_x", "sdq_linear_group_x_f32", "sdq_linear_group_x_ws", "sdq_linear_group_x_f32_ws", "sdq_mx4_size", "sdq_mx4_quantize", "sdq_mx4_import", "sdq_mx4_export", "sdq_mx4_dequantize", "sdq_mx4_linear",
           "sdq_mx4_experts_size", "sdq_mx4_experts_quantize", "sdq_mx4_experts_import",
           "sdq_moe_route", "sdq_mx4_moe_workspace_size", "sdq_mx4_moe", "sdq_diag_l2_copy", "sdq_diag_wait_timeout", "sdq_diag_decompose_timeout", "sdq_diag_linear_plan", "sdq_diag_linear_rings", "sdq_diag_group_plan", "sdq_diag_linear_memory", "sdq_diag_group_memory", "sdq_diag_mx4_quantize_rows", "sdq_device_status", "sdq_status_string"]

_lib = None


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise RuntimeError("libsdq_b200.so is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                               "(the SDQ path has no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB)
        vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
        L.sdq_packed_size.argtypes = [i64, i64, ctypes.POINTER(Config), ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.sdq_decompose.argtypes = [vp, i64, i64, i64, ctypes.POINTER(Config), vp, sz, ctypes.POINTER(_Packed), vp]
        L.sdq_decompose_metric.argtypes = [vp, i64, i64, i64, ctypes.POINTER(Config), vp, vp, sz, ctypes.POINTER(_Packed), vp]
        L.sdq_channel_norm.argtypes = [vp, i64, i64, i64, vp, vp]
        L.sdq_diag_l2_copy.argtypes = [vp, sz, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(sz), vp]
        L.sdq_packed_export.argtypes = [ctypes.POINTER(_Packed), ctypes.POINTER(_Canon), vp]
        L.sdq_packed_attach.argtypes = [vp, sz, ctypes.POINTER(_Packed), vp]
        L.sdq_diag_wait_timeout.argtypes = [ctypes.c_int, vp]
        L.sdq_diag_decompose_timeout.argtypes = L.sdq_decompose.argtypes
        L.sdq_act_size.argtypes = [i64, i64, ctypes.POINTER(Config), ctypes.POINTER(sz)]
        L.sdq_quantize_act.argtypes = [vp, i64, i64, i64, ctypes.POINTER(Config), vp, sz, ctypes.POINTER(_Act), vp]
        L.sdq_act_export.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_ActCanon), vp]
        L.sdq_linear.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_Packed), vp, i64, vp]
        L.sdq_linear_f32.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_Packed), vp, i64, vp]
        L.sdq_workspace_size.argtypes = [i64, i64, i64, ctypes.POINTER(Config), ctypes.POINTER(sz)]
        L.sdq_workspace_init.argtypes = [vp, sz, vp]
        L.sdq_linear_ws.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_Packed), vp, i64, vp, sz, vp]
        L.sdq_linear_f32_ws.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_Packed), vp, i64, vp, sz, vp]
        L.sdq_linear_noalloc.argtypes = [ctypes.POINTER(_Act), ctypes.POINTER(_Packed), vp, i64, vp]
        L.sdq_linear_group.argtypes = [ctypes.c_int, vp, vp, vp, vp, vp]
        L.sdq_linear_group_f32.argtypes = [ctypes.c_int, vp, vp, vp, vp, vp]
        i32, m4 = ctypes.c_int32, ctypes.POINTER(_Mx4)
        L.sdq_mx4_size.argtypes = [i64, i64, i32, ctypes.POINTER(sz)]
        L.sdq_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, sz, m4, vp]
        L.sdq_mx4_import.argtypes = [vp, vp, vp, i64, i64, i32, vp, sz, m4, vp]
        L.sdq_mx4_export.argtypes = [m4, vp, vp, vp, vp]
        L.sdq_mx4_dequantize.argtypes = [m4, vp, i32, i64, vp]
        L.sdq_mx4_linear.argtypes = [m4, m4, vp, i32, vp, i64, vp]
        L.sdq_mx4_experts_size.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
        L.sdq_mx4_experts_quantize.argtypes = [vp, i32, i64, i64, i64, i32, vp, sz, m4, vp]
        L.sdq_mx4_experts_import.argtypes = [vp, vp, i64, i64, i64, vp, sz, m4, vp]
        L.sdq_moe_route.argtypes = [vp, i32, i64, i64, i64, vp, i64, i64, vp, i32, i32, i32, ctypes.c_float, vp, vp, vp]
        L.sdq_mx4_moe_workspace_size.argtypes = [i64, i32, i64, i64, ctypes.POINTER(sz)]
        L.sdq_mx4_moe.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, m4, m4, m4, vp, i64, vp, sz, vp]
        L.sdq_device_status.argtypes = [vp]
        L.sdq_status_string.argtypes = [ctypes.c_int]
        L.sdq_status_string.restype = ctypes.c_char_p
        for n in EXPORTS[:-1]:
            getattr(L, n).restype = ctypes.c_int
        _lib = L
    return _lib


_fast = None


class _NoNative:
    """In the place of the native module where it is missing or does not load: leaves every call to the ctypes form."""

    def __getattr__(self, name):
        return lambda *args: None


def _native():
    """The binding's native module (csrc/sdq_python.cpp), loaded at first use like the CUDA library."""
    global _fast
    if _fast is None:
        lib()
        try:
            loader = importlib.machinery.ExtensionFileLoader("_binding", BINDING)
            mod = importlib.util.module_from_spec(importlib.util.spec_from_loader("_binding", loader))
            loader.exec_module(mod)
            mod.bind(_Act, _Packed, Config, QuantAct, PackedWeight, SdqError, _Mx4, Mx4Matrix, Mx4Experts)
        except ImportError as e:
            warnings.warn("the binding's native half does not load (%s): calls go through ctypes, 6 to 12 us slower each; "
                          "`python -c 'import __graft_entry__ as g; g.build()'` builds it for this torch" % e)
            mod = _NoNative()
        _fast = mod
    return _fast


def _check(code: int, where: str):
    if code != 0:
        raise SdqError(code, where)


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _need_cuda(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (the SDQ path has no CPU fallback)" % name)


@dataclass
class PackedWeight:
    """A decomposed + packed weight matrix: caller-owned device buffer plus its host descriptor."""
    buf: torch.Tensor
    desc: _Packed
    N: int
    K: int
    cfg: Config
    algorithmic_bytes: int


@dataclass
class QuantAct:
    buf: torch.Tensor
    desc: _Act
    M: int
    K: int
    cfg: Config


def packed_size(N: int, K: int, cfg: Config):
    b, a = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().sdq_packed_size(N, K, ctypes.byref(cfg), ctypes.byref(b), ctypes.byref(a)), "sdq_packed_size")
    return b.value, a.value


def act_size(M: int, K: int, cfg: Config) -> int:
    b = ctypes.c_size_t()
    _check(lib().sdq_act_size(M, K, ctypes.byref(cfg), ctypes.byref(b)), "sdq_act_size")
    return b.value


def sdq_decompose(W: torch.Tensor, cfg: Config | None = None, buf: torch.Tensor | None = None,
                  col_weight: torch.Tensor | None = None) -> PackedWeight:
    """W [N, K] bf16 CUDA tensor -> packed inlier/outlier parts (sdq_decompose of the C-ABI; with col_weight [K] fp32,
    sdq_decompose_metric: selections rank by the weight-activation product |w| * col_weight[k])."""
    cfg = cfg or Config()
    p = (_fast or _native()).decompose(W, cfg, buf, col_weight)
    if p is not None:
        return p
    _need_cuda(W, "W")
    assert W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    N, K = W.shape
    nbytes, algo = packed_size(N, K, cfg)
    if buf is None:
        buf = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    d = _Packed()
    if col_weight is None:
        _check(lib().sdq_decompose(W.data_ptr(), N, K, W.stride(0), ctypes.byref(cfg), buf.data_ptr(), buf.numel(),
                                   ctypes.byref(d), _stream()), "sdq_decompose")
    else:
        _need_cuda(col_weight, "col_weight")
        assert col_weight.dtype == torch.float32 and col_weight.shape == (K,) and col_weight.is_contiguous()
        _check(lib().sdq_decompose_metric(W.data_ptr(), N, K, W.stride(0), ctypes.byref(cfg), col_weight.data_ptr(), buf.data_ptr(),
                                          buf.numel(), ctypes.byref(d), _stream()), "sdq_decompose_metric")
    return PackedWeight(buf, d, N, K, cfg, algo)


def packed_attach(buf: torch.Tensor) -> PackedWeight:
    """uint8 CUDA tensor holding a packed buffer (e.g. restored from a file) -> PackedWeight, from the buffer's own header."""
    _need_cuda(buf, "buf")
    assert buf.dtype == torch.uint8 and buf.is_contiguous()
    d = _Packed()
    _check(lib().sdq_packed_attach(buf.data_ptr(), buf.numel(), ctypes.byref(d), _stream()), "sdq_packed_attach")
    cfg = Config(d.cfg.out_n, d.cfg.in_gran, d.cfg.in_block, d.cfg.scale_rule, d.cfg.out_order, d.cfg.out_fmt)
    _, algo = packed_size(d.N, d.K, cfg)
    return PackedWeight(buf, d, d.N, d.K, cfg, algo)


def packed_compact(p: PackedWeight) -> PackedWeight:
    """The packed matrix without its 2:4 outlier containers (4.2 instead of 9.1 bits per weight): the form the grouped
    few-token calls stream.  Returns a new PackedWeight in its own buffer (see sdq_packed_compact in include/sdq.h)."""
    q = (_fast or _native()).compact(p)
    if q is not None:
        return q
    n = ctypes.c_size_t(0)
    _check(lib().sdq_packed_compact_size(ctypes.c_int64(p.N), ctypes.c_int64(p.K), ctypes.byref(p.cfg), ctypes.byref(n)), "sdq_packed_compact_size")
    buf = torch.empty(int(n.value), dtype=torch.uint8, device=p.buf.device)
    d = _Packed()
    _check(lib().sdq_packed_compact(ctypes.byref(p.desc), ctypes.c_void_p(buf.data_ptr()), ctypes.c_size_t(buf.numel()), ctypes.byref(d), _stream()),
           "sdq_packed_compact")
    return PackedWeight(buf, d, p.N, p.K, p.cfg, p.algorithmic_bytes)


def diag_wait_timeout(polls: int = 64) -> None:
    """Enqueues the failure-detection self-test: a bounded device-side wait that is made to run out (include/sdq_diag.h)."""
    _check(lib().sdq_diag_wait_timeout(polls, _stream()), "sdq_diag_wait_timeout")


def channel_norm(X: torch.Tensor) -> torch.Tensor:
    """X [M, K] bf16 CUDA tensor -> fp32 [K]: Euclidean norm of every input channel over the tokens
    (the per-channel weight of the product metric)."""
    c = (_fast or _native()).channel_norm(X)
    if c is not None:
        return c
    _need_cuda(X, "X")
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M, K = X.shape
    c = torch.empty(K, dtype=torch.float32, device=X.device)
    _check(lib().sdq_channel_norm(X.data_ptr(), M, K, X.stride(0), c.data_ptr(), _stream()), "sdq_channel_norm")
    return c


def sdq_quantize_act(X: torch.Tensor, cfg: Config | None = None, buf: torch.Tensor | None = None) -> QuantAct:
    """X [M, K] bf16 CUDA tensor -> 4-bit block-scaled and 8-bit per-token-scaled activations."""
    cfg = cfg or Config()
    q = (_fast or _native()).quantize_act(X, cfg, buf)
    if q is not None:
        return q
    _need_cuda(X, "X")
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M, K = X.shape
    if buf is None:
        buf = torch.empty(act_size(M, K, cfg), dtype=torch.uint8, device=X.device)
    d = _Act()
    _check(lib().sdq_quantize_act(X.data_ptr(), M, K, X.stride(0), ctypes.byref(cfg), buf.data_ptr(), buf.numel(),
                                  ctypes.byref(d), _stream()), "sdq_quantize_act")
    return QuantAct(buf, d, M, K, cfg)


def workspace_size(M: int, N: int, K: int, cfg: Config) -> int:
    b = ctypes.c_size_t()
    _check(lib().sdq_workspace_size(M, N, K, ctypes.byref(cfg), ctypes.byref(b)), "sdq_workspace_size")
    return b.value


def make_workspace(M: int, N: int, K: int, cfg: Config, device) -> torch.Tensor | None:
    """Allocates (with torch) and zeroes the split-K scratch buffer for a call shape; None if none is needed."""
    n = workspace_size(M, N, K, cfg)
    if n == 0:
        return None
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _check(lib().sdq_workspace_init(ws.data_ptr(), ws.numel(), _stream()), "sdq_workspace_init")
    return ws


def sdq_linear(xq: QuantAct, p: PackedWeight, out: torch.Tensor | None = None, f32: bool = False,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y [M, N] = A_i W_i^T + A_o W_o^T (bf16, or the fp32 accumulator itself with f32=True).
    `workspace` (from make_workspace) enables the split-K path for few tokens."""
    y = (_fast or _native()).linear(xq, p, out, f32, workspace)
    if y is not None:
        return y
    dt = torch.float32 if f32 else torch.bfloat16
    if out is None:
        out = torch.empty((xq.M, p.N), dtype=dt, device=p.buf.device)
    assert out.dtype == dt and out.shape == (xq.M, p.N) and out.stride(1) == 1
    if workspace is None:
        fn = lib().sdq_linear_f32 if f32 else lib().sdq_linear
        _check(fn(ctypes.byref(xq.desc), ctypes.byref(p.desc), out.data_ptr(), out.stride(0), _stream()), "sdq_linear")
    else:
        fn = lib().sdq_linear_f32_ws if f32 else lib().sdq_linear_ws
        _check(fn(ctypes.byref(xq.desc), ctypes.byref(p.desc), out.data_ptr(), out.stride(0), workspace.data_ptr(),
                  workspace.numel(), _stream()), "sdq_linear_ws")
    return out


def sdq_linear_group(xqs, ps, outs=None, f32: bool = False):
    """Y[i] = sdq_linear(xqs[i], ps[i]) for independent layers in one call (one persistent launch when every layer has few
    tokens and the group is large enough; see sdq_linear_group in include/sdq.h).  Returns the list of outputs."""
    ys = (_fast or _native()).linear_group(xqs, ps, outs, f32)
    if ys is not None:
        return ys
    n = len(ps)
    assert n == len(xqs) and n > 0
    dt = torch.float32 if f32 else torch.bfloat16
    if outs is None:
        outs = [torch.empty((x.M, p.N), dtype=dt, device=p.buf.device) for x, p in zip(xqs, ps)]
    for o, x, p in zip(outs, xqs, ps):
        assert o.dtype == dt and o.shape == (x.M, p.N) and o.stride(1) == 1
    XA = (ctypes.POINTER(_Act) * n)(*[ctypes.pointer(x.desc) for x in xqs])
    PA = (ctypes.POINTER(_Packed) * n)(*[ctypes.pointer(p.desc) for p in ps])
    YA = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    LD = (ctypes.c_int64 * n)(*[o.stride(0) for o in outs])
    fn = lib().sdq_linear_group_f32 if f32 else lib().sdq_linear_group
    _check(fn(n, XA, PA, YA, LD, _stream()), "sdq_linear_group")
    return outs


def sdq_linear_group_x(X: torch.Tensor, ps, outs=None, f32: bool = False):
    """Y[i] = sdq_linear(sdq_quantize_act(X), ps[i]) for layers that share the bf16 activations X [M <= 16, K], in one call (see
    sdq_linear_group_x_ws in include/sdq.h; the ctypes way takes sdq_linear_group_x, which needs no scratch).  Returns the list
    of outputs."""
    ys = (_fast or _native()).linear_group_x(X, ps, outs, f32)
    if ys is not None:
        return ys
    _need_cuda(X, "X")
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    n, M, K = len(ps), X.shape[0], X.shape[1]
    assert n > 0
    dt = torch.float32 if f32 else torch.bfloat16
    if outs is None:
        outs = [torch.empty((M, p.N), dtype=dt, device=X.device) for p in ps]
    for o, p in zip(outs, ps):
        assert o.dtype == dt and o.shape == (M, p.N) and o.stride(1) == 1
    PA = (ctypes.POINTER(_Packed) * n)(*[ctypes.pointer(p.desc) for p in ps])
    YA = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    LD = (ctypes.c_int64 * n)(*[o.stride(0) for o in outs])
    fn = lib().sdq_linear_group_x_f32 if f32 else lib().sdq_linear_group_x
    _check(fn(n, ctypes.c_void_p(X.data_ptr()), ctypes.c_int64(M), ctypes.c_int64(K), ctypes.c_int64(X.stride(0)), PA, YA, LD, _stream()),
           "sdq_linear_group_x")
    return outs


def diag_l2_copy(src: torch.Tensor, slot_bytes: int, nslot: int, iters: int, issuers: int = 1) -> int:
    """Enqueues the copy-only L2 -> shared-memory kernel on `src` (uint8 CUDA tensor); returns the bytes it stages."""
    _need_cuda(src, "src")
    n = ctypes.c_size_t(0)
    _check(lib().sdq_diag_l2_copy(src.data_ptr(), src.numel() * src.element_size(), slot_bytes, nslot, issuers, iters, ctypes.byref(n), _stream()),
           "sdq_diag_l2_copy")
    return int(n.value)


STATIC_WS_BYTES = 4 << 20


def sdq_linear_noalloc(xq: QuantAct, p: PackedWeight, out: torch.Tensor) -> torch.Tensor:
    """sdq_linear for callers that may not allocate device memory: the split-K scratch is a fixed array inside the
    library (STATIC_WS_BYTES); `out` must be supplied.  Calls that can overlap on the GPU must not share it."""
    assert out.dtype == torch.bfloat16 and out.shape == (xq.M, p.N) and out.stride(1) == 1
    _check(lib().sdq_linear_noalloc(ctypes.byref(xq.desc), ctypes.byref(p.desc), out.data_ptr(), out.stride(0), _stream()),
           "sdq_linear_noalloc")
    return out


def packed_export(p: PackedWeight) -> dict:
    N, K, on = p.N, p.K, p.cfg.out_n
    dev = p.buf.device
    dense = p.cfg.in_gran >= GRAN_DENSE
    nmeta = 0 if dense else (K // 8 if p.cfg.in_gran == GRAN_PAIR else K // 4)
    t = dict(in_code=torch.zeros((N, K if dense else K // 2), dtype=torch.uint8, device=dev),
             in_meta=torch.zeros((N, nmeta), dtype=torch.uint8, device=dev),
             in_scale=torch.zeros((N, K // p.cfg.in_block), dtype=torch.uint8, device=dev),
             out_code=torch.zeros((N, K // 8, max(on, 1)), dtype=torch.uint8, device=dev),
             out_idx=torch.zeros((N, K // 8, max(on, 1)), dtype=torch.uint8, device=dev),
             out_sexp=torch.zeros((N,), dtype=torch.int32, device=dev),
             in_texp=torch.zeros((N,), dtype=torch.int32, device=dev))
    c = _Canon(*[t[n].data_ptr() for n in ("in_code", "in_meta", "in_scale", "out_code", "out_idx", "out_sexp", "in_texp")])
    _check(lib().sdq_packed_export(ctypes.byref(p.desc), ctypes.byref(c), _stream()), "sdq_packed_export")
    if on == 0:
        t["out_code"] = t["out_code"][:, :, :0]
        t["out_idx"] = t["out_idx"][:, :, :0]
    return t


def act_export(xq: QuantAct) -> dict:
    M, K = xq.M, xq.K
    dev = xq.buf.device
    t = dict(xq4_code=torch.zeros((M, K), dtype=torch.uint8, device=dev),
             xq4_scale=torch.zeros((M, K // xq.cfg.in_block), dtype=torch.uint8, device=dev),
             xq8_code=torch.zeros((M, K), dtype=torch.uint8, device=dev),
             xq8_sexp=torch.zeros((M,), dtype=torch.int32, device=dev))
    c = _ActCanon(*[t[n].data_ptr() for n in ("xq4_code", "xq4_scale", "xq8_code", "xq8_sexp")])
    _check(lib().sdq_act_export(ctypes.byref(xq.desc), ctypes.byref(c), _stream()), "sdq_act_export")
    return t


# ---- plain microscaled 4-bit matrices and the expert layer over them (include/sdq_mx4.h) ------------------------------------
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


@dataclass
class Mx4Matrix:
    """A matrix in MXFP4 or NVFP4 (weights or activations): device buffer plus host descriptor."""
    buf: torch.Tensor
    desc: _Mx4
    R: int
    K: int
    fmt: int


@dataclass
class Mx4Experts:
    """E stacked weight matrices [R, K] in MXFP4, in the form sdq_mx4_moe streams."""
    buf: torch.Tensor
    desc: _Mx4
    E: int
    R: int
    K: int


def _operand(t, name: str, dtypes, dim: int, rows_only: bool = True) -> torch.Tensor:
    """a CUDA tensor of the current device, of one of the types and as many dimensions, its last one dense"""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    _need_cuda(t, name)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, the current device is cuda:%d" % (name, t.device, torch.cuda.current_device()))
    if t.dtype not in dtypes:
        raise ValueError("%s has type %s, not one of %s" % (name, t.dtype, ", ".join(str(d) for d in dtypes)))
    if t.dim() != dim:
        raise ValueError("%s has %d dimensions, not %d" % (name, t.dim(), dim))
    if t.shape[-1] > 1 and t.stride(-1) != 1 or not rows_only and not t.is_contiguous():
        raise ValueError("%s must be contiguous%s" % (name, " along its last dimension" if rows_only else ""))
    return t


def _row_stride(t: torch.Tensor) -> int:
    """elements from one row to the next (of a single row: its length)"""
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError("rows overlap")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _buffer(buf, nbytes: int, device) -> torch.Tensor:
    if buf is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    return _operand(buf, "buf", (torch.uint8,), 1, False)


def _same_device(q, name: str):
    if q.buf.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, the current device is cuda:%d" % (name, q.buf.device, torch.cuda.current_device()))


def mx4_size(R: int, K: int, fmt: int = FMT_MXFP4) -> int:
    b = ctypes.c_size_t()
    _check(lib().sdq_mx4_size(R, K, fmt, ctypes.byref(b)), "sdq_mx4_size")
    return b.value


def sdq_mx4_quantize(X: torch.Tensor, fmt: int = FMT_MXFP4, rule: int = SCALE_OCP_FLOOR, buf: torch.Tensor | None = None) -> Mx4Matrix:
    """X [R, K] (bf16, fp16 or fp32 CUDA tensor; any sizes, rows may be strided) -> MXFP4 or NVFP4, weights and activations alike."""
    q = (_fast or _native()).mx4_quantize(X, fmt, rule, buf)
    if q is not None:
        return q
    _operand(X, "X", _DTYPES, 2)
    R, K = X.shape
    buf = _buffer(buf, mx4_size(R, K, fmt), X.device)
    d = _Mx4()
    _check(lib().sdq_mx4_quantize(X.data_ptr(), _DTYPES[X.dtype], R, K, _row_stride(X), fmt, rule, buf.data_ptr(), buf.numel(), ctypes.byref(d), _stream()),
           "sdq_mx4_quantize")
    return Mx4Matrix(buf, d, R, K, fmt)


def sdq_mx4_import(codes: torch.Tensor, scales: torch.Tensor, fmt: int = FMT_MXFP4, K: int | None = None, factor: torch.Tensor | None = None,
                   buf: torch.Tensor | None = None) -> Mx4Matrix:
    """Packed codes [R, ceil(K / 2)] and scale codes [R, ceil(K / 32)] (NVFP4: ceil(K / 16), with an fp32 factor [R] or None) as a
    checkpoint holds them -> Mx4Matrix.  K defaults to twice the code bytes."""
    _operand(codes, "codes", (torch.uint8,), 2, False)
    R = codes.shape[0]
    K = 2 * codes.shape[1] if K is None else K
    nbytes = mx4_size(R, K, fmt)
    _operand(scales, "scales", (torch.uint8,), 2, False)
    if codes.shape[1] != (K + 1) // 2 or tuple(scales.shape) != (R, -(-K // (16 if fmt == FMT_NVFP4 else 32))):
        raise ValueError("codes %s and scales %s do not belong to a [%d, %d] matrix" % (tuple(codes.shape), tuple(scales.shape), R, K))
    if factor is not None:
        if fmt != FMT_NVFP4:
            raise ValueError("only NVFP4 has row factors")
        _operand(factor, "factor", (torch.float32,), 1, False)
        if factor.shape[0] != R:
            raise ValueError("factor has %d entries for %d rows" % (factor.shape[0], R))
    buf = _buffer(buf, nbytes, codes.device)
    d = _Mx4()
    _check(lib().sdq_mx4_import(codes.data_ptr(), scales.data_ptr(), None if factor is None else factor.data_ptr(), R, K, fmt, buf.data_ptr(), buf.numel(),
                                ctypes.byref(d), _stream()), "sdq_mx4_import")
    return Mx4Matrix(buf, d, R, K, fmt)


def mx4_export(q) -> dict:
    """Plain arrays of an Mx4Matrix or Mx4Experts: code (two to a byte), scale and, for NVFP4, factor, shaped as sdq_mx4_import and
    sdq_mx4_experts_import take them."""
    _same_device(q, "q")
    experts, nv = isinstance(q, Mx4Experts), q.desc.fmt == FMT_NVFP4
    lead = (q.E, q.R) if experts else (q.R,)
    t = dict(code=torch.empty(lead + ((q.K + 1) // 2,), dtype=torch.uint8, device=q.buf.device),
             scale=torch.empty(lead + (-(-q.K // (16 if nv else 32)),), dtype=torch.uint8, device=q.buf.device))
    if nv:
        t["factor"] = torch.empty(q.R, dtype=torch.float32, device=q.buf.device)
    _check(lib().sdq_mx4_export(ctypes.byref(q.desc), t["code"].data_ptr(), t["scale"].data_ptr(), t["factor"].data_ptr() if nv else None, _stream()),
           "sdq_mx4_export")
    return t


def sdq_mx4_dequantize(q, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values an Mx4Matrix ([R, K]) or Mx4Experts ([E, R, K]) holds."""
    if dtype not in _DTYPES:
        raise ValueError("no output of type %s" % dtype)
    if out is None:
        y = (_fast or _native()).mx4_dequantize(q, _DTYPES[dtype])
        if y is not None:
            return y
    _same_device(q, "q")
    experts = isinstance(q, Mx4Experts)
    shape = (q.E, q.R, q.K) if experts else (q.R, q.K)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.buf.device)
    else:
        _operand(out, "out", (dtype,), len(shape), not experts)
        if tuple(out.shape) != shape:
            raise ValueError("out has shape %s, not %s" % (tuple(out.shape), shape))
    _check(lib().sdq_mx4_dequantize(ctypes.byref(q.desc), out.data_ptr(), _DTYPES[dtype], q.K if experts else _row_stride(out), _stream()), "sdq_mx4_dequantize")
    return out


def sdq_mx4_experts(W: torch.Tensor, rule: int = SCALE_OCP_FLOOR) -> Mx4Experts:
    """W [E, R, K] (bf16, fp16 or fp32, contiguous CUDA tensor) -> the experts' MXFP4 form."""
    _operand(W, "W", _DTYPES, 3, False)
    E, R, K = W.shape
    b = ctypes.c_size_t()
    _check(lib().sdq_mx4_experts_size(E, R, K, ctypes.byref(b)), "sdq_mx4_experts_size")
    buf = torch.empty(b.value, dtype=torch.uint8, device=W.device)
    d = _Mx4()
    _check(lib().sdq_mx4_experts_quantize(W.data_ptr(), _DTYPES[W.dtype], E, R, K, rule, buf.data_ptr(), buf.numel(), ctypes.byref(d), _stream()),
           "sdq_mx4_experts_quantize")
    return Mx4Experts(buf, d, E, R, K)


def sdq_mx4_experts_import(codes: torch.Tensor, scales: torch.Tensor, K: int | None = None) -> Mx4Experts:
    """Packed codes [E, R, ceil(K / 2)] and E8M0 scale codes [E, R, ceil(K / 32)] as a checkpoint holds them -> the experts' form."""
    _operand(codes, "codes", (torch.uint8,), 3, False)
    _operand(scales, "scales", (torch.uint8,), 3, False)
    E, R = codes.shape[:2]
    K = 2 * codes.shape[2] if K is None else K
    b = ctypes.c_size_t()
    _check(lib().sdq_mx4_experts_size(E, R, K, ctypes.byref(b)), "sdq_mx4_experts_size")
    if codes.shape[2] != (K + 1) // 2 or tuple(scales.shape) != (E, R, -(-K // 32)):
        raise ValueError("codes %s and scales %s do not belong to [%d, %d, %d] experts" % (tuple(codes.shape), tuple(scales.shape), E, R, K))
    buf = torch.empty(b.value, dtype=torch.uint8, device=codes.device)
    d = _Mx4()
    _check(lib().sdq_mx4_experts_import(codes.data_ptr(), scales.data_ptr(), E, R, K, buf.data_ptr(), buf.numel(), ctypes.byref(d), _stream()),
           "sdq_mx4_experts_import")
    return Mx4Experts(buf, d, E, R, K)


def sdq_mx4_linear(xq: Mx4Matrix, wq: Mx4Matrix, bias: torch.Tensor | None = None, out: torch.Tensor | None = None,
                   dtype: torch.dtype | None = None) -> torch.Tensor:
    """Y [M, N] = Xq Wq^T + bias, fp32 sums on the tensor core, rounded once to `dtype` (of `out` if that is given, else bf16)."""
    dtype = dtype or (out.dtype if out is not None else torch.bfloat16)
    if dtype not in _DTYPES:
        raise ValueError("no output of type %s" % dtype)
    y = (_fast or _native()).mx4_linear(xq, wq, bias, out, _DTYPES[dtype])
    if y is not None:
        return y
    _same_device(xq, "xq")
    _same_device(wq, "wq")
    if bias is not None:
        _operand(bias, "bias", (dtype,), 1, False)
        if bias.shape[0] != wq.R:
            raise ValueError("bias has %d entries for %d outputs" % (bias.shape[0], wq.R))
    if out is None:
        out = torch.empty((xq.R, wq.R), dtype=dtype, device=wq.buf.device)
    else:
        _operand(out, "out", (dtype,), 2)
        if tuple(out.shape) != (xq.R, wq.R):
            raise ValueError("out has shape %s, not %s" % (tuple(out.shape), (xq.R, wq.R)))
    _check(lib().sdq_mx4_linear(ctypes.byref(xq.desc), ctypes.byref(wq.desc), None if bias is None else bias.data_ptr(), _DTYPES[dtype], out.data_ptr(),
                                _row_stride(out), _stream()), "sdq_mx4_linear")
    return out


def sdq_moe_route(X: torch.Tensor, router: torch.Tensor, k: int, bias: torch.Tensor | None = None, scoring: int = ROUTE_SOFTMAX, renorm: bool = True,
                  scale: float = 1.0):
    """X [T, H], router [E, H] (one type of bf16, fp16, fp32) -> (ids int32 [T, k], weights fp32 [T, k]): the k experts of the largest score
    (softmax or sigmoid of X router^T) + bias (fp32 [E]), in descending order, and their scores, divided by their sum if `renorm`, times
    `scale`."""
    r = (_fast or _native()).moe_route(X, router, k, bias, scoring, renorm, float(scale))
    if r is not None:
        return r
    _operand(X, "X", _DTYPES, 2)
    _operand(router, "router", (X.dtype,), 2)
    T, H = X.shape
    E = router.shape[0]
    if router.shape[1] != H:
        raise ValueError("router has %d channels, X %d" % (router.shape[1], H))
    if bias is not None:
        _operand(bias, "bias", (torch.float32,), 1, False)
        if bias.shape[0] != E:
            raise ValueError("bias has %d entries for %d experts" % (bias.shape[0], E))
    ids = torch.empty((T, k), dtype=torch.int32, device=X.device)
    weights = torch.empty((T, k), dtype=torch.float32, device=X.device)
    _check(lib().sdq_moe_route(X.data_ptr(), _DTYPES[X.dtype], T, H, _row_stride(X), router.data_ptr(), E, _row_stride(router),
                               None if bias is None else bias.data_ptr(), k, scoring, int(renorm), scale, ids.data_ptr(), weights.data_ptr(), _stream()),
           "sdq_moe_route")
    return ids, weights


def mx4_moe_workspace(T: int, k: int, H: int, I: int, device) -> torch.Tensor:
    """Scratch of sdq_mx4_moe for up to T tokens and k choices; calls that can overlap on the GPU must not share one."""
    b = ctypes.c_size_t()
    _check(lib().sdq_mx4_moe_workspace_size(T, k, H, I, ctypes.byref(b)), "sdq_mx4_moe_workspace_size")
    return torch.empty(b.value, dtype=torch.uint8, device=device)


def sdq_mx4_moe(X: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, w1: Mx4Experts, w3: Mx4Experts, w2: Mx4Experts,
                out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y[t] = sum_j weights[t, j] * W2[e](silu(W1[e] x_t) * W3[e] x_t), e = ids[t, j], for up to 64 tokens.  X [T, H] bf16 or fp16, ids int32 and
    weights fp32 [T, k]; ids outside [0, E) add nothing.  `workspace` from mx4_moe_workspace (else allocated for the call)."""
    y = (_fast or _native()).mx4_moe(X, ids, weights, w1, w3, w2, out, workspace)
    if y is not None:
        return y
    _operand(X, "X", (torch.bfloat16, torch.float16), 2)
    T, H = X.shape
    _operand(ids, "ids", (torch.int32,), 2, False)
    _operand(weights, "weights", (torch.float32,), 2, False)
    if ids.shape[0] != T or weights.shape != ids.shape:
        raise ValueError("ids %s and weights %s do not belong to %d tokens" % (tuple(ids.shape), tuple(weights.shape), T))
    for n, w in (("w1", w1), ("w3", w3), ("w2", w2)):
        _same_device(w, n)
    k = ids.shape[1]
    if out is None:
        out = torch.empty((T, H), dtype=X.dtype, device=X.device)
    else:
        _operand(out, "out", (X.dtype,), 2)
        if out.shape != X.shape:
            raise ValueError("out has shape %s, not %s" % (tuple(out.shape), tuple(X.shape)))
    if workspace is None:
        workspace = mx4_moe_workspace(T, k, H, w1.R, X.device)
    else:
        _operand(workspace, "workspace", (torch.uint8,), 1, False)
    _check(lib().sdq_mx4_moe(X.data_ptr(), _DTYPES[X.dtype], T, H, _row_stride(X), ids.data_ptr(), weights.data_ptr(), k, ctypes.byref(w1.desc),
                             ctypes.byref(w3.desc), ctypes.byref(w2.desc), out.data_ptr(), _row_stride(out), workspace.data_ptr(), workspace.numel(), _stream()),
           "sdq_mx4_moe")
    return out


def device_status() -> int:
    """Synchronises the current stream and returns (and clears) the sticky device-side status."""
    return lib().sdq_device_status(_stream())

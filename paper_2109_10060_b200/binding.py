"""ctypes binding of libdsn: same names as the C ABI, argument marshalling only.

Tensors are torch CUDA tensors (PyTorch supplies device memory and streams, nothing else);
slice-width lists are Python ints.  Every compute step runs inside the library's kernels.
Loading fails loudly when the shared library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libdsn.so")

OK = 0
ERR_INVALID_ARG, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_UNSUPPORTED = -1, -2, -3, -4
ERR_BAD_INDEX, ERR_CUDA, ERR_TIMEOUT, ERR_NONFINITE, ERR_CACHE_FULL = -5, -6, -7, -8, -9
F32, BF16 = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU = 0, 1, 2
INPUT_ORDER, GROUPED = 0, 1
TAIL_UNTOUCHED, TAIL_ZERO = 0, 1
ROTARY_SHARED, ROTARY_PER_AXIS = 0, 1
ROTARY_HALVES, ROTARY_INTERLEAVED = 0, 1
LAYER_LINEAR, LAYER_CONV, LAYER_ATTENTION, LAYER_DEPTHWISE = 0, 1, 2, 3
MAX_SLICES, MAX_GROUPS, MAX_CHAIN = 64, 4096, 6

EXPORTS = [
    "dsn_create", "dsn_destroy", "dsn_strerror", "dsn_get_status", "dsn_set_wait_limit", "dsn_selftest_bounded_wait", "dsn_map_cache_stats", "dsn_get_stats", "dsn_widths_from_ratios",
    "dsn_executed_macs", "dsn_gate_workspace_bytes", "dsn_gate", "dsn_gate_static", "dsn_gate_attention", "dsn_scale_channels", "dsn_resbn_fold", "dsn_route", "dsn_permute_rows",
    "dsn_sliced_attention", "dsn_sliced_depthwise", "dsn_linear_workspace_bytes", "dsn_conv_workspace_bytes", "dsn_sliced_linear", "dsn_sliced_conv",
    "dsn_layer_workspace_bytes", "dsn_layer_forward",
    "dsn_rmsnorm_quant", "dsn_linear_i8_workspace_bytes", "dsn_sliced_linear_i8", "dsn_rotary_axes",
    "dsn_cache_bytes", "dsn_cache_reset", "dsn_cache_plan", "dsn_cache_write_q4", "dsn_cache_attention_q4_workspace_bytes",
    "dsn_cache_attention_q4",
]


class DsnError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: dsn status {code}")
        self.code = code


class Routing(C.Structure):
    _fields_ = [("B", C.c_int32), ("G", C.c_int32), ("counts", C.c_void_p), ("offsets", C.c_void_p),
                ("perm", C.c_void_p), ("inv_perm", C.c_void_p), ("group_slice", C.c_void_p)]


class GateDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("R", C.c_int32), ("C_full", C.c_int32),
                ("c_valid", C.c_int32), ("C_mlp", C.c_int32), ("T", C.c_int32), ("ldx", C.c_int64),
                ("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p)]


class LinearDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("R", C.c_int32), ("C_in", C.c_int32), ("C_out", C.c_int32),
                ("ldx", C.c_int64), ("ldw", C.c_int64), ("ldy", C.c_int64), ("T", C.c_int32),
                ("k_in", C.POINTER(C.c_int32)), ("k_out", C.POINTER(C.c_int32)), ("W", C.c_void_p),
                ("bias", C.c_void_p), ("bn_scale", C.c_void_p), ("bn_shift", C.c_void_p), ("residual", C.c_void_p),
                ("act", C.c_int32), ("in_order", C.c_int32), ("out_order", C.c_int32), ("tail", C.c_int32)]


class ConvDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("H", C.c_int32), ("W_", C.c_int32), ("K", C.c_int32), ("pad", C.c_int32),
                ("C_in", C.c_int32), ("C_out", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64),
                ("T", C.c_int32), ("k_in", C.POINTER(C.c_int32)), ("k_out", C.POINTER(C.c_int32)),
                ("W", C.c_void_p), ("bias", C.c_void_p), ("bn_scale", C.c_void_p), ("bn_shift", C.c_void_p),
                ("residual", C.c_void_p), ("act", C.c_int32), ("in_order", C.c_int32), ("out_order", C.c_int32),
                ("tail", C.c_int32)]


class AttentionDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("N", C.c_int32), ("H", C.c_int32), ("D_h", C.c_int32), ("ld_qkv", C.c_int64),
                ("ld_out", C.c_int64), ("T", C.c_int32), ("heads", C.POINTER(C.c_int32)), ("order", C.c_int32)]


class DepthwiseDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("H", C.c_int32), ("W_", C.c_int32), ("K", C.c_int32), ("stride", C.c_int32),
                ("C", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64), ("T", C.c_int32),
                ("c", C.POINTER(C.c_int32)), ("ksize", C.POINTER(C.c_int32)), ("W", C.c_void_p), ("bias", C.c_void_p),
                ("bn_scale", C.c_void_p), ("bn_shift", C.c_void_p), ("act", C.c_int32), ("in_order", C.c_int32),
                ("out_order", C.c_int32)]


class NormDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("R", C.c_int32), ("C", C.c_int32), ("ldx", C.c_int64), ("ld_res", C.c_int64),
                ("ld_sum", C.c_int64), ("ldy", C.c_int64), ("ldq", C.c_int64), ("T", C.c_int32), ("k", C.POINTER(C.c_int32)),
                ("weight", C.c_void_p), ("eps", C.c_float), ("in_order", C.c_int32), ("out_order", C.c_int32)]
    _at = None   # device of the tensors


class LinearI8Desc(C.Structure):
    _fields_ = [("R", C.c_int32), ("C_in", C.c_int32), ("C_out", C.c_int32), ("ldx", C.c_int64), ("ldw", C.c_int64),
                ("ldy", C.c_int64), ("T", C.c_int32), ("k_in", C.POINTER(C.c_int32)), ("k_out", C.POINTER(C.c_int32)),
                ("W", C.c_void_p), ("w_scale", C.c_void_p), ("bias", C.c_void_p), ("bn_scale", C.c_void_p), ("bn_shift", C.c_void_p),
                ("residual", C.c_void_p), ("y_dtype", C.c_int32), ("act", C.c_int32), ("in_order", C.c_int32),
                ("out_order", C.c_int32), ("tail", C.c_int32)]
    _at = None   # device of the tensors


class RotaryDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("N", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("vectors", C.c_int32),
                ("rotated", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64), ("T", C.c_int32), ("heads", C.POINTER(C.c_int32)),
                ("order", C.c_int32), ("n_axes", C.c_int32), ("pairs", C.c_int32 * 3), ("ladder", C.c_int32), ("pairing", C.c_int32),
                ("base", C.c_double), ("shared_positions", C.c_int32), ("inverse", C.c_int32)]


class CacheDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("R", C.c_int32), ("H", C.c_int32), ("D_h", C.c_int32), ("group", C.c_int32), ("page", C.c_int32),
                ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("ld_qkv", C.c_int64), ("ld_out", C.c_int64), ("ld_values", C.c_int64),
                ("T", C.c_int32), ("heads", C.POINTER(C.c_int32)), ("order", C.c_int32), ("scale", C.c_float), ("window", C.c_int32)]


class Cache(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("table", C.c_void_p), ("lengths", C.c_void_p), ("placed", C.c_void_p), ("slots", C.c_void_p),
                ("pool", C.c_void_p), ("pool_state", C.c_void_p)]
    _at = None   # device of the tensors


class Stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("calls", "launches", "launches_gemm_pair", "launches_gemm_halo", "launches_gemm_chain",
                                          "launches_gemm_one_cta", "launches_linear_f32", "launches_attention",
                                          "launches_depthwise", "launches_dwpw", "launches_gate", "launches_route",
                                          "launches_copy", "map_hits", "map_misses", "launches_gemm_chain_tmem",
                                          "launches_norm", "launches_gemm_i8", "launches_rows_i8", "launches_rotary",
                                          "launches_cache_plan", "launches_cache_write", "launches_cache_attention")]


class LayerDesc(C.Structure):
    _fields_ = [("gate", C.POINTER(GateDesc)), ("B", C.c_int32), ("T", C.c_int32), ("n_layers", C.c_int32),
                ("kind", C.c_int32 * MAX_CHAIN), ("layer", C.c_void_p * MAX_CHAIN)]


_lib = None


def load_library():
    """Loads libdsn.so (building it is `python -m paper_2109_10060_b200.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2109_10060_b200.build`; "
                          "there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.dsn_create.argtypes = [C.POINTER(vp), C.c_int]
    lib.dsn_destroy.argtypes = [vp]
    lib.dsn_strerror.argtypes = [C.c_int]
    lib.dsn_strerror.restype = C.c_char_p
    lib.dsn_get_status.argtypes = [vp, vp, C.POINTER(i32), C.POINTER(i32)]
    lib.dsn_set_wait_limit.argtypes = [vp, C.c_uint32, vp]
    lib.dsn_selftest_bounded_wait.argtypes = [vp, vp]
    lib.dsn_get_stats.argtypes = [vp, C.POINTER(Stats)]
    lib.dsn_map_cache_stats.argtypes = [vp, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    lib.dsn_widths_from_ratios.argtypes = [i32, C.POINTER(C.c_double), i32, i32, C.POINTER(i32)]
    lib.dsn_executed_macs.argtypes = [C.POINTER(i32), i32, i32, C.POINTER(i32), C.POINTER(i32), i32]
    lib.dsn_executed_macs.restype = i64
    lib.dsn_gate_workspace_bytes.argtypes = [C.POINTER(GateDesc)]
    lib.dsn_gate_workspace_bytes.restype = sz
    lib.dsn_gate.argtypes = [vp, C.POINTER(GateDesc), vp, vp, vp, vp, sz, vp]
    lib.dsn_gate_static.argtypes = [vp, C.POINTER(GateDesc), vp, vp, vp, vp]
    lib.dsn_gate_attention.argtypes = [vp, C.POINTER(GateDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.dsn_scale_channels.argtypes = [vp, C.POINTER(Routing), i32, i32, i32, i32, i32, vp, i64, vp, vp, i64, vp]
    lib.dsn_resbn_fold.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.dsn_route.argtypes = [vp, vp, i32, i32, C.POINTER(Routing), vp]
    lib.dsn_permute_rows.argtypes = [vp, C.POINTER(Routing), i32, i32, i32, C.POINTER(i32), vp, i64, vp, i64, i32, vp]
    lib.dsn_linear_workspace_bytes.argtypes = [C.POINTER(LinearDesc), i32]
    lib.dsn_linear_workspace_bytes.restype = sz
    lib.dsn_conv_workspace_bytes.argtypes = [C.POINTER(ConvDesc), i32]
    lib.dsn_conv_workspace_bytes.restype = sz
    lib.dsn_sliced_linear.argtypes = [vp, C.POINTER(LinearDesc), C.POINTER(Routing), vp, vp, vp, sz, vp]
    lib.dsn_sliced_conv.argtypes = [vp, C.POINTER(ConvDesc), C.POINTER(Routing), vp, vp, vp, sz, vp]
    lib.dsn_sliced_attention.argtypes = [vp, C.POINTER(AttentionDesc), C.POINTER(Routing), vp, vp, vp]
    lib.dsn_sliced_depthwise.argtypes = [vp, C.POINTER(DepthwiseDesc), C.POINTER(Routing), vp, vp, vp]
    lib.dsn_layer_workspace_bytes.argtypes = [C.POINTER(LayerDesc)]
    lib.dsn_layer_workspace_bytes.restype = sz
    lib.dsn_layer_forward.argtypes = [vp, C.POINTER(LayerDesc), vp, vp, vp, C.POINTER(Routing), vp, vp, sz, vp]
    lib.dsn_rmsnorm_quant.argtypes = [vp, C.POINTER(NormDesc), C.POINTER(Routing), vp, vp, vp, vp, vp, vp, vp]
    lib.dsn_linear_i8_workspace_bytes.argtypes = [C.POINTER(LinearI8Desc), i32]
    lib.dsn_linear_i8_workspace_bytes.restype = sz
    lib.dsn_sliced_linear_i8.argtypes = [vp, C.POINTER(LinearI8Desc), C.POINTER(Routing), vp, vp, vp, vp, sz, vp]
    lib.dsn_rotary_axes.argtypes = [vp, C.POINTER(RotaryDesc), C.POINTER(Routing), vp, vp, vp, vp]
    lib.dsn_cache_bytes.argtypes = [C.POINTER(CacheDesc)]
    lib.dsn_cache_bytes.restype = sz
    lib.dsn_cache_reset.argtypes = [vp, C.POINTER(CacheDesc), C.POINTER(Cache), i32, vp]
    lib.dsn_cache_plan.argtypes = [vp, C.POINTER(CacheDesc), C.POINTER(Cache), i32, vp, vp, vp, vp]
    lib.dsn_cache_write_q4.argtypes = [vp, C.POINTER(CacheDesc), C.POINTER(Cache), C.POINTER(Routing), vp, vp, vp]
    lib.dsn_cache_attention_q4_workspace_bytes.argtypes = [C.POINTER(CacheDesc), i32]
    lib.dsn_cache_attention_q4_workspace_bytes.restype = sz
    lib.dsn_cache_attention_q4.argtypes = [vp, C.POINTER(CacheDesc), C.POINTER(Cache), C.POINTER(Routing), vp, vp, vp, sz, vp]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("dsn_strerror", "dsn_executed_macs") and not name.endswith(("workspace_bytes", "cache_bytes")):
            fn.restype = C.c_int
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _i32_array(vals: Sequence[int]):
    return (C.c_int32 * len(vals))(*[int(v) for v in vals])


def _check(code: int, what: str):
    if code != OK:
        raise DsnError(code, what)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() or None
    return int(stream.cuda_stream) or None


def _current_stream() -> int:
    """Handle of the current device's current stream (torch.cuda.current_stream() builds two Python objects for it, 4 us a call)."""
    global _current_stream
    import torch
    raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    torch.cuda.init()
    if raw and dev:
        _current_stream = lambda: raw(dev())
    else:
        _current_stream = lambda: int(torch.cuda.current_stream().cuda_stream)
    return _current_stream()


def dsn_strerror(code: int) -> str:
    return load_library().dsn_strerror(code).decode()


def dsn_widths_from_ratios(C_full: int, ratios: Sequence[float], granule: int = 0):
    lib = load_library()
    T = len(ratios)
    out = (C.c_int32 * T)()
    _check(lib.dsn_widths_from_ratios(C_full, (C.c_double * T)(*ratios), T, granule, out), "dsn_widths_from_ratios")
    return list(out)


def dsn_executed_macs(counts: Sequence[int], R: int, k_in: Sequence[int], k_out: Sequence[int], K: int = 1) -> int:
    lib = load_library()
    return int(lib.dsn_executed_macs(_i32_array(counts), len(counts), R, _i32_array(k_in), _i32_array(k_out), K))


class Context:
    """Owns a dsn_ctx on one CUDA device."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = device
        self.handle = C.c_void_p()
        _check(self.lib.dsn_create(C.byref(self.handle), device), "dsn_create")

    def close(self):
        if self.handle:
            self.lib.dsn_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_wait_limit(self, microseconds: int, stream=None):
        """Limit of the kernels' bounded waits (0 = the 2 s default)."""
        _check(self.lib.dsn_set_wait_limit(self.handle, int(microseconds), _stream_handle(stream)), "dsn_set_wait_limit")

    def selftest_bounded_wait(self, stream=None):
        """Launches the kernel that waits on a barrier nobody arrives at; it returns after the wait limit."""
        _check(self.lib.dsn_selftest_bounded_wait(self.handle, _stream_handle(stream)), "dsn_selftest_bounded_wait")

    def map_cache_stats(self):
        """(hits, misses) of the context's tensor-map cache."""
        h, m = C.c_uint64(), C.c_uint64()
        _check(self.lib.dsn_map_cache_stats(self.handle, C.byref(h), C.byref(m)), "dsn_map_cache_stats")
        return h.value, m.value

    def stats(self) -> dict:
        """Launch counters of this context (kernels of the library, by family)."""
        st = Stats()
        _check(self.lib.dsn_get_stats(self.handle, C.byref(st)), "dsn_get_stats")
        return {n: int(getattr(st, n)) for n, _ in Stats._fields_}

    def get_status(self, stream=None):
        code, detail = C.c_int32(), C.c_int32()
        _check(self.lib.dsn_get_status(self.handle, _stream_handle(stream), C.byref(code), C.byref(detail)),
               "dsn_get_status")
        return code.value, detail.value


def make_routing(B, G, counts, offsets, perm, inv_perm, group_slice=None) -> Routing:
    r = Routing(B, G, _ptr(counts), _ptr(offsets), _ptr(perm), _ptr(inv_perm), _ptr(group_slice))
    r._keep = (counts, offsets, perm, inv_perm, group_slice)
    return r


def make_gate_desc(dtype, B, R, C_full, C_mlp, T, W1, W2, b1=None, b2=None, c_valid=None, ldx=None) -> GateDesc:
    g = GateDesc(dtype, B, R, C_full, C_full if c_valid is None else c_valid, C_mlp, T,
                 C_full if ldx is None else ldx, _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2))
    g._keep = (W1, W2, b1, b2)
    return g


def make_linear_desc(dtype, R, C_in, C_out, k_in, k_out, W, bias=None, act=ACT_NONE, in_order=INPUT_ORDER,
                     out_order=INPUT_ORDER, tail=TAIL_UNTOUCHED, ldx=None, ldw=None, ldy=None, bn_scale=None,
                     bn_shift=None, residual=None) -> LinearDesc:
    ki, ko = _i32_array(k_in), _i32_array(k_out)
    d = LinearDesc(dtype, R, C_in, C_out, C_in if ldx is None else ldx, C_in if ldw is None else ldw,
                   C_out if ldy is None else ldy, len(k_in), ki, ko, _ptr(W), _ptr(bias), _ptr(bn_scale), _ptr(bn_shift),
                   _ptr(residual), act, in_order, out_order, tail)
    d._keep = (ki, ko, W, bias, bn_scale, bn_shift, residual)
    return d


def make_conv_desc(dtype, H, Wd, K, pad, C_in, C_out, k_in, k_out, W, bias=None, act=ACT_NONE,
                   in_order=INPUT_ORDER, out_order=INPUT_ORDER, tail=TAIL_UNTOUCHED, ldx=None, ldy=None, bn_scale=None,
                   bn_shift=None, residual=None) -> ConvDesc:
    ki, ko = _i32_array(k_in), _i32_array(k_out)
    d = ConvDesc(dtype, H, Wd, K, pad, C_in, C_out, C_in if ldx is None else ldx, C_out if ldy is None else ldy,
                 len(k_in), ki, ko, _ptr(W), _ptr(bias), _ptr(bn_scale), _ptr(bn_shift), _ptr(residual), act, in_order,
                 out_order, tail)
    d._keep = (ki, ko, W, bias, bn_scale, bn_shift, residual)
    return d


def make_layer_desc(B, T, layers, gate: Optional[GateDesc] = None) -> LayerDesc:
    L = LayerDesc()
    L.gate = C.pointer(gate) if gate is not None else None
    L.B, L.T, L.n_layers = B, T, len(layers)
    for j, d in enumerate(layers):
        L.kind[j] = (LAYER_CONV if isinstance(d, ConvDesc) else LAYER_ATTENTION if isinstance(d, AttentionDesc)
                     else LAYER_DEPTHWISE if isinstance(d, DepthwiseDesc) else LAYER_LINEAR)
        L.layer[j] = C.cast(C.pointer(d), C.c_void_p)
    L._keep = (gate, list(layers))
    return L


def dsn_gate_workspace_bytes(g: GateDesc) -> int:
    return int(load_library().dsn_gate_workspace_bytes(C.byref(g)))


def dsn_gate(ctx: Context, g: GateDesc, x, idx_out, logits_out=None, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(ctx.lib.dsn_gate(ctx.handle, C.byref(g), _ptr(x), _ptr(idx_out), _ptr(logits_out), _ptr(workspace),
                            ws_bytes, _stream_handle(stream)), "dsn_gate")


def dsn_gate_static(ctx: Context, g: GateDesc, x, idx_out, logits_out=None, stream=None):
    """dsn_gate without a workspace: for callers that may not allocate device memory (a serving loop
    that must stay out of the allocator, a plug-in that only receives its inputs and outputs).  The
    scratch is a fixed 4 MiB array inside the library, shared by all calls on a GPU, so calls must not
    overlap on the device, and problems beyond 1,048,576 scratch floats raise ERR_WORKSPACE."""
    _check(ctx.lib.dsn_gate_static(ctx.handle, C.byref(g), _ptr(x), _ptr(idx_out), _ptr(logits_out),
                                   _stream_handle(stream)), "dsn_gate_static")


def dsn_gate_attention(ctx: Context, g: GateDesc, W3, b3, x, idx_out, scale_out, logits_out=None, workspace=None,
                       stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(ctx.lib.dsn_gate_attention(ctx.handle, C.byref(g), _ptr(W3), _ptr(b3), _ptr(x), _ptr(idx_out),
                                      _ptr(logits_out), _ptr(scale_out), _ptr(workspace), ws_bytes,
                                      _stream_handle(stream)), "dsn_gate_attention")


def dsn_scale_channels(ctx: Context, routing, to_grouped, dtype, B, R, c_valid, x, ldx, scale, y, ldy, stream=None):
    _check(ctx.lib.dsn_scale_channels(ctx.handle, C.byref(routing) if routing is not None else None,
                                      1 if to_grouped else 0, dtype, B, R, c_valid, _ptr(x), ldx, _ptr(scale), _ptr(y),
                                      ldy, _stream_handle(stream)), "dsn_scale_channels")


def dsn_resbn_fold(ctx: Context, T, Cn, gamma, beta, mu, sigma, scale_out, shift_out, stream=None):
    _check(ctx.lib.dsn_resbn_fold(ctx.handle, T, Cn, _ptr(gamma), _ptr(beta), _ptr(mu), _ptr(sigma), _ptr(scale_out),
                                  _ptr(shift_out), _stream_handle(stream)), "dsn_resbn_fold")


def dsn_route(ctx: Context, idx, B: int, T: int, routing: Routing, stream=None):
    _check(ctx.lib.dsn_route(ctx.handle, _ptr(idx), B, T, C.byref(routing), _stream_handle(stream)), "dsn_route")


def dsn_permute_rows(ctx: Context, routing: Routing, dtype, R, k, src, ld_src, dst, ld_dst, to_grouped, stream=None):
    _check(ctx.lib.dsn_permute_rows(ctx.handle, C.byref(routing), dtype, R, len(k), _i32_array(k), _ptr(src), ld_src,
                                    _ptr(dst), ld_dst, 1 if to_grouped else 0, _stream_handle(stream)),
           "dsn_permute_rows")


def dsn_sliced_linear(ctx: Context, d: LinearDesc, routing: Routing, x, y, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(ctx.lib.dsn_sliced_linear(ctx.handle, C.byref(d), C.byref(routing), _ptr(x), _ptr(y), _ptr(workspace),
                                     ws_bytes, _stream_handle(stream)), "dsn_sliced_linear")


def dsn_sliced_conv(ctx: Context, d: ConvDesc, routing: Routing, x, y, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(ctx.lib.dsn_sliced_conv(ctx.handle, C.byref(d), C.byref(routing), _ptr(x), _ptr(y), _ptr(workspace),
                                   ws_bytes, _stream_handle(stream)), "dsn_sliced_conv")


def make_attention_desc(N, H, D_h, heads, order=INPUT_ORDER, ld_qkv=None, ld_out=None) -> AttentionDesc:
    hs = _i32_array(heads)
    d = AttentionDesc(BF16, N, H, D_h, 3 * H * D_h if ld_qkv is None else ld_qkv, H * D_h if ld_out is None else ld_out,
                      len(heads), hs, order)
    d._keep = (hs,)
    return d


def dsn_sliced_attention(ctx: Context, d: AttentionDesc, routing: Routing, qkv, out, stream=None):
    _check(ctx.lib.dsn_sliced_attention(ctx.handle, C.byref(d), C.byref(routing), _ptr(qkv), _ptr(out),
                                        _stream_handle(stream)), "dsn_sliced_attention")


def make_depthwise_desc(H, Wd, K, stride, Cn, c, ksize, W, bias=None, act=ACT_NONE, in_order=INPUT_ORDER,
                        out_order=INPUT_ORDER, ldx=None, ldy=None, bn_scale=None, bn_shift=None) -> DepthwiseDesc:
    ca, ka = _i32_array(c), _i32_array(ksize)
    d = DepthwiseDesc(BF16, H, Wd, K, stride, Cn, Cn if ldx is None else ldx, Cn if ldy is None else ldy, len(c), ca, ka,
                      _ptr(W), _ptr(bias), _ptr(bn_scale), _ptr(bn_shift), act, in_order, out_order)
    d._keep = (ca, ka, W, bias, bn_scale, bn_shift)
    return d


def dsn_sliced_depthwise(ctx: Context, d: DepthwiseDesc, routing: Routing, x, y, stream=None):
    _check(ctx.lib.dsn_sliced_depthwise(ctx.handle, C.byref(d), C.byref(routing), _ptr(x), _ptr(y),
                                        _stream_handle(stream)), "dsn_sliced_depthwise")


def dsn_layer_workspace_bytes(L: LayerDesc) -> int:
    return int(load_library().dsn_layer_workspace_bytes(C.byref(L)))


def dsn_layer_forward(ctx: Context, L: LayerDesc, x, idx_in, y, workspace, r_out: Optional[Routing] = None,
                      idx_out=None, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(ctx.lib.dsn_layer_forward(ctx.handle, C.byref(L), _ptr(x), _ptr(idx_in), _ptr(y),
                                     C.byref(r_out) if r_out is not None else None, _ptr(idx_out), _ptr(workspace),
                                     ws_bytes, _stream_handle(stream)), "dsn_layer_forward")


# ---- transformer blocks in 8 bits.  These calls also check what a pointer cannot say: type, device, strides and extent of every tensor.

class _Types:
    """torch's types by the library's codes, looked up once."""
    of_code = None

    @classmethod
    def load(cls):
        import torch
        cls.i8, cls.i32, cls.f32 = torch.int8, torch.int32, torch.float32
        cls.of_code = {F32: torch.float32, BF16: torch.bfloat16}
        return cls


def _types():
    return _Types if _Types.of_code else _Types.load()


def _placed(what: str, t, dtype, device: Optional[int]) -> None:
    at = t.get_device()
    if t.dtype is not dtype or at < 0 or (device is not None and at != device):
        raise DsnError(ERR_INVALID_ARG, f"{what}: {t.dtype} on {t.device}, expected {dtype} on cuda" + ("" if device is None else f":{device}"))


def _buf(what: str, t, dtype, need: int, device: Optional[int] = None) -> Optional[int]:
    """Pointer of a dense device tensor of this type with at least `need` elements."""
    if t is None:
        return None
    _placed(what, t, dtype, device)
    if not t.is_contiguous():
        raise DsnError(ERR_INVALID_ARG, f"{what}: not contiguous")
    if t.numel() < need:
        raise DsnError(ERR_INVALID_ARG, f"{what}: {t.numel()} elements, at least {need} are read or written")
    return t.data_ptr()


def _rows(what: str, t, dtype, rows: int, ld: int, width: int, device: Optional[int] = None) -> Optional[int]:
    """Pointer of a device tensor whose memory, from its first element on, holds `rows` rows of `width` elements that lie `ld` apart: a dense
    tensor of any shape, or a view whose inner dimensions are dense and whose outer ones step by `ld` from row to row (a column range of a wider
    buffer).  Expanded and transposed tensors have no such rows: the kernels would run past the storage, or read another order."""
    if t is None:
        return None
    _placed(what, t, dtype, device)
    if not t.is_contiguous():
        step, outer = 1, False   # what the stride of the next dimension outwards has to be
        for n, stride in zip(reversed(t.shape), reversed(t.stride())):
            if n == 1:
                continue
            if stride != step and not outer:
                step, outer = ld, True
            if stride != step:
                raise DsnError(ERR_INVALID_ARG,
                               f"{what}: strides {tuple(t.stride())} of shape {tuple(t.shape)} are not those of rows {ld} elements apart")
            step *= n
    need = _span(rows, ld, width)
    if not (t.is_contiguous() and t.numel() >= need) and t.untyped_storage().nbytes() // t.element_size() - t.storage_offset() < need:
        raise DsnError(ERR_INVALID_ARG, f"{what}: {t.numel()} elements, at least {need} are read or written")
    return t.data_ptr()


def _same_device(**tensors) -> Optional[int]:
    """The one device of a descriptor's tensors (None: it has no tensors); the calls compare it with the context's."""
    at = None
    for what, t in tensors.items():
        if t is None:
            continue
        if at is not None and t.get_device() != at:
            raise DsnError(ERR_INVALID_ARG, f"{what} on cuda:{t.get_device()}, the descriptor's other tensors on cuda:{at}")
        at = t.get_device()
    return at


def _check_desc(d, ctx) -> None:
    if d._at is not None and d._at != ctx.device:
        raise DsnError(ERR_INVALID_ARG, f"{type(d).__name__}: tensors on cuda:{d._at}, the context on cuda:{ctx.device}")


def _span(rows: int, ld: int, width: int) -> int:
    return (rows - 1) * ld + width if rows > 0 else 0


def make_norm_desc(dtype, R, Cn, k, weight=None, eps=1e-6, ldx=None, ld_res=None, ld_sum=None, ldq=None, ldy=None,
                   in_order=INPUT_ORDER, out_order=INPUT_ORDER) -> NormDesc:
    """Residual + root-mean-square norm + 8-bit codes; leading dimensions default to Cn."""
    _buf("weight", weight, _types().f32, Cn)
    ka = _i32_array(k)
    d = NormDesc(dtype, R, Cn, *(Cn if v is None else v for v in (ldx, ld_res, ld_sum, ldy, ldq)), len(k), ka, _ptr(weight), eps,
                 in_order, out_order)
    d._keep, d._at = (ka, weight), _same_device(weight=weight)
    return d


# The calls below look at each tensor in place and hand it to _rows only where it is no dense tensor that holds all rows whole: a Python call
# a tensor is a fifth of the host's time for a small one.

def dsn_rmsnorm_quant(ctx: Context, d: NormDesc, routing: Routing, x, q=None, scale=None, y=None, residual=None, sum_out=None, stream=None):
    ty, rows, dev, Cn = _Types if _Types.of_code else _types(), routing.B * d.R, ctx.device, d.C
    dt = ty.of_code.get(d.dtype)
    n = rows * max(d.ldx, d.ldy, d.ld_res, d.ld_sum, d.ldq)   # a dense tensor of so many elements holds any of the spans
    _check_desc(d, ctx)
    _check(ctx.lib.dsn_rmsnorm_quant(
        ctx.handle, d, routing,
        x.data_ptr() if x is not None and x.dtype is dt and x.get_device() == dev and x.numel() >= n and x.is_contiguous()
        else _rows("x", x, dt, rows, d.ldx, Cn, dev),
        None if residual is None else residual.data_ptr()
        if residual.dtype is dt and residual.get_device() == dev and residual.numel() >= n and residual.is_contiguous()
        else _rows("residual", residual, dt, rows, d.ld_res, Cn, dev),
        None if sum_out is None else sum_out.data_ptr()
        if sum_out.dtype is dt and sum_out.get_device() == dev and sum_out.numel() >= n and sum_out.is_contiguous()
        else _rows("sum_out", sum_out, dt, rows, d.ld_sum, Cn, dev),
        None if q is None else q.data_ptr() if q.dtype is ty.i8 and q.get_device() == dev and q.numel() >= n and q.is_contiguous()
        else _rows("q", q, ty.i8, rows, d.ldq, Cn, dev),
        None if scale is None else _buf("scale", scale, ty.f32, rows, dev),
        None if y is None else y.data_ptr() if y.dtype is dt and y.get_device() == dev and y.numel() >= n and y.is_contiguous()
        else _rows("y", y, dt, rows, d.ldy, Cn, dev),
        _stream_handle(stream)), "dsn_rmsnorm_quant")


def make_linear_i8_desc(R, C_in, C_out, k_in, k_out, W, w_scale, bias=None, bn_scale=None, bn_shift=None, residual=None, y_dtype=BF16,
                        act=ACT_NONE, in_order=INPUT_ORDER, out_order=INPUT_ORDER, tail=TAIL_UNTOUCHED, ldx=None, ldw=None,
                        ldy=None) -> LinearI8Desc:
    """Linear layer on int8 rows and weights; leading dimensions default to the extents."""
    ldx, ldw, ldy = C_in if ldx is None else ldx, C_in if ldw is None else ldw, C_out if ldy is None else ldy
    f = _types().f32
    _rows("W", W, _types().i8, C_out, ldw, C_in)
    for what, t, n in (("w_scale", w_scale, C_out), ("bias", bias, C_out), ("bn_scale", bn_scale, len(k_out) * C_out),
                       ("bn_shift", bn_shift, len(k_out) * C_out)):
        _buf(what, t, f, n)
    ki, ko = _i32_array(k_in), _i32_array(k_out)
    d = LinearI8Desc(R, C_in, C_out, ldx, ldw, ldy, len(k_in), ki, ko, _ptr(W), _ptr(w_scale), _ptr(bias), _ptr(bn_scale), _ptr(bn_shift),
                     _ptr(residual), y_dtype, act, in_order, out_order, tail)
    d._keep = (ki, ko, W, w_scale, bias, bn_scale, bn_shift, residual)
    d._at = _same_device(W=W, w_scale=w_scale, bias=bias, bn_scale=bn_scale, bn_shift=bn_shift)
    return d


def dsn_linear_i8_workspace_bytes(d: LinearI8Desc, B: int) -> int:
    return int(load_library().dsn_linear_i8_workspace_bytes(C.byref(d), B))


def dsn_sliced_linear_i8(ctx: Context, d: LinearI8Desc, routing: Routing, x, x_scale, y, workspace=None, stream=None):
    ty, rows, dev = _Types if _Types.of_code else _types(), routing.B * d.R, ctx.device
    dt, residual, ws_bytes = ty.of_code.get(d.y_dtype), d._keep[-1], 0
    n = rows * d.ldy
    _check_desc(d, ctx)
    if residual is not None and not (residual.dtype is dt and residual.get_device() == dev and residual.numel() >= n
                                     and residual.is_contiguous()):
        _rows("residual", residual, dt, rows, d.ldy, d.C_out, dev)
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise DsnError(ERR_INVALID_ARG,
                           f"workspace: strides {tuple(workspace.stride())} on {workspace.device}, expected a dense tensor on cuda:{dev}")
    _check(ctx.lib.dsn_sliced_linear_i8(
        ctx.handle, d, routing,
        x.data_ptr() if x is not None and x.dtype is ty.i8 and x.get_device() == dev and x.numel() >= rows * d.ldx and x.is_contiguous()
        else _rows("x", x, ty.i8, rows, d.ldx, d.C_in, dev),
        _buf("x_scale", x_scale, ty.f32, rows, dev),
        y.data_ptr() if y is not None and y.dtype is dt and y.get_device() == dev and y.numel() >= n and y.is_contiguous()
        else _rows("y", y, dt, rows, d.ldy, d.C_out, dev),
        _ptr(workspace), ws_bytes, _stream_handle(stream)), "dsn_sliced_linear_i8")


def make_rotary_desc(dtype, N, H, D, heads, pairs, vectors=3, rotated=2, base=10000.0, ladder=ROTARY_SHARED, pairing=ROTARY_HALVES,
                     shared_positions=True, inverse=False, order=INPUT_ORDER, ldx=None, ldy=None) -> RotaryDesc:
    """Rotary positions; `pairs` lists the pairs of elements that follow each axis (one to three axes)."""
    hs = _i32_array(heads)
    if not 1 <= len(pairs) <= 3:
        raise DsnError(ERR_INVALID_ARG, f"make_rotary_desc: {len(pairs)} axes")
    row = H * vectors * D
    d = RotaryDesc(dtype, N, H, D, vectors, rotated, row if ldx is None else ldx, row if ldy is None else ldy, len(heads), hs, order,
                   len(pairs), (C.c_int32 * 3)(*pairs), ladder, pairing, base, int(shared_positions), int(inverse))
    d._keep = (hs,)
    return d


def dsn_rotary_axes(ctx: Context, d: RotaryDesc, routing: Routing, positions, x, y, stream=None):
    ty, rows, dev = _types(), routing.B * d.N, ctx.device
    dt = ty.of_code.get(d.dtype)
    row = d.H * d.vectors * d.D
    _check(ctx.lib.dsn_rotary_axes(ctx.handle, d, routing,
                                   _buf("positions", positions, ty.i32, d.n_axes * (d.N if d.shared_positions else rows), dev),
                                   _rows("x", x, dt, rows, d.ldx, row, dev), _rows("y", y, dt, rows, d.ldy, row, dev),
                                   _stream_handle(stream)), "dsn_rotary_axes")


# ---- attention over a 4-bit cache

def make_cache_desc(R, H, D_h, heads, group=1, page=64, n_pages=1, max_pages=1, order=INPUT_ORDER, scale=0.0, window=0, ld_qkv=None, ld_out=None,
                    ld_values=None) -> CacheDesc:
    """Paged cache of keys and values in 4 bits, rows [head][q x group | k | v][D_h]; leading dimensions default to the rows' extents."""
    hs = _i32_array(heads)
    d = CacheDesc(BF16, R, H, D_h, group, page, n_pages, max_pages, H * (group + 2) * D_h if ld_qkv is None else ld_qkv,
                  H * group * D_h if ld_out is None else ld_out, H * 2 * D_h if ld_values is None else ld_values, len(heads), hs, order, scale,
                  window)
    d._keep = (hs,)
    return d


def dsn_cache_bytes(d: CacheDesc) -> int:
    return int(load_library().dsn_cache_bytes(C.byref(d)))


def make_cache(pages=None, table=None, lengths=None, placed=None, slots=None, pool=None, pool_state=None) -> Cache:
    """Where a cache lies: dense tensors, pages of uint8 (or int8), the others of int32.  A call checks the sizes of those it uses; the others
    may be left out."""
    import torch
    for what, t in (("table", table), ("lengths", lengths), ("placed", placed), ("slots", slots), ("pool", pool), ("pool_state", pool_state)):
        _buf(what, t, torch.int32, 0)
    if pages is not None:
        _buf("pages", pages, torch.int8 if pages.dtype is torch.int8 else torch.uint8, 0)
    c = Cache(*(_ptr(t) for t in (pages, table, lengths, placed, slots, pool, pool_state)))
    c._at = _same_device(pages=pages, table=table, lengths=lengths, placed=placed, slots=slots, pool=pool, pool_state=pool_state)
    c._keep = (pages, table, lengths, placed, slots, pool, pool_state)
    c._n = tuple(-1 if t is None else t.numel() for t in c._keep)
    return c


def _check_cache(what: str, ctx: Context, c: Cache, need) -> None:
    """`need`: least number of elements of pages, table, lengths, placed, slots, pool, pool_state (0: not used)."""
    if c._at is not None and c._at != ctx.device:
        raise DsnError(ERR_INVALID_ARG, f"{what}: cache on cuda:{c._at}, the context on cuda:{ctx.device}")
    for (name, _), have, n in zip(Cache._fields_, c._n, need):
        if 0 <= have < n:
            raise DsnError(ERR_INVALID_ARG, f"{what}: {name} has {have} elements, at least {n} are read or written")


def dsn_cache_reset(ctx: Context, d: CacheDesc, cache: Cache, B: int, stream=None):
    _check_cache("dsn_cache_reset", ctx, cache, (0, 0, B, 0, 0, d.n_pages, 2))
    _check(ctx.lib.dsn_cache_reset(ctx.handle, d, cache, B, _stream_handle(stream)), "dsn_cache_reset")


def dsn_cache_plan(ctx: Context, d: CacheDesc, cache: Cache, B: int, new_tokens, lengths_out=None, pool_state_out=None, stream=None):
    i32, dev = _types().i32, ctx.device
    _check_cache("dsn_cache_plan", ctx, cache, (0, B * d.max_pages, B, B, B * d.R, d.n_pages, 2))
    _check(ctx.lib.dsn_cache_plan(ctx.handle, d, cache, B, _buf("new_tokens", new_tokens, i32, B, dev),
                                  _buf("lengths_out", lengths_out, i32, B, dev), _buf("pool_state_out", pool_state_out, i32, 2, dev),
                                  _stream_handle(stream)), "dsn_cache_plan")


def dsn_cache_write_q4(ctx: Context, d: CacheDesc, cache: Cache, routing: Routing, qkv, values=None, stream=None):
    dt, rows, dev = _types().of_code.get(d.dtype), routing.B * d.R, ctx.device
    _check_cache("dsn_cache_write_q4", ctx, cache, (d.n_pages * d.H * (d.page // 16) * 18 * d.D_h, 0, 0, 0, rows, 0, 0))
    _check(ctx.lib.dsn_cache_write_q4(
        ctx.handle, d, cache, routing,
        qkv.data_ptr() if qkv is not None and qkv.dtype is dt and qkv.get_device() == dev and qkv.numel() >= rows * d.ld_qkv and qkv.is_contiguous()
        else _rows("qkv", qkv, dt, rows, d.ld_qkv, d.H * (d.group + 2) * d.D_h, dev),
        _rows("values", values, dt, rows, d.ld_values, d.H * 2 * d.D_h, dev), _stream_handle(stream)), "dsn_cache_write_q4")


def dsn_cache_attention_q4_workspace_bytes(d: CacheDesc, B: int) -> int:
    return int(load_library().dsn_cache_attention_q4_workspace_bytes(C.byref(d), B))


def dsn_cache_attention_q4(ctx: Context, d: CacheDesc, cache: Cache, routing: Routing, qkv, out, workspace=None, stream=None):
    dt, B, dev, ws_bytes = _types().of_code.get(d.dtype), routing.B, ctx.device, 0
    rows = B * d.R
    _check_cache("dsn_cache_attention_q4", ctx, cache, (d.n_pages * d.H * (d.page // 16) * 18 * d.D_h, B * d.max_pages, B, B, 0, 0, 0))
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise DsnError(ERR_INVALID_ARG,
                           f"workspace: strides {tuple(workspace.stride())} on {workspace.device}, expected a dense tensor on cuda:{dev}")
    _check(ctx.lib.dsn_cache_attention_q4(
        ctx.handle, d, cache, routing,
        qkv.data_ptr() if qkv is not None and qkv.dtype is dt and qkv.get_device() == dev and qkv.numel() >= rows * d.ld_qkv and qkv.is_contiguous()
        else _rows("qkv", qkv, dt, rows, d.ld_qkv, d.H * (d.group + 2) * d.D_h, dev),
        out.data_ptr() if out is not None and out.dtype is dt and out.get_device() == dev and out.numel() >= rows * d.ld_out and out.is_contiguous()
        else _rows("out", out, dt, rows, d.ld_out, d.H * d.group * d.D_h, dev),
        _ptr(workspace), ws_bytes, _stream_handle(stream)), "dsn_cache_attention_q4")

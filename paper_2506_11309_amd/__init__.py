"""Python binding of libswiftspec.so: the tree-verification step of
speculative decoding on AMD Instinct MI355X (gfx950).

Argument marshalling only: every computation runs in the library's HIP
kernels.  PyTorch supplies device memory and the current HIP stream; the
functions below pass tensor pointers, shapes and the stream handle through
the C ABI declared in ``include/swiftspec.h`` and raise ``SwiftSpecError``
on a non-zero status.  There is no fallback: if the compiled library is
missing, importing a function raises.

fp16 tensors may be ``torch.float16`` or ``torch.int16``/``torch.uint16``
views of the same bits.
"""
from __future__ import annotations

import ctypes
import os
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libswiftspec.so")

_lib = None

i32, i64, f32, f64, vp, sz = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double,
                              ctypes.c_void_p, ctypes.c_size_t)

OK, INVALID_ARG, UNSUPPORTED, MISALIGNED, WORKSPACE_TOO_SMALL, BAD_TREE, HIP_ERROR, CAPACITY = range(8)
DEVERR_BAD_TREE, DEVERR_BAD_PREFIX, DEVERR_BAD_ACCEPTED, DEVERR_BAD_GROUPS = 1, 2, 4, 8
WS_HEADER_BYTES = 65536
MAX_TREE = 64
MAX_M = 64
MAX_EXPERTS = 512
MAX_TOPK = 16


class SwiftSpecError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = _load().swiftspec_status_string(status).decode()
        if status == HIP_ERROR:
            msg += f" (hipError {_load().swiftspec_last_hip_error()})"
        super().__init__(f"{where}: {msg} [status {status}]")
        self.status = status


class W4(ctypes.Structure):
    _fields_ = [("qweight", vp), ("scales", vp), ("zeros", vp), ("K", i32), ("N", i32), ("packed", vp)]


class MX4(ctypes.Structure):
    _fields_ = [("codes", vp), ("scales", vp), ("K", i32), ("N", i32), ("E", i32), ("packed", vp)]
    device = None  # index of the GPU that make_mx4 found the codes on
    unpacked = ()  # codes and scales, until prepack_mx4 has read them


class FP8(ctypes.Structure):
    _fields_ = [("codes", vp), ("scales", vp), ("K", i32), ("N", i32), ("E", i32), ("packed", vp)]
    device = None  # index of the GPU that make_fp8 found the codes on
    unpacked = ()  # codes and scales, until prepack_fp8 has read them


class _Scoring(ctypes.Structure):
    _fields_ = [("score", i32), ("groups", i32), ("top_groups", i32), ("group_best", i32), ("renormalize", i32), ("scale", f32),
                ("bias", vp)]


class _Groups(ctypes.Structure):
    _fields_ = [("T", i32), ("k", i32), ("E", i32), ("offsets", vp), ("rows", vp), ("pos", vp)]


class Dims(ctypes.Structure):
    _fields_ = [("H", i32), ("Hq", i32), ("Hkv", i32), ("D", i32), ("F", i32), ("S_max", i32),
                ("eps", f32), ("rope_theta", f32)]


class Layer(ctypes.Structure):
    _fields_ = [("attn_norm", vp), ("mlp_norm", vp), ("wqkv", W4), ("wo", W4), ("wgate", W4),
                ("wup", W4), ("wdown", W4), ("k_cache", vp), ("v_cache", vp)]


_SIGS = {
    "swiftspec_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "swiftspec_last_hip_error": ([], ctypes.c_int),
    "swiftspec_workspace_init": ([vp, sz, vp], ctypes.c_int),
    "swiftspec_draft_tree_attention": ([vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, i32, vp, i32, i32, i32, i32, vp,
                                        f32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_kv_reorganize": ([vp, vp, i32, i64, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, i32, vp, sz, vp],
                                ctypes.c_int),
    "swiftspec_topk_logprobs_workspace_bytes": ([i32], sz),
    "swiftspec_topk_logprobs": ([vp, i32, i32, i32, i32, vp, vp, vp, sz, vp], ctypes.c_int),
    "swiftspec_draft_tree_create": ([i32, i32, ctypes.POINTER(vp)], ctypes.c_int),
    "swiftspec_draft_tree_destroy": ([vp], None),
    "swiftspec_draft_tree_size": ([vp], i32),
    "swiftspec_draft_tree_rows": ([vp], i32),
    "swiftspec_draft_tree_nodes": ([vp, vp, vp, vp, vp, vp], ctypes.c_int),
    "swiftspec_draft_tree_forest": ([vp, vp], ctypes.c_int),
    "swiftspec_draft_tree_select_leaves": ([vp, i32, vp, vp, vp], ctypes.c_int),
    "swiftspec_draft_tree_expand": ([vp, i32, vp, i32, vp, vp], ctypes.c_int),
    "swiftspec_draft_tree_select_subgraph": ([vp, i32, vp, vp, vp, vp], ctypes.c_int),
    "swiftspec_draft_tree_reroot": ([vp, vp, i32, vp, vp, vp, vp, vp], ctypes.c_int),
    "swiftspec_greedy_accept_workspace_bytes": ([i32], sz),
    "swiftspec_greedy_accept": ([vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
    "swiftspec_read_device_error": ([vp, vp, ctypes.POINTER(ctypes.c_uint32)], ctypes.c_int),
    "swiftspec_clock_sample": ([vp, i32, vp], ctypes.c_int),
    "swiftspec_w4_packed_bytes": ([i32, i32], sz),
    "swiftspec_w4_prepack": ([ctypes.POINTER(W4), vp, sz, vp], ctypes.c_int),
    "swiftspec_w4a16_gemm": ([ctypes.POINTER(W4), vp, i32, i32, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_w4a16_gemm_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_w4a16_swiglu": ([ctypes.POINTER(W4), ctypes.POINTER(W4), vp, i32, i32, vp, i32, vp, sz, vp],
                               ctypes.c_int),
    "swiftspec_w4a16_swiglu_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_prepared_bytes": ([i32, i32], sz),
    "swiftspec_prepare_activations": ([vp, i32, i32, i32, vp, vp], ctypes.c_int),
    "swiftspec_w4a16_gemm_prepared": ([ctypes.POINTER(W4), vp, i32, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_w4a16_swiglu_prepared": ([ctypes.POINTER(W4), ctypes.POINTER(W4), vp, i32, vp, i32, vp, sz, vp],
                                        ctypes.c_int),
    "swiftspec_rmsnorm": ([vp, i32, i32, i32, vp, f32, vp, i32, vp], ctypes.c_int),
    "swiftspec_rmsnorm_w4a16_gemm": ([ctypes.POINTER(W4), vp, i32, i32, vp, f32, vp, i32, vp, sz, vp],
                                     ctypes.c_int),
    "swiftspec_rmsnorm_w4a16_swiglu": ([ctypes.POINTER(W4), ctypes.POINTER(W4), vp, i32, i32, vp, f32, vp, i32,
                                       vp, sz, vp], ctypes.c_int),
    "swiftspec_tree_attention": ([vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, i32, i32, i32, i32, vp, f32,
                                  vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_tree_attention_workspace_bytes": ([i32, i32, i32, i32, i32], sz),
    "swiftspec_tree_attention_noalloc": ([vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, i32, i32, i32, i32, vp, f32,
                                          vp, i32, vp, vp], ctypes.c_int),
    "swiftspec_rope_table": ([f64, i32, i32, vp], ctypes.c_int),
    "swiftspec_tree_masks": ([vp, i32, i32, vp, vp, vp, vp], ctypes.c_int),
    "swiftspec_tree_validate": ([vp, i32, vp], ctypes.c_int),
    "swiftspec_kv_commit": ([vp, vp, i32, i64, i32, i32, i32, vp, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_verify_layer": ([ctypes.POINTER(Layer), ctypes.POINTER(Dims), vp, i32, vp, vp, vp, vp, sz, vp],
                               ctypes.c_int),
    "swiftspec_verify_layer_workspace_bytes": ([ctypes.POINTER(Dims), i32], sz),
    "swiftspec_verify_layer_workspace_layout": ([ctypes.POINTER(Dims), i32, ctypes.POINTER(sz)], ctypes.c_int),
    "swiftspec_lm_head": ([vp, i32, i32, vp, f32, vp, i32, vp, vp, sz, vp], ctypes.c_int),
    "swiftspec_lm_head_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_verify_step": ([ctypes.POINTER(Layer), i32, ctypes.POINTER(Dims), vp, i32, vp, vp, vp, vp, vp,
                               i32, vp, vp, sz, vp], ctypes.c_int),
    "swiftspec_verify_step_workspace_bytes": ([ctypes.POINTER(Dims), i32, i32], sz),
    "swiftspec_w4a16_gemm_valu": ([ctypes.POINTER(W4), vp, i32, i32, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_w4a16_gemm_valu_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_mx4_packed_bytes": ([i32, i32, i32], sz),
    "swiftspec_mx4_prepack": ([ctypes.POINTER(MX4), vp, sz, vp], ctypes.c_int),
    "swiftspec_mx4_quantize": ([vp, i64, i32, i64, vp, vp, vp], ctypes.c_int),
    "swiftspec_mx4_dequantize": ([vp, vp, i64, i32, vp, i64, vp], ctypes.c_int),
    "swiftspec_mx4_gemm": ([ctypes.POINTER(MX4), vp, i32, i32, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_mx4_gemm_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_fp8_packed_bytes": ([i32, i32, i32], sz),
    "swiftspec_fp8_prepack": ([ctypes.POINTER(FP8), vp, sz, vp], ctypes.c_int),
    "swiftspec_fp8_quantize": ([vp, i64, i32, i64, i32, vp, vp, vp], ctypes.c_int),
    "swiftspec_fp8_dequantize": ([vp, vp, i64, i32, i32, vp, i64, vp], ctypes.c_int),
    "swiftspec_fp8_gemm": ([ctypes.POINTER(FP8), vp, i32, i32, vp, i32, vp, i32, vp, sz, vp], ctypes.c_int),
    "swiftspec_fp8_gemm_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_moe_route": ([vp, i32, i32, vp, vp, ctypes.POINTER(_Groups), vp, sz, vp], ctypes.c_int),
    "swiftspec_moe_route_scored": ([vp, i32, i32, ctypes.POINTER(_Scoring), vp, vp, ctypes.POINTER(_Groups), vp, sz, vp],
                                   ctypes.c_int),
    "swiftspec_moe_group": ([vp, ctypes.POINTER(_Groups), vp, sz, vp], ctypes.c_int),
    "swiftspec_moe_route_workspace_bytes": ([i32, i32, i32], sz),
    "swiftspec_moe_mx4_swiglu": ([ctypes.POINTER(MX4), ctypes.POINTER(MX4), vp, i32, ctypes.POINTER(_Groups), vp, i32,
                                  vp, sz, vp], ctypes.c_int),
    "swiftspec_moe_mx4_swiglu_workspace_bytes": ([i32, i32, i32, i32, i32], sz),
    "swiftspec_moe_mx4_down": ([ctypes.POINTER(MX4), vp, i32, ctypes.POINTER(_Groups), vp, vp, i32, vp, i32, vp, sz,
                                vp], ctypes.c_int),
    "swiftspec_moe_mx4_down_workspace_bytes": ([i32, i32, i32, i32, i32], sz),
    "swiftspec_moe_fp8_swiglu": ([ctypes.POINTER(FP8), ctypes.POINTER(FP8), vp, i32, ctypes.POINTER(_Groups), vp, i32,
                                  vp, sz, vp], ctypes.c_int),
    "swiftspec_moe_fp8_swiglu_workspace_bytes": ([i32, i32, i32, i32, i32], sz),
    "swiftspec_moe_fp8_down": ([ctypes.POINTER(FP8), vp, i32, ctypes.POINTER(_Groups), vp, vp, i32, vp, i32, vp, sz,
                                vp], ctypes.c_int),
    "swiftspec_moe_fp8_down_workspace_bytes": ([i32, i32, i32, i32, i32], sz),
    "swiftspec_graph_begin": ([vp], ctypes.c_int),
    "swiftspec_graph_end": ([vp, ctypes.POINTER(vp)], ctypes.c_int),
    "swiftspec_graph_launch": ([vp, vp], ctypes.c_int),
    "swiftspec_graph_destroy": ([vp], ctypes.c_int),
}
EXPORTS = tuple(_SIGS)


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"libswiftspec.so is not built ({LIB_PATH}); run __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (args, res) in _SIGS.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def lib():
    return _load()


def _check(status: int, where: str):
    if status != OK:
        raise SwiftSpecError(status, where)


def _ptr(t):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


# ------------------------------------------------------------------ helpers

def workspace(nbytes: int, device="cuda"):
    """A zero-filled device workspace (its header must start at zero)."""
    import torch
    return torch.zeros(int(nbytes), dtype=torch.uint8, device=device)


def make_w4(qweight, scales, zeros, packed=None) -> W4:
    """Describe an int4 matrix held in device tensors qweight [N][K/2] u8,
    scales [N][K/128] fp16, zeros [N][K/128] u8, and optionally its
    kernel-native copy `packed` (see prepack_w4)."""
    N, half_k = qweight.shape
    return W4(qweight.data_ptr(), scales.data_ptr(), zeros.data_ptr(), 2 * half_k, N,
              packed.data_ptr() if packed is not None else None)


def packed_bytes(K: int, N: int) -> int:
    return int(_load().swiftspec_w4_packed_bytes(K, N))


def prepack_w4(W: W4, stream=None):
    """Allocate and fill the kernel-native copy of W; returns the uint8
    device tensor and sets W.packed to it (keep the tensor alive)."""
    import torch
    t = torch.empty(packed_bytes(W.K, W.N), dtype=torch.uint8, device="cuda")
    _check(_load().swiftspec_w4_prepack(ctypes.byref(W), _ptr(t), t.numel(), _stream(stream)), "w4_prepack")
    W.packed = t.data_ptr()
    return t


def prepack_w4_into(W: W4, out, stream=None):
    """Fill the caller's uint8 device tensor `out` (at least
    packed_bytes(K, N) bytes, 16-byte aligned) with the kernel-native copy of
    W and set W.packed to it."""
    _check(_load().swiftspec_w4_prepack(ctypes.byref(W), _ptr(out), out.numel(), _stream(stream)), "w4_prepack")
    W.packed = out.data_ptr()


def rope_table(theta: float, S_max: int, D: int):
    """Host fp32 (cos, sin) table [S_max][D/2][2] built in fp64 by the library."""
    import numpy as np
    out = np.empty((S_max, D // 2, 2), np.float32)
    _check(_load().swiftspec_rope_table(theta, S_max, D, out.ctypes.data), "rope_table")
    return out


def tree_validate(parent):
    import numpy as np
    p = np.ascontiguousarray(parent, dtype=np.int32)
    depth = np.empty(len(p), np.int32)
    st = _load().swiftspec_tree_validate(p.ctypes.data, len(p), depth.ctypes.data)
    return st, depth


def read_device_error(ws, stream=None) -> int:
    out = ctypes.c_uint32(0)
    _check(_load().swiftspec_read_device_error(_ptr(ws), _stream(stream), ctypes.byref(out)),
           "read_device_error")
    return int(out.value)


def clock_sample(out, window_us: int = 20, stream=None):
    """Enqueue the clock sample on `stream` into `out` (an int64 device
    tensor of at least 4 elements): shader-clock and real-time counters
    before and after a window_us wait."""
    assert out.numel() >= 4 and out.element_size() == 8
    _check(_load().swiftspec_clock_sample(_ptr(out), window_us, _stream(stream)), "clock_sample")


def clock_ghz(sample) -> float:
    """Shader clock in GHz from a clock_sample result (host sequence of 4)."""
    c0, r0, c1, r1 = (int(v) for v in sample[:4])
    return (c1 - c0) / max(1, r1 - r0) / 10.0


def workspace_init(ws, stream=None):
    _check(_load().swiftspec_workspace_init(_ptr(ws), ws.numel(), _stream(stream)), "workspace_init")


# ------------------------------------------------------------ operations

def gemm_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(_load().swiftspec_w4a16_gemm_workspace_bytes(M, K, N))


def gemm_valu_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(_load().swiftspec_w4a16_gemm_valu_workspace_bytes(M, K, N))


def w4a16_gemm_valu(W: W4, x, y, ws, residual=None, stream=None):
    """As w4a16_gemm, on the vector ALUs only (comparison variant)."""
    st = _load().swiftspec_w4a16_gemm_valu(ctypes.byref(W), _ptr(x), x.shape[0], x.stride(0), _ptr(y), y.stride(0),
                                           _ptr(residual), residual.stride(0) if residual is not None else 0,
                                           _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "w4a16_gemm_valu")


def swiglu_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(_load().swiftspec_w4a16_swiglu_workspace_bytes(M, K, N))


def w4a16_gemm(W: W4, x, y, ws, residual=None, stream=None):
    M, ldx = x.shape[0], x.stride(0)
    st = _load().swiftspec_w4a16_gemm(ctypes.byref(W), _ptr(x), M, ldx, _ptr(y), y.stride(0),
                                      _ptr(residual), residual.stride(0) if residual is not None else 0,
                                      _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "w4a16_gemm")


def w4a16_swiglu(Wg: W4, Wu: W4, x, y, ws, stream=None):
    st = _load().swiftspec_w4a16_swiglu(ctypes.byref(Wg), ctypes.byref(Wu), _ptr(x), x.shape[0],
                                        x.stride(0), _ptr(y), y.stride(0), _ptr(ws), ws.numel(),
                                        _stream(stream))
    _check(st, "w4a16_swiglu")


def prepared_bytes(M: int, K: int) -> int:
    return int(_load().swiftspec_prepared_bytes(M, K))


def prepare_activations(x, xp, stream=None):
    """x [M][>=K] fp16 -> xp (uint8/int16 device buffer of prepared_bytes(M, K))."""
    M, K = x.shape
    _check(_load().swiftspec_prepare_activations(_ptr(x), M, x.stride(0), K, _ptr(xp), _stream(stream)),
           "prepare_activations")


def w4a16_gemm_prepared(W: W4, xp, M: int, y, ws, residual=None, stream=None):
    st = _load().swiftspec_w4a16_gemm_prepared(ctypes.byref(W), _ptr(xp), M, _ptr(y), y.stride(0),
                                               _ptr(residual), residual.stride(0) if residual is not None else 0,
                                               _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "w4a16_gemm_prepared")


def w4a16_swiglu_prepared(Wg: W4, Wu: W4, xp, M: int, y, ws, stream=None):
    st = _load().swiftspec_w4a16_swiglu_prepared(ctypes.byref(Wg), ctypes.byref(Wu), _ptr(xp), M, _ptr(y),
                                                 y.stride(0), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "w4a16_swiglu_prepared")


def rmsnorm(x, gamma, out, eps=1e-5, stream=None):
    st = _load().swiftspec_rmsnorm(_ptr(x), x.shape[0], x.shape[1], x.stride(0), _ptr(gamma), eps,
                                   _ptr(out), out.stride(0), _stream(stream))
    _check(st, "rmsnorm")


def rmsnorm_w4a16_gemm(W: W4, x, gamma, y, ws, eps=1e-5, stream=None):
    """y = rmsnorm(x, gamma) . W'^T (workspace of gemm_workspace_bytes)."""
    st = _load().swiftspec_rmsnorm_w4a16_gemm(ctypes.byref(W), _ptr(x), x.shape[0], x.stride(0), _ptr(gamma), eps,
                                              _ptr(y), y.stride(0), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "rmsnorm_w4a16_gemm")


def rmsnorm_w4a16_swiglu(Wg: W4, Wu: W4, x, gamma, y, ws, eps=1e-5, stream=None):
    """y = silu(xn . Wg'^T) * (xn . Wu'^T), xn = rmsnorm(x, gamma)
    (workspace of swiglu_workspace_bytes)."""
    st = _load().swiftspec_rmsnorm_w4a16_swiglu(ctypes.byref(Wg), ctypes.byref(Wu), _ptr(x), x.shape[0],
                                                x.stride(0), _ptr(gamma), eps, _ptr(y), y.stride(0), _ptr(ws),
                                                ws.numel(), _stream(stream))
    _check(st, "rmsnorm_w4a16_swiglu")


def tree_attention_workspace_bytes(T, Hq, Hkv, D, S_max) -> int:
    return int(_load().swiftspec_tree_attention_workspace_bytes(T, Hq, Hkv, D, S_max))


def tree_attention(q, k, v, k_cache, v_cache, prefix_len, parent, Hq, Hkv, D, rope, out, ws,
                   softmax_scale=None, stream=None):
    """q [T][>=Hq*D], k/v [T][>=Hkv*D] (row strides are the leading dims),
    caches [Hkv][S_max][D], prefix_len int32[1] and parent int32[T] on device."""
    T = parent.shape[0]
    S_max = k_cache.shape[-2]
    if softmax_scale is None:
        softmax_scale = 1.0 / (D ** 0.5)
    st = _load().swiftspec_tree_attention(_ptr(q), q.stride(0), _ptr(k), _ptr(v), k.stride(0),
                                          _ptr(k_cache), _ptr(v_cache), S_max, _ptr(prefix_len),
                                          _ptr(parent), T, Hq, Hkv, D, _ptr(rope), softmax_scale,
                                          _ptr(out), out.stride(0), _ptr(ws), ws.numel(),
                                          _stream(stream))
    _check(st, "tree_attention")


NOALLOC_SCRATCH_BYTES = 32 << 20


def tree_attention_noalloc(q, k, v, k_cache, v_cache, prefix_len, parent, Hq, Hkv, D, rope, out, error=None,
                           softmax_scale=None, stream=None):
    """tree_attention without a workspace (partials in the library's own
    device array); error: device int32[1] that receives the device error
    bits, or None."""
    T = parent.shape[0]
    S_max = k_cache.shape[-2]
    if softmax_scale is None:
        softmax_scale = 1.0 / (D ** 0.5)
    st = _load().swiftspec_tree_attention_noalloc(_ptr(q), q.stride(0), _ptr(k), _ptr(v), k.stride(0),
                                                  _ptr(k_cache), _ptr(v_cache), S_max, _ptr(prefix_len),
                                                  _ptr(parent), T, Hq, Hkv, D, _ptr(rope), softmax_scale,
                                                  _ptr(out), out.stride(0), _ptr(error), _stream(stream))
    _check(st, "tree_attention_noalloc")


def tree_masks(parents, anc, depth, status, stream=None):
    n, T = parents.shape
    st = _load().swiftspec_tree_masks(_ptr(parents), n, T, _ptr(anc), _ptr(depth), _ptr(status),
                                      _stream(stream))
    _check(st, "tree_masks")


def kv_commit(k_cache, v_cache, prefix_len, parent, accepted, n_layers=1, layer_stride=None,
              advance=False, ws=None, stream=None):
    """Caches [n_layers][Hkv][S_max][D] (or [Hkv][S_max][D]); prefix_len,
    parent and accepted are device int32 tensors."""
    Hkv, S_max, D = k_cache.shape[-3:]
    if layer_stride is None:
        layer_stride = Hkv * S_max * D
    st = _load().swiftspec_kv_commit(_ptr(k_cache), _ptr(v_cache), n_layers, layer_stride, Hkv, S_max,
                                     D, _ptr(prefix_len), _ptr(parent), parent.shape[0], _ptr(accepted),
                                     int(bool(advance)), _ptr(ws), ws.numel() if ws is not None else 0,
                                     _stream(stream))
    _check(st, "kv_commit")


def draft_tree_attention(q, k, v, k_cache, v_cache, prefix_len, cache_parent, leaf_parent, Hq, Hkv, rope, out, ws,
                         softmax_scale=None, stream=None):
    """Draft-model attention with the non-square mask: q [w][>=Hq*D],
    k / v [w][>=Hkv*D] (strided views allowed), caches [Hkv][S_max][D],
    cache_parent [N] (None or empty for N = 0) and leaf_parent [w] device
    int32."""
    Hkv_, S_max, D = k_cache.shape
    w = q.shape[0]
    N = 0 if cache_parent is None else cache_parent.shape[0]
    scale = softmax_scale if softmax_scale is not None else 1.0 / (D ** 0.5)
    st = _load().swiftspec_draft_tree_attention(_ptr(q), q.stride(0), _ptr(k), _ptr(v), k.stride(0), _ptr(k_cache),
                                                _ptr(v_cache), S_max, _ptr(prefix_len),
                                                _ptr(cache_parent) if N else None, N, _ptr(leaf_parent), w, Hq, Hkv,
                                                D, _ptr(rope), scale, _ptr(out), out.stride(0), _ptr(ws), ws.numel(),
                                                _stream(stream))
    _check(st, "draft_tree_attention")


def kv_reorganize(k_cache, v_cache, prefix_len, parent, last, keep, new_parent=None, n_kept=None, n_layers=1,
                  layer_stride=None, advance=False, ws=None, stream=None):
    """Draft-side reorganisation on caches [n_layers][Hkv][S_max][D] (or
    [Hkv][S_max][D]); prefix_len, parent [N], last, keep and the outputs
    new_parent [N], n_kept are device int32 tensors."""
    Hkv, S_max, D = k_cache.shape[-3:]
    if layer_stride is None:
        layer_stride = Hkv * S_max * D
    st = _load().swiftspec_kv_reorganize(_ptr(k_cache), _ptr(v_cache), n_layers, layer_stride, Hkv, S_max, D,
                                         _ptr(prefix_len), _ptr(parent), parent.shape[0], _ptr(last), _ptr(keep),
                                         _ptr(new_parent), _ptr(n_kept), int(bool(advance)), _ptr(ws),
                                         ws.numel() if ws is not None else 0, _stream(stream))
    _check(st, "kv_reorganize")


def greedy_accept_workspace_bytes(T) -> int:
    return int(_load().swiftspec_greedy_accept_workspace_bytes(T))


def greedy_accept(logits, tokens, parent, argmax, accepted, bonus, ws, path_len=None, V=None,
                  stream=None):
    """logits [T][ldl] fp16 (first V columns; default all); tokens, parent
    [T] and the outputs argmax [T], accepted, bonus, path_len [1] are device
    int32 tensors."""
    T, ldl = logits.shape
    st = _load().swiftspec_greedy_accept(_ptr(logits), ldl, T, ldl if V is None else V, _ptr(tokens),
                                         _ptr(parent), _ptr(argmax), _ptr(accepted), _ptr(bonus),
                                         _ptr(path_len), _ptr(ws), ws.numel() if ws is not None else 0,
                                         _stream(stream))
    _check(st, "greedy_accept")


def topk_logprobs_workspace_bytes(n) -> int:
    return int(_load().swiftspec_topk_logprobs_workspace_bytes(n))


def topk_logprobs(logits, tokens, logprobs, ws, V=None, stream=None):
    """logits [n][ldl] fp16 (first V columns; default all) -> the k most
    probable tokens of each row (device int32 tokens [n][k]) and their
    log-softmax values (device float32 logprobs [n][k])."""
    n, ldl = logits.shape
    k = tokens.shape[1]
    st = _load().swiftspec_topk_logprobs(_ptr(logits), ldl, n, ldl if V is None else V, k, _ptr(tokens),
                                         _ptr(logprobs), _ptr(ws), ws.numel() if ws is not None else 0,
                                         _stream(stream))
    _check(st, "topk_logprobs")


class DraftTree:
    """Host-side draft tree (swiftspec_draft_tree_*): host numpy arrays in
    and out, no device work."""

    def __init__(self, capacity: int, root_token: int):
        import numpy as np
        self._np = np
        h = vp()
        _check(_load().swiftspec_draft_tree_create(capacity, root_token, ctypes.byref(h)), "draft_tree_create")
        self._h = h

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.swiftspec_draft_tree_destroy(self._h)
            self._h = None

    def _a(self, n, dtype):
        return self._np.zeros(max(int(n), 1), dtype)

    @staticmethod
    def _p(a):
        return a.ctypes.data if a is not None else None

    def size(self) -> int:
        return int(_load().swiftspec_draft_tree_size(self._h))

    def rows(self) -> int:
        return int(_load().swiftspec_draft_tree_rows(self._h))

    def nodes(self):
        """(token, parent, weight, row, expanded) arrays over all nodes."""
        np = self._np
        n = self.size()
        tok, par, row, exp = (self._a(n, np.int32) for _ in range(4))
        w = self._a(n, np.float64)
        _check(_load().swiftspec_draft_tree_nodes(self._h, self._p(tok), self._p(par), self._p(w), self._p(row),
                                                  self._p(exp)), "draft_tree_nodes")
        return tok[:n], par[:n], w[:n], row[:n], exp[:n]

    def forest(self):
        f = self._a(self.rows(), self._np.int32)
        _check(_load().swiftspec_draft_tree_forest(self._h, self._p(f)), "draft_tree_forest")
        return f[:self.rows()]

    def select_leaves(self, w: int):
        np = self._np
        leaves, prow, n = self._a(w, np.int32), self._a(w, np.int32), np.zeros(1, np.int32)
        _check(_load().swiftspec_draft_tree_select_leaves(self._h, w, self._p(leaves), self._p(prow),
                                                          self._p(n)), "draft_tree_select_leaves")
        return leaves[:n[0]], prow[:n[0]]

    def expand(self, leaves, tokens, logprobs):
        np = self._np
        leaves = np.ascontiguousarray(leaves, np.int32)
        tokens = np.ascontiguousarray(tokens, np.int32).reshape(len(leaves), -1)
        logprobs = np.ascontiguousarray(logprobs, np.float32).reshape(len(leaves), -1)
        _check(_load().swiftspec_draft_tree_expand(self._h, len(leaves), self._p(leaves), tokens.shape[1],
                                                   self._p(tokens), self._p(logprobs)), "draft_tree_expand")

    def select_subgraph(self, bs: int):
        """(nodes, parent positions, tokens) of the bs most probable nodes."""
        np = self._np
        nodes, par, tok, n = self._a(bs, np.int32), self._a(bs, np.int32), self._a(bs, np.int32), np.zeros(1, np.int32)
        _check(_load().swiftspec_draft_tree_select_subgraph(self._h, bs, self._p(nodes), self._p(par), self._p(tok),
                                                            self._p(n)), "draft_tree_select_subgraph")
        m = int(n[0])
        return nodes[:m], par[:m], tok[:m]

    def reroot(self, verified):
        """dict(last, path_rows, keep, pending) as swiftspec_draft_tree_reroot."""
        np = self._np
        ver = np.ascontiguousarray(verified, np.int32)
        out = np.zeros(4, np.int32)
        pend = self._a(len(ver), np.int32)
        _check(_load().swiftspec_draft_tree_reroot(self._h, self._p(ver), len(ver), self._p(out[0:1]),
                                                   self._p(out[1:2]), self._p(out[2:3]), self._p(pend),
                                                   self._p(out[3:4])), "draft_tree_reroot")
        return {"last": int(out[0]), "path_rows": int(out[1]), "keep": int(out[2]),
                "pending": [int(x) for x in pend[:out[3]]]}


# ---- microscaled 4-bit and block-scaled 8-bit matrices, mixture of experts

# a call's own cost on the host counts where the kernels take a few
# microseconds: the checks below keep to a handful of attribute reads
_cuda = None  # (handle of a device's current stream, current device)
_half = None  # torch.float16
_single = None  # torch.float32
_e4m3 = None  # the types of e4m3 codes
_TOP = 2**31 - 1  # the largest number that the library takes for a size


def _size(name, *n):
    """A size query; numbers of more than 32 bits are as far outside as the largest of 32."""
    return int(getattr(_load(), "swiftspec_" + name)(*(max(-1, min(v, _TOP)) for v in n)))


def _rows(t, what, cols, most=_TOP, dtype=None):
    """(rows, row stride) of an fp16 matrix (or of `dtype`) of `cols` contiguous columns: the
    library takes a pointer and a leading dimension (both of them 32-bit numbers
    but in the quantisation), so a tensor that it would read differently is
    refused here."""
    global _half
    if _half is None:
        import torch
        _half = torch.float16
    if t.dim() != 2:
        raise SwiftSpecError(INVALID_ARG, what)
    (M, K), (ld, step) = t.shape, t.stride()
    if K != cols or t.dtype is not (dtype or _half) or (step != 1 and K > 1):
        raise SwiftSpecError(INVALID_ARG, what)
    if M <= 1 and ld <= K:
        ld = K
    if M > most or ld > most or K > _TOP:
        raise SwiftSpecError(UNSUPPORTED, what)
    return M, ld


def _dense(t, what, shape, dtype_bytes, real=None):
    """t, if it is a contiguous tensor of these sizes: floats (`real`), integers
    (real=False) or any bytes."""
    if t is None or t.shape != shape or t.itemsize != dtype_bytes or not t.is_contiguous():
        raise SwiftSpecError(INVALID_ARG, what)
    if real is not None and t.dtype.is_floating_point != real:
        raise SwiftSpecError(INVALID_ARG, what)
    return t


def _run(where, fn, stream, dev, *args):
    """Call fn(*args, stream handle) with device `dev` current, on `stream` (of
    that device) or on the device's current stream."""
    global _cuda
    if _cuda is None:
        import torch
        _cuda = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    if stream is None:
        s = _cuda[0](dev)
    elif getattr(stream, "device_index", dev) == dev:
        s = stream.cuda_stream
    else:
        raise SwiftSpecError(INVALID_ARG, where)
    if _cuda[1]() == dev:
        st = fn(*args, s)
    else:
        import torch
        with torch.cuda.device(dev):
            st = fn(*args, s)
    if st:
        raise SwiftSpecError(st, where)


def _same_device(where, W, t, *others):
    """The GPU that all of a call's tensors (None: not given) and its matrix W
    (None: no matrix) are on."""
    dev = t.get_device()
    for o in others:
        if o is not None and o.get_device() != dev:
            raise SwiftSpecError(INVALID_ARG, where)
    if dev < 0 or (W is not None and W.device not in (None, dev)):
        raise SwiftSpecError(INVALID_ARG, where)
    return dev


def _matrix(kind, where, codes, scales, K, packed):
    """The description of a matrix, or of E of them, whose scales were checked;
    codes [..., N][bytes of a row], `packed` all of its kernel-native copy or None."""
    if max(*codes.shape, K) > _TOP:
        raise SwiftSpecError(UNSUPPORTED, where)
    E, N = codes.shape[0] if codes.dim() == 3 else 1, codes.shape[-2]
    size = mx4_packed_bytes if kind is MX4 else fp8_packed_bytes
    if packed is not None and (not packed.is_contiguous() or packed.numel() * packed.itemsize < size(K, N, E)):
        raise SwiftSpecError(INVALID_ARG, where)
    W = kind(codes.data_ptr(), scales.data_ptr(), K, N, E, packed.data_ptr() if packed is not None else None)
    W.device = _same_device(where, None, codes, scales, packed)
    if packed is None:
        W.unpacked = codes, scales
    return W


def _codes(where, codes):
    if codes.dim() not in (2, 3) or not codes.is_contiguous() or codes.element_size() != 1:
        raise SwiftSpecError(INVALID_ARG, where)


def make_mx4(codes, scales, packed=None) -> MX4:
    """Describe an MXFP4 matrix held in device tensors codes [N][K/2] u8 and
    scales [N][K/32] u8, or E of them (codes [E][N][K/2], scales [E][N][K/32]),
    and optionally its kernel-native copy `packed` (see prepack_mx4), all of it:
    mx4_packed_bytes contiguous bytes.  The matrix keeps codes and scales until
    prepack_mx4 has read them; it does not keep `packed`."""
    _codes("make_mx4", codes)
    _dense(scales, "make_mx4", (*codes.shape[:-1], codes.shape[-1] // 16), 1)
    return _matrix(MX4, "make_mx4", codes, scales, 2 * codes.shape[-1], packed)


def mx4_packed_bytes(K: int, N: int, E: int = 1) -> int:
    return _size("mx4_packed_bytes", K, N, E)


def _let_go(W, dev, stream):
    """Codes and scales that W holds are not needed behind the launch on `stream` that
    made its copy; in a graph every replay reads them, and W keeps them."""
    import torch
    if W.unpacked and W.unpacked[0].is_cuda:
        used = torch.cuda.current_stream(dev) if stream is None else torch.cuda.ExternalStream(stream.cuda_stream, device=dev)
        with torch.cuda.stream(used):
            if torch.cuda.is_current_stream_capturing():
                return
        for source in W.unpacked:
            # held by W's tuple, `source` and the argument alone: its memory goes now, but
            # not to another stream before the launch has read it
            if sys.getrefcount(source) <= 3:
                source.record_stream(used)
    W.unpacked = ()


def _prepack(where, W, size, device, stream):
    import torch
    t = torch.empty(size, dtype=torch.uint8, device=device)
    dev = _same_device(where, W, t)
    _run(where, getattr(_load(), "swiftspec_" + where), stream, dev, ctypes.byref(W), t.data_ptr(), t.numel())
    _let_go(W, dev, stream)
    W.packed = t.data_ptr()
    return t


def prepack_mx4(W: MX4, device="cuda", stream=None):
    """Allocate and fill the kernel-native copy of W on `device` (the GPU that
    holds its codes; another one is refused); returns the uint8 device tensor and
    sets W.packed to it (keep the tensor alive)."""
    return _prepack("mx4_prepack", W, mx4_packed_bytes(W.K, W.N, W.E), device, stream)


def mx4_quantize(x, codes, scales, stream=None):
    """x [M][K] fp16 (rows contiguous) -> codes [M][K/2], scales [M][K/32] u8."""
    K = x.shape[-1]
    M, ld = _rows(x, "mx4_quantize", K, 2**63 - 1)
    _dense(codes, "mx4_quantize", (M, K // 2), 1)
    _dense(scales, "mx4_quantize", (M, K // 32), 1)
    _run("mx4_quantize", _load().swiftspec_mx4_quantize, stream, _same_device("mx4_quantize", None, x, codes, scales), x.data_ptr(), M, K, ld,
         codes.data_ptr(), scales.data_ptr())


def mx4_dequantize(codes, scales, y, stream=None):
    """codes [M][K/2], scales [M][K/32] u8 -> y [M][K] fp16 (rows contiguous)."""
    K = y.shape[-1]
    M, ld = _rows(y, "mx4_dequantize", K, 2**63 - 1)
    _dense(codes, "mx4_dequantize", (M, K // 2), 1)
    _dense(scales, "mx4_dequantize", (M, K // 32), 1)
    _run("mx4_dequantize", _load().swiftspec_mx4_dequantize, stream, _same_device("mx4_dequantize", None, codes, scales, y), codes.data_ptr(),
         scales.data_ptr(), M, K, y.data_ptr(), ld)


def mx4_gemm_workspace_bytes(M: int, K: int, N: int) -> int:
    return _size("mx4_gemm_workspace_bytes", M, K, N)


def _gemm(where, fn, W, x, y, ws, residual, stream):
    M, ldx = _rows(x, where, W.K)
    m, ldy = _rows(y, where, W.N)
    r, ldr, res = M, 0, None
    if residual is not None:
        r, ldr = _rows(residual, where, W.N)
        res = residual.data_ptr()
    if m != M or r != M:
        raise SwiftSpecError(INVALID_ARG, where)
    _run(where, fn, stream, _same_device(where, W, x, y, ws, residual), ctypes.byref(W), x.data_ptr(), M, ldx, y.data_ptr(), ldy, res, ldr,
         ws.data_ptr(), ws.numel() * ws.element_size())


def mx4_gemm(W: MX4, x, y, ws, residual=None, stream=None):
    """y = fp16(Q(x) . W'^T + residual): x [M][K], y and residual [M][N] fp16."""
    _gemm("mx4_gemm", _load().swiftspec_mx4_gemm, W, x, y, ws, residual, stream)


def _e4m3_codes(where, codes):
    """Refuse codes of a type that stands for other values than e4m3."""
    global _e4m3
    if _e4m3 is None:
        import torch
        _e4m3 = frozenset((torch.uint8, torch.int8, torch.float8_e4m3fn))
    if codes.dtype not in _e4m3:
        raise SwiftSpecError(INVALID_ARG, where)


def make_fp8(codes, scales, packed=None) -> FP8:
    """Describe an 8-bit matrix held in device tensors codes [N][K] (e4m3: bytes,
    signed or not, or torch.float8_e4m3fn) and scales [ceil(N/128)][ceil(K/128)]
    float32, or E of them (codes [E][N][K], scales [E][...][...]), and optionally its
    kernel-native copy `packed` (see prepack_fp8), all of it: fp8_packed_bytes
    contiguous bytes.  The matrix keeps codes and scales until prepack_fp8 has read
    them; it does not keep `packed`."""
    _codes("make_fp8", codes)
    _e4m3_codes("make_fp8", codes)
    _dense(scales, "make_fp8", (*codes.shape[:-2], -(-codes.shape[-2] // 128), -(-codes.shape[-1] // 128)), 4, real=True)
    return _matrix(FP8, "make_fp8", codes, scales, codes.shape[-1], packed)


def fp8_packed_bytes(K: int, N: int, E: int = 1) -> int:
    return _size("fp8_packed_bytes", K, N, E)


def prepack_fp8(W: FP8, device="cuda", stream=None):
    """Allocate and fill the kernel-native copy of W, as prepack_mx4."""
    return _prepack("fp8_prepack", W, fp8_packed_bytes(W.K, W.N, W.E), device, stream)


def _fp8_convert(where, values, codes, scales, rows, stream):
    K = values.shape[-1]
    M, ld = _rows(values, where, K, 2**63 - 1)
    if rows not in (1, 128):
        raise SwiftSpecError(INVALID_ARG, where)
    _dense(codes, where, (M, K), 1)
    _e4m3_codes(where, codes)
    _dense(scales, where, (-(-M // rows), -(-K // 128)), 4, real=True)
    return M, K, ld, _same_device(where, None, values, codes, scales)


def fp8_quantize(x, codes, scales, rows=1, stream=None):
    """x [M][K] fp16 (rows contiguous) -> codes [M][K] (e4m3, as make_fp8), scales
    [ceil(M/rows)][ceil(K/128)] float32 of blocks of `rows` (1 or 128) rows and 128
    columns."""
    M, K, ld, dev = _fp8_convert("fp8_quantize", x, codes, scales, rows, stream)
    _run("fp8_quantize", _load().swiftspec_fp8_quantize, stream, dev, x.data_ptr(), M, K, ld, rows, codes.data_ptr(), scales.data_ptr())


def fp8_dequantize(codes, scales, y, rows=1, stream=None):
    """codes [M][K], scales [ceil(M/rows)][ceil(K/128)] -> y [M][K] fp16 (rows contiguous)."""
    M, K, ld, dev = _fp8_convert("fp8_dequantize", y, codes, scales, rows, stream)
    _run("fp8_dequantize", _load().swiftspec_fp8_dequantize, stream, dev, codes.data_ptr(), scales.data_ptr(), M, K, rows, y.data_ptr(), ld)


def fp8_gemm_workspace_bytes(M: int, K: int, N: int) -> int:
    return _size("fp8_gemm_workspace_bytes", M, K, N)


def fp8_gemm(W: FP8, x, y, ws, residual=None, stream=None):
    """y = fp16(Q(x) . W'^T + residual): x [M][K], y and residual [M][N] fp16."""
    _gemm("fp8_gemm", _load().swiftspec_fp8_gemm, W, x, y, ws, residual, stream)


class MoeGroups:
    """The groups of a mixture's (token, slot) pairs by expert: device int32
    tensors offsets [E + 1], rows [T k] and pos [T k] (allocated if not given),
    written by moe_route or moe_group and read by the experts' products."""

    def __init__(self, T: int, k: int, E: int, offsets=None, rows=None, pos=None, device="cuda"):
        import torch
        if max(T, k, E) > _TOP:
            raise SwiftSpecError(UNSUPPORTED, "MoeGroups")
        new = lambda n: torch.empty(n, dtype=torch.int32, device=device)  # noqa: E731
        self.T, self.k, self.E = T, k, E
        self.offsets = _dense(new(E + 1) if offsets is None else offsets, "MoeGroups", (E + 1,), 4, real=False)
        self.rows = _dense(new(T * k) if rows is None else rows, "MoeGroups", (T * k,), 4, real=False)
        self.pos = _dense(new(T * k) if pos is None else pos, "MoeGroups", (T * k,), 4, real=False)
        _same_device("MoeGroups", None, self.offsets, self.rows, self.pos)
        self._c = _Groups(T, k, E, self.offsets.data_ptr(), self.rows.data_ptr() or None, self.pos.data_ptr() or None)

    def _ref(self):
        return ctypes.byref(self._c)

    def _tensors(self):
        return self.offsets, self.rows, self.pos


def moe_route_workspace_bytes(T: int, E: int, k: int) -> int:
    return _size("moe_route_workspace_bytes", T, E, k)


def moe_route(logits, experts, weights, groups: MoeGroups, ws, renormalize=True, stream=None):
    """logits [T][E] fp16 -> experts [T][k] int32 and weights [T][k] float32 of
    the k largest scores of each token, and the groups."""
    T, ldl = _rows(logits, "moe_route", groups.E)
    if T != groups.T:
        raise SwiftSpecError(INVALID_ARG, "moe_route")
    _dense(experts, "moe_route", (T, groups.k), 4, real=False)
    _dense(weights, "moe_route", (T, groups.k), 4, real=True)
    _run("moe_route", _load().swiftspec_moe_route, stream, _same_device("moe_route", None, groups.offsets, logits, experts, weights, ws),
         logits.data_ptr(), ldl, int(bool(renormalize)), experts.data_ptr(), weights.data_ptr(), groups._ref(),
         ws.data_ptr(), ws.numel() * ws.element_size())


class MoeScoring:
    """How moe_route_scored makes scores and compares experts: `score` "softmax" or
    "sigmoid"; `bias` [E] float32 (device) added before they are compared, not to the
    weights; of `groups` groups of consecutive experts only the `top_groups` with the
    largest sum of `group_best` (1 or 2) largest compete; weights divided by their sum
    (`renormalize`) and multiplied by `scale`."""

    def __init__(self, score="softmax", bias=None, groups: int = 1, top_groups: int = 1, group_best: int = 1, renormalize=True,
                 scale: float = 1.0):
        if score not in ("softmax", "sigmoid"):
            raise SwiftSpecError(INVALID_ARG, "MoeScoring")
        if max(groups, top_groups, group_best) > _TOP or min(groups, top_groups, group_best) < 1:
            raise SwiftSpecError(INVALID_ARG, "MoeScoring")
        if bias is not None:
            _dense(bias, "MoeScoring", (bias.numel(),), 4, real=True)
            _same_device("MoeScoring", None, bias)
        self.bias = bias
        self._c = _Scoring(("softmax", "sigmoid").index(score), groups, top_groups, group_best, int(bool(renormalize)), scale,
                           bias.data_ptr() if bias is not None else None)


def moe_route_scored(logits, scoring: MoeScoring, experts, weights, groups: MoeGroups, ws, stream=None):
    """logits [T][E] fp16 or float32 (rows contiguous) -> experts [T][k] int32 and
    weights [T][k] float32 of the k experts that `scoring` puts first, and the groups;
    the workspace is that of moe_route."""
    global _single
    if _single is None:
        import torch
        _single = torch.float32
    wide = logits.dtype is _single
    T, ldl = _rows(logits, "moe_route_scored", groups.E, dtype=_single if wide else None)
    if T != groups.T or (scoring.bias is not None and scoring.bias.numel() != groups.E):
        raise SwiftSpecError(INVALID_ARG, "moe_route_scored")
    _dense(experts, "moe_route_scored", (T, groups.k), 4, real=False)
    _dense(weights, "moe_route_scored", (T, groups.k), 4, real=True)
    _run("moe_route_scored", _load().swiftspec_moe_route_scored, stream,
         _same_device("moe_route_scored", None, groups.offsets, logits, scoring.bias, experts, weights, ws), logits.data_ptr(),
         32 if wide else 16, ldl, ctypes.byref(scoring._c), experts.data_ptr(), weights.data_ptr(), groups._ref(), ws.data_ptr(),
         ws.numel() * ws.element_size())


def moe_group(experts, groups: MoeGroups, ws, stream=None):
    """The groups of given experts [T][k] int32 (outside [0, E): none)."""
    _dense(experts, "moe_group", (groups.T, groups.k), 4, real=False)
    _run("moe_group", _load().swiftspec_moe_group, stream, _same_device("moe_group", None, groups.offsets, experts, ws), experts.data_ptr(),
         groups._ref(), ws.data_ptr(), ws.numel() * ws.element_size())


def moe_mx4_swiglu_workspace_bytes(T: int, k: int, E: int, K: int, N: int) -> int:
    return _size("moe_mx4_swiglu_workspace_bytes", T, k, E, K, N)


def _swiglu(where, fn, Wg, Wu, x, groups, h, ws, stream):
    T, ldx = _rows(x, where, Wg.K)
    P, ldh = _rows(h, where, Wg.N)
    if T != groups.T or P != groups.T * groups.k or Wu.device not in (None, Wg.device):
        raise SwiftSpecError(INVALID_ARG, where)
    _run(where, fn, stream, _same_device(where, Wg, groups.offsets, x, h, ws), ctypes.byref(Wg), ctypes.byref(Wu), x.data_ptr(),
         ldx, groups._ref(), h.data_ptr(), ldh, ws.data_ptr(), ws.numel() * ws.element_size())


def _down(where, fn, Wd, h, groups, weights, y, ws, residual, stream):
    P, ldh = _rows(h, where, Wd.K)
    T, ldy = _rows(y, where, Wd.N)
    r, ldr, res = T, 0, None
    if residual is not None:
        r, ldr = _rows(residual, where, Wd.N)
        res = residual.data_ptr()
    if T != groups.T or r != T or P != T * groups.k:
        raise SwiftSpecError(INVALID_ARG, where)
    _dense(weights, where, (T, groups.k), 4, real=True)
    _run(where, fn, stream, _same_device(where, Wd, groups.offsets, h, weights, y, ws, residual), ctypes.byref(Wd), h.data_ptr(),
         ldh, groups._ref(), weights.data_ptr(), y.data_ptr(), ldy, res, ldr, ws.data_ptr(), ws.numel() * ws.element_size())


def moe_mx4_swiglu(Wg: MX4, Wu: MX4, x, groups: MoeGroups, h, ws, stream=None):
    """x [T][K] fp16 -> h [T k][N] fp16, a row for each place of the groups."""
    _swiglu("moe_mx4_swiglu", _load().swiftspec_moe_mx4_swiglu, Wg, Wu, x, groups, h, ws, stream)


def moe_mx4_down_workspace_bytes(T: int, k: int, E: int, K: int, N: int) -> int:
    return _size("moe_mx4_down_workspace_bytes", T, k, E, K, N)


def moe_mx4_down(Wd: MX4, h, groups: MoeGroups, weights, y, ws, residual=None, stream=None):
    """h [T k][K] fp16 (as moe_mx4_swiglu wrote it), weights [T][k] float32 ->
    y [T][N] fp16, the weighted sum of each token's experts plus residual."""
    _down("moe_mx4_down", _load().swiftspec_moe_mx4_down, Wd, h, groups, weights, y, ws, residual, stream)


def moe_fp8_swiglu_workspace_bytes(T: int, k: int, E: int, K: int, N: int) -> int:
    return _size("moe_fp8_swiglu_workspace_bytes", T, k, E, K, N)


def moe_fp8_swiglu(Wg: FP8, Wu: FP8, x, groups: MoeGroups, h, ws, stream=None):
    """moe_mx4_swiglu with 8-bit matrices."""
    _swiglu("moe_fp8_swiglu", _load().swiftspec_moe_fp8_swiglu, Wg, Wu, x, groups, h, ws, stream)


def moe_fp8_down_workspace_bytes(T: int, k: int, E: int, K: int, N: int) -> int:
    return _size("moe_fp8_down_workspace_bytes", T, k, E, K, N)


def moe_fp8_down(Wd: FP8, h, groups: MoeGroups, weights, y, ws, residual=None, stream=None):
    """moe_mx4_down with 8-bit matrices."""
    _down("moe_fp8_down", _load().swiftspec_moe_fp8_down, Wd, h, groups, weights, y, ws, residual, stream)


def make_dims(H, Hq, Hkv, D, F, S_max, eps=1e-5, rope_theta=500000.0) -> Dims:
    return Dims(H, Hq, Hkv, D, F, S_max, eps, rope_theta)


def make_layer(attn_norm, mlp_norm, wqkv: W4, wo: W4, wgate: W4, wup: W4, wdown: W4, k_cache,
               v_cache) -> Layer:
    return Layer(attn_norm.data_ptr(), mlp_norm.data_ptr(), wqkv, wo, wgate, wup, wdown,
                 k_cache.data_ptr(), v_cache.data_ptr())


def verify_layer_workspace_bytes(dims: Dims, T: int) -> int:
    return int(_load().swiftspec_verify_layer_workspace_bytes(ctypes.byref(dims), T))


def verify_layer_intermediates(dims: Dims, T: int, ws):
    """Views (int16 bits) of the layer intermediates qkv, o, h, m held in a
    verify_layer workspace."""
    offs = (sz * 4)()
    _check(_load().swiftspec_verify_layer_workspace_layout(ctypes.byref(dims), T, offs),
           "verify_layer_workspace_layout")
    import torch
    n_qkv = (dims.Hq + 2 * dims.Hkv) * dims.D
    cols = [n_qkv, dims.Hq * dims.D, dims.H, dims.F]
    names = ["qkv", "o", "h", "m"]
    out = {}
    for name, off, c in zip(names, offs, cols):
        out[name] = ws[off:off + T * c * 2].view(torch.int16).view(T, c)
    return out


def verify_layer(layer: Layer, dims: Dims, hidden, prefix_len, parent, rope, ws, stream=None):
    st = _load().swiftspec_verify_layer(ctypes.byref(layer), ctypes.byref(dims), _ptr(hidden),
                                        hidden.shape[0], _ptr(prefix_len), _ptr(parent), _ptr(rope),
                                        _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "verify_layer")


def lm_head_workspace_bytes(M, H, V) -> int:
    return int(_load().swiftspec_lm_head_workspace_bytes(M, H, V))


def lm_head(h, gamma, W, logits, ws, eps=1e-5, stream=None):
    M, H = h.shape
    V = W.shape[0]
    st = _load().swiftspec_lm_head(_ptr(h), M, H, _ptr(gamma), eps, _ptr(W), V, _ptr(logits), _ptr(ws),
                                   ws.numel(), _stream(stream))
    _check(st, "lm_head")


def verify_step_workspace_bytes(dims: Dims, T: int, V: int) -> int:
    return int(_load().swiftspec_verify_step_workspace_bytes(ctypes.byref(dims), T, V))


def make_layers(layers):
    """A contiguous ctypes array of Layer descriptors for verify_step."""
    arr = (Layer * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = l
    return arr


def verify_step(layers, dims: Dims, hidden, prefix_len, parent, rope, ws, final_norm=None, lm_head_w=None,
                logits=None, stream=None):
    """All decoder layers in order, then (if lm_head_w is given) the final
    RMSNorm and LM head into logits.  `layers` is a make_layers() array."""
    V = 0 if lm_head_w is None else lm_head_w.shape[0]
    st = _load().swiftspec_verify_step(layers, len(layers), ctypes.byref(dims), _ptr(hidden), hidden.shape[0],
                                       _ptr(prefix_len), _ptr(parent), _ptr(rope), _ptr(final_norm),
                                       _ptr(lm_head_w), V, _ptr(logits), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "verify_step")


class Graph:
    """A HIP graph captured from the library calls issued on `stream`
    between begin() and end()."""

    def __init__(self):
        self._g = ctypes.c_void_p(None)

    def begin(self, stream=None):
        _check(_load().swiftspec_graph_begin(_stream(stream)), "graph_begin")

    def end(self, stream=None):
        _check(_load().swiftspec_graph_end(_stream(stream), ctypes.byref(self._g)), "graph_end")

    def launch(self, stream=None):
        _check(_load().swiftspec_graph_launch(self._g, _stream(stream)), "graph_launch")

    def __del__(self):
        if self._g and self._g.value and _lib is not None:
            _lib.swiftspec_graph_destroy(self._g)
            self._g = ctypes.c_void_p(None)

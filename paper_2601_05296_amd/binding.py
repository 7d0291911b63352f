"""ctypes binding of libmoeblaze.so: one Python function per C entry point,
same names, argument marshalling only.

Tensors are torch tensors on the GPU (PyTorch supplies device memory and
streams); every computation runs in the library's HIP kernels. If the library
is not built, or no GPU is present when a call is made, the call raises: there
is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from array import array

import torch

from .build import LIB

MOE_OK = 0
MOE_ERR_INVALID_ARG = -1
MOE_ERR_UNSUPPORTED = -2
MOE_ERR_WORKSPACE = -3
MOE_ERR_HIP = -4

MOE_BF16 = 0
MOE_F32 = 1
MOE_RENORM = 2
MOE_ACCUMULATE = 4
MOE_ACT_SILU = 8
MOE_ACT_RELU = 16
MOE_H_ON_LOAD = 32
MOE_ACCUMULATE_DW = 64
MOE_ATOMIC_COMBINE = 128
MOE_NORM_POST = 256
MOE_NORM_PRE = 512
MOE_GATE_CHANNEL = 1024
MOE_GATE_TOKEN = 2048
MOE_TRANSPOSED = 4096
MOE_GATED = 8192
ACT_FLAG = {"swiglu": 0, "silu": MOE_ACT_SILU, "relu": MOE_ACT_RELU}

# Every symbol declared in include/moeblaze.h.
EXPORTS = ("moe_strerror", "moe_last_error", "moe_route", "moe_build_index_workspace_size",
           "moe_build_index", "moe_build_index_noalloc", "moe_ffn_fwd_workspace_size", "moe_ffn_fwd", "moe_combine", "moe_ffn_bwd_workspace_size",
           "moe_ffn_bwd", "moe_ffn_recompute", "moe_ffn_fwd_combine_workspace_size",
           "moe_ffn_fwd_combine",
           "moe_ffn_bwd_combine_workspace_size", "moe_ffn_bwd_combine",
           "moe_route_bwd_workspace_size", "moe_route_bwd", "moe_norm_fwd",
           "moe_norm_bwd_workspace_size", "moe_norm_bwd", "moe_grad_norm_workspace_size",
           "moe_grad_norm", "moe_grad_clip", "moe_mx_quantize", "moe_mx_dequantize",
           "moe_mx_gemm", "moe_probe_enable",
           "moe_probe_disable", "moe_probe_count", "moe_probe_dropped", "moe_probe_get")


class MoEError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__("%s: %s" % (_status_name(status), detail))
        self.status = status


_lib = None


def _status_name(s: int) -> str:
    return {0: "MOE_OK", -1: "MOE_ERR_INVALID_ARG", -2: "MOE_ERR_UNSUPPORTED",
            -3: "MOE_ERR_WORKSPACE", -4: "MOE_ERR_HIP"}.get(s, "status %d" % s)


def load_library(path: str = LIB):
    """Load libmoeblaze.so and declare the C signatures. Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError("libmoeblaze.so is not built (%s); run "
                          "`python -m paper_2601_05296_amd.build`" % path)
    lib = ctypes.CDLL(path)
    P, I64, I, U, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint, ctypes.c_size_t
    F = ctypes.c_float
    sig = {
        "moe_strerror": (ctypes.c_char_p, [I]),
        "moe_last_error": (ctypes.c_char_p, []),
        "moe_route": (I, [P, P, P, I64, I, I, I, U, P, P, P, P]),
        "moe_build_index_workspace_size": (SZ, [I64, I, I]),
        "moe_build_index": (I, [P, I64, I, I, P, P, P, P, P, P, SZ, P]),
        "moe_build_index_noalloc": (I, [P, I64, I, I, P, P, P, P, P, P]),
        "moe_ffn_fwd_workspace_size": (SZ, [I64, I, I, I, I, U]),
        "moe_ffn_fwd": (I, [P, P, P, P, P, P, I64, I, I, I, I, U, P, P, P, P, SZ, P]),
        "moe_combine": (I, [P, P, P, I64, I, I, U, P, P]),
        "moe_ffn_bwd_workspace_size": (SZ, [I64, I, I, I, I, U]),
        "moe_ffn_bwd": (I, [P] * 11 + [I64, I, I, I, I, U] + [P] * 6 + [SZ, P]),
        "moe_ffn_recompute": (I, [P] * 5 + [I64, I, I, I, I, U, P, P, P]),
        "moe_ffn_fwd_combine_workspace_size": (SZ, [I64, I, I, I, I, U]),
        "moe_ffn_fwd_combine": (I, [P] * 8 + [I64, I, I, I, I, U] + [P] * 4 + [SZ, P]),
        "moe_ffn_bwd_combine_workspace_size": (SZ, [I64, I, I, I, I, U]),
        "moe_ffn_bwd_combine": (I, [P] * 12 + [I64, I, I, I, I, U] + [P] * 6 + [SZ, P]),
        "moe_route_bwd_workspace_size": (SZ, [I64, I, I, I, U]),
        "moe_route_bwd": (I, [P] * 6 + [I64, I, I, I, U, P, P, P, SZ, P]),
        "moe_norm_fwd": (I, [P] * 5 + [F, F, I64, I, U] + [P] * 5),
        "moe_norm_bwd_workspace_size": (SZ, [I64, I, U]),
        "moe_norm_bwd": (I, [P] * 9 + [F, I64, I, U] + [P] * 6 + [SZ, P]),
        "moe_grad_norm_workspace_size": (SZ, [I]),
        "moe_grad_norm": (I, [P, P, P, I, P, P, P, SZ, P]),
        "moe_grad_clip": (I, [P, P, P, P, I, P, ctypes.c_double, P]),
        "moe_mx_quantize": (I, [P, I64, I64, I, U, P, P, P]),
        "moe_mx_dequantize": (I, [P, P, I64, I, U, P, P]),
        "moe_mx_gemm": (I, [P] * 8 + [I64, I64, I, I, I, U, P, P]),
        "moe_probe_enable": (I, [I]),
        "moe_probe_disable": (None, []),
        "moe_probe_count": (I, []),
        "moe_probe_dropped": (I, []),
        "moe_probe_get": (I, [I, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _ptr(t):
    if t is None or t.__class__ is int:
        return t
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _elt(flags: int):
    """Element type of the activation and weight tensors under `flags`."""
    return torch.float32 if flags & MOE_F32 else torch.bfloat16


def _gated(flags: int) -> bool:
    return not flags & (MOE_ACT_SILU | MOE_ACT_RELU)


def _need(t, n: int, name: str, dtype=None):
    """Check, before the library sees a bare pointer, that tensor `t` holds at
    least `n` elements of `dtype` (None or a raw address: not checked here)."""
    if t is None or isinstance(t, int):
        return
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s: dtype %s, expected %s" % (name, t.dtype, dtype))
    if t.numel() < n:
        raise ValueError("%s: %d elements, at least %d needed" % (name, t.numel(), n))


def _need_bytes(t, nbytes: int, name: str = "workspace"):
    if t is None or isinstance(t, int):
        return
    if t.numel() * t.element_size() < nbytes:
        raise ValueError("%s: %d bytes, workspace_bytes says %d" %
                         (name, t.numel() * t.element_size(), nbytes))


def _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, w2, offsets, eti):
    el, S = _elt(flags), T * k
    _need(x, T * d, "x", el)
    _need(w1, E * d * f, "w1", el)
    if _gated(flags):
        _need(w3, E * d * f, "w3", el)
    if w2 is not None:
        _need(w2, E * f * d, "w2", el)
    _need(offsets, E + 1, "offsets", torch.int32)
    _need(eti, S, "expert_token_indices", torch.int32)


def _first_outputs(flags, T, f, k, A, B):
    _need(A, T * k * f, "A", _elt(flags))
    if _gated(flags):
        _need(B, T * k * f, "B", _elt(flags))


def _ffn_grads(flags, T, d, f, E, k, dy, gates, slot_src, dw1, dw3, dw2, d_gates):
    f32 = torch.float32
    _need(dy, T * d, "dy", _elt(flags))
    _need(gates, T * k, "gates", f32)
    _need(slot_src, T * k, "slot_src", torch.int32)
    _need(dw1, E * d * f, "dw1", f32)
    if _gated(flags):
        _need(dw3, E * d * f, "dw3", f32)
    _need(dw2, E * f * d, "dw2", f32)
    _need(d_gates, T * k, "d_gates", f32)


# torch's current stream as a raw handle. The handle alone, where torch offers it,
# costs a tenth of building a torch.cuda.Stream around it (0.2 against 2.3 us).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _check(status: int):
    if status != MOE_OK:
        raise MoEError(status, load_library().moe_last_error().decode())


def dtype_flag(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    if t.dtype == torch.float32:
        return MOE_F32
    raise ValueError("unsupported dtype %s" % t.dtype)


def moe_route(x, w_gate, bias, T, d, E, k, flags, topk_ids, gates, logits, stream=None):
    _need(x, T * d, "x", _elt(flags))
    _need(w_gate, E * d, "w_gate", _elt(flags))
    _need(bias, E, "bias", torch.float32)
    _need(topk_ids, T * k, "topk_ids", torch.int32)
    _need(gates, T * k, "gates", torch.float32)
    _need(logits, T * E, "logits", torch.float32)
    _check(load_library().moe_route(_ptr(x), _ptr(w_gate), _ptr(bias), T, d, E, k, flags,
                                    _ptr(topk_ids), _ptr(gates), _ptr(logits), _stream(stream)))


# The workspace queries are functions of the sizes alone: their answers are kept
# (a ctypes call takes about 1 us).
@functools.lru_cache(maxsize=256, typed=True)
def moe_build_index_workspace_size(T, E, k) -> int:
    return load_library().moe_build_index_workspace_size(T, E, k)


def moe_build_index(topk_ids, T, E, k, counts, offsets, expert_token_indices, token_index_map,
                    slot_src, workspace, workspace_bytes, stream=None):
    i32 = torch.int32
    _need(topk_ids, T * k, "topk_ids", i32)
    _need(counts, E, "counts", i32)
    _need(offsets, E + 1, "offsets", i32)
    _need(expert_token_indices, T * k, "expert_token_indices", i32)
    _need(token_index_map, T * k, "token_index_map", i32)
    _need(slot_src, T * k, "slot_src", i32)
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_build_index(_ptr(topk_ids), T, E, k, _ptr(counts), _ptr(offsets),
                                          _ptr(expert_token_indices), _ptr(token_index_map),
                                          _ptr(slot_src), _ptr(workspace), workspace_bytes,
                                          _stream(stream)))


def moe_build_index_noalloc(topk_ids, T, E, k, counts, offsets, expert_token_indices,
                            token_index_map, slot_src, stream=None):
    i32 = torch.int32
    _need(topk_ids, T * k, "topk_ids", i32)
    _need(counts, E, "counts", i32)
    _need(offsets, E + 1, "offsets", i32)
    _need(expert_token_indices, T * k, "expert_token_indices", i32)
    _need(token_index_map, T * k, "token_index_map", i32)
    _need(slot_src, T * k, "slot_src", i32)
    _check(load_library().moe_build_index_noalloc(_ptr(topk_ids), T, E, k, _ptr(counts),
                                                  _ptr(offsets), _ptr(expert_token_indices),
                                                  _ptr(token_index_map), _ptr(slot_src),
                                                  _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_ffn_fwd_workspace_size(T, d, f, E, k, flags) -> int:
    return load_library().moe_ffn_fwd_workspace_size(T, d, f, E, k, flags)


def moe_ffn_fwd(x, w1, w3, w2, offsets, expert_token_indices, T, d, f, E, k, flags, A, B, O,
                workspace, workspace_bytes, stream=None):
    _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, w2, offsets, expert_token_indices)
    _first_outputs(flags, T, f, k, A, B)
    _need(O, T * k * d, "O", _elt(flags))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_ffn_fwd(_ptr(x), _ptr(w1), _ptr(w3), _ptr(w2), _ptr(offsets),
                                      _ptr(expert_token_indices), T, d, f, E, k, flags, _ptr(A),
                                      _ptr(B), _ptr(O), _ptr(workspace), workspace_bytes,
                                      _stream(stream)))


def moe_ffn_recompute(x, w1, w3, offsets, expert_token_indices, T, d, f, E, k, flags, A, B,
                      stream=None):
    _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, None, offsets, expert_token_indices)
    _first_outputs(flags, T, f, k, A, B)
    _check(load_library().moe_ffn_recompute(_ptr(x), _ptr(w1), _ptr(w3), _ptr(offsets),
                                            _ptr(expert_token_indices), T, d, f, E, k, flags,
                                            _ptr(A), _ptr(B), _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_ffn_fwd_combine_workspace_size(T, d, f, E, k, flags) -> int:
    return load_library().moe_ffn_fwd_combine_workspace_size(T, d, f, E, k, flags)


def moe_ffn_fwd_combine(x, w1, w3, w2, offsets, expert_token_indices, gates, token_index_map,
                        T, d, f, E, k, flags, A, B, y, workspace, workspace_bytes, stream=None):
    _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, w2, offsets, expert_token_indices)
    _first_outputs(flags, T, f, k, A, B)
    _need(gates, T * k, "gates", torch.float32)
    _need(token_index_map, T * k, "token_index_map", torch.int32)
    _need(y, T * d, "y", _elt(flags))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_ffn_fwd_combine(
        _ptr(x), _ptr(w1), _ptr(w3), _ptr(w2), _ptr(offsets), _ptr(expert_token_indices),
        _ptr(gates), _ptr(token_index_map), T, d, f, E, k, flags, _ptr(A), _ptr(B), _ptr(y),
        _ptr(workspace), workspace_bytes, _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_ffn_bwd_combine_workspace_size(T, d, f, E, k, flags) -> int:
    return load_library().moe_ffn_bwd_combine_workspace_size(T, d, f, E, k, flags)


def moe_ffn_bwd_combine(dy, x, w1, w3, w2, gates, offsets, expert_token_indices, slot_src,
                        token_index_map, A, B, T, d, f, E, k, flags, dw1, dw3, dw2, d_gates, dx,
                        workspace, workspace_bytes, stream=None):
    _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, w2, offsets, expert_token_indices)
    _first_outputs(flags, T, f, k, A, B)
    _ffn_grads(flags, T, d, f, E, k, dy, gates, slot_src, dw1, dw3, dw2, d_gates)
    _need(token_index_map, T * k, "token_index_map", torch.int32)
    _need(dx, T * d, "dx", _elt(flags))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_ffn_bwd_combine(
        _ptr(dy), _ptr(x), _ptr(w1), _ptr(w3), _ptr(w2), _ptr(gates), _ptr(offsets),
        _ptr(expert_token_indices), _ptr(slot_src), _ptr(token_index_map), _ptr(A), _ptr(B), T, d,
        f, E, k, flags, _ptr(dw1), _ptr(dw3), _ptr(dw2), _ptr(d_gates), _ptr(dx), _ptr(workspace),
        workspace_bytes, _stream(stream)))


def moe_combine(src, weights, token_index_map, T, d, k, flags, out, stream=None):
    _need(src, T * k * d, "src", _elt(flags))
    _need(weights, T * k, "weights", torch.float32)
    _need(token_index_map, T * k, "token_index_map", torch.int32)
    _need(out, T * d, "out", _elt(flags))
    _check(load_library().moe_combine(_ptr(src), _ptr(weights), _ptr(token_index_map), T, d, k,
                                      flags, _ptr(out), _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_ffn_bwd_workspace_size(T, d, f, E, k, flags) -> int:
    return load_library().moe_ffn_bwd_workspace_size(T, d, f, E, k, flags)


def moe_ffn_bwd(dy, x, w1, w3, w2, gates, offsets, expert_token_indices, slot_src, A, B, T, d,
                f, E, k, flags, dw1, dw3, dw2, d_gates, dX_slot, workspace, workspace_bytes,
                stream=None):
    _ffn_inputs(flags, T, d, f, E, k, x, w1, w3, w2, offsets, expert_token_indices)
    _first_outputs(flags, T, f, k, A, B)
    _ffn_grads(flags, T, d, f, E, k, dy, gates, slot_src, dw1, dw3, dw2, d_gates)
    _need(dX_slot, T * k * d, "dX_slot", _elt(flags))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_ffn_bwd(_ptr(dy), _ptr(x), _ptr(w1), _ptr(w3), _ptr(w2),
                                      _ptr(gates), _ptr(offsets), _ptr(expert_token_indices),
                                      _ptr(slot_src), _ptr(A), _ptr(B), T, d, f, E, k, flags,
                                      _ptr(dw1), _ptr(dw3), _ptr(dw2), _ptr(d_gates),
                                      _ptr(dX_slot), _ptr(workspace), workspace_bytes,
                                      _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_route_bwd_workspace_size(T, d, E, k, flags) -> int:
    return load_library().moe_route_bwd_workspace_size(T, d, E, k, flags)


def moe_route_bwd(d_gates, logits, topk_ids, gates, x, w_gate, T, d, E, k, flags, dw_gate, dx,
                  workspace, workspace_bytes, stream=None):
    f32 = torch.float32
    _need(d_gates, T * k, "d_gates", f32)
    _need(logits, T * E, "logits", f32)
    _need(topk_ids, T * k, "topk_ids", torch.int32)
    _need(gates, T * k, "gates", f32)
    _need(x, T * d, "x", _elt(flags))
    _need(w_gate, E * d, "w_gate", _elt(flags))
    _need(dw_gate, E * d, "dw_gate", f32)
    _need(dx, T * d, "dx", _elt(flags))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_route_bwd(_ptr(d_gates), _ptr(logits), _ptr(topk_ids),
                                        _ptr(gates), _ptr(x), _ptr(w_gate), T, d, E, k, flags,
                                        _ptr(dw_gate), _ptr(dx), _ptr(workspace),
                                        workspace_bytes, _stream(stream)))


def _current() -> int:
    """torch's current device (-2 before any GPU tensor exists)."""
    if not torch.cuda.is_initialized():
        return -2
    return _device() if _device is not None else torch.cuda.current_device()


def _args(dev: int, *specs):
    """The addresses of the tensors in `specs`, (tensor, least elements, dtype, name) each
    (None and raw addresses as they are), after all checks of the operators around the layer:
    types and sizes first, then that each is dense and on the current device `dev`, to whose
    stream the call goes."""
    ptrs, odd = [], None
    for t, n, dtype, name in specs:
        if t is None or t.__class__ is int:
            ptrs.append(t)
            continue
        if t.dtype != dtype:
            raise ValueError("%s: dtype %s, expected %s" % (name, t.dtype, dtype))
        if t.numel() < n:
            raise ValueError("%s: %d elements, at least %d needed" % (name, t.numel(), n))
        if odd is None and (t.get_device() != dev or not t.is_contiguous()):
            odd = (t, name)
        ptrs.append(t.data_ptr())
    if odd is not None:
        _misplaced(*odd, dev)
    return ptrs


def _misplaced(t, name, dev):
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if t.get_device() != dev:
        raise ValueError("%s: tensor on %s, the current device is cuda:%d" % (name, t.device, dev))
    raise ValueError("tensor must be contiguous")


def _gate_count(flags, T, d):
    """Elements of the gate of a norm call under `flags` (0: no gate)."""
    kind = flags & (MOE_GATE_CHANNEL | MOE_GATE_TOKEN)
    return {0: 0, MOE_GATE_CHANNEL: d, MOE_GATE_TOKEN: T}.get(kind, T * d)


def moe_norm_fwd(res, y, gate, w_post, w_pre, res_scale, eps, T, d, flags, r, n, rstd_post=None,
                 rstd_pre=None, stream=None):
    el, f32, m = _elt(flags), torch.float32, T * d
    p = _args(_current(), (res, m, el, "res"), (y, m, el, "y"), (gate, _gate_count(flags, T, d), el, "gate"),
              (w_post, d, el, "w_post"), (w_pre, d, el, "w_pre"), (r, m, el, "r"), (n, m, el, "n"),
              (rstd_post, T, f32, "rstd_post"), (rstd_pre, T, f32, "rstd_pre"))
    _check(load_library().moe_norm_fwd(*p[:5], res_scale, eps, T, d, flags, *p[5:], _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_norm_bwd_workspace_size(T, d, flags) -> int:
    return load_library().moe_norm_bwd_workspace_size(T, d, flags)


def moe_norm_bwd(dr, dn, y, r, gate, w_post, w_pre, rstd_post, rstd_pre, res_scale, T, d, flags,
                 dres, dy, dgate, dw_post, dw_pre, workspace, workspace_bytes, stream=None):
    el, f32, m = _elt(flags), torch.float32, T * d
    ng = _gate_count(flags, T, d)
    full = flags & MOE_GATE_CHANNEL and flags & MOE_GATE_TOKEN
    p = _args(_current(), (dr, m, el, "dr"), (dn, m, el, "dn"), (y, m, el, "y"), (r, m, el, "r"),
              (gate, ng, el, "gate"), (w_post, d, el, "w_post"), (w_pre, d, el, "w_pre"),
              (rstd_post, T, f32, "rstd_post"), (rstd_pre, T, f32, "rstd_pre"), (dres, m, el, "dres"),
              (dy, m, el, "dy"), (dgate, ng, el if full else f32, "dgate"), (dw_post, d, f32, "dw_post"),
              (dw_pre, d, f32, "dw_pre"))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_norm_bwd(*p[:9], res_scale, T, d, flags, *p[9:], _ptr(workspace),
                                       workspace_bytes, _stream(stream)))


@functools.lru_cache(maxsize=256, typed=True)
def moe_grad_norm_workspace_size(n) -> int:
    return load_library().moe_grad_norm_workspace_size(n)


class TensorList:
    """The host arrays (addresses, element counts, types) that the gradient calls take of a
    list of contiguous bfloat16 and float32 tensors. The tensors have to live on, in place."""

    def __init__(self, tensors):
        self.tensors = tensors = list(tensors)
        dev, f32, bf16 = _current(), torch.float32, torch.bfloat16
        ptrs, sizes, types = [], [], []
        for t in tensors:
            dt = t.dtype
            if dt is f32:
                types.append(MOE_F32)
            elif dt is bf16:
                types.append(MOE_BF16)
            else:
                raise ValueError("unsupported dtype %s" % dt)
            if t.get_device() != dev or not t.is_contiguous():
                _misplaced(t, "gradient", dev)
            ptrs.append(t.data_ptr())
            sizes.append(t.numel())
        self.n = len(tensors)
        self.ptrs, self.sizes, self.types = array("Q", ptrs), array("q", sizes), array("I", types)

    def addresses(self):
        return (self.ptrs.buffer_info()[0], self.sizes.buffer_info()[0], self.types.buffer_info()[0])


def moe_grad_norm(grads: TensorList, sumsq, norm, workspace, workspace_bytes, stream=None):
    ps, pn = _args(_current(), (sumsq, 1, torch.float64, "sumsq"), (norm, 1, torch.float32, "norm"))
    _need_bytes(workspace, workspace_bytes)
    _check(load_library().moe_grad_norm(*grads.addresses(), grads.n, ps, pn, _ptr(workspace),
                                        workspace_bytes, _stream(stream)))


def moe_grad_clip(grads: TensorList, outs, sumsq, max_norm, stream=None):
    """`outs`: a TensorList of the same sizes and types, or None (in place)."""
    ps, = _args(_current(), (sumsq, 1, torch.float64, "sumsq"))
    if outs is not None and (outs.sizes != grads.sizes or outs.types != grads.types):
        raise ValueError("outs: not the gradients' sizes and types")
    p, sizes, types = grads.addresses()
    _check(load_library().moe_grad_clip(p, None if outs is None else outs.addresses()[0], sizes, types,
                                        grads.n, ps, max_norm, _stream(stream)))


def moe_mx_quantize(src, batch, R, K, flags, codes, scales, stream=None):
    n, u8 = batch * R * K, torch.uint8
    p = _args(_current(), (src, n, _elt(flags), "src"), (codes, n // 2, u8, "codes"),
              (scales, n // 32, u8, "scales"))
    _check(load_library().moe_mx_quantize(p[0], batch, R, K, flags, p[1], p[2], _stream(stream)))


def moe_mx_dequantize(codes, scales, R, K, flags, out, stream=None):
    n, u8 = R * K, torch.uint8
    p = _args(_current(), (codes, n // 2, u8, "codes"), (scales, n // 32, u8, "scales"),
              (out, n, _elt(flags), "out"))
    _check(load_library().moe_mx_dequantize(p[0], p[1], R, K, flags, p[2], _stream(stream)))


def moe_mx_gemm(x, x_scales, w, w_scales, w3, w3_scales, offsets, rows, T, S, K, N, E, flags, out,
                stream=None):
    u8, i32, m, mx = torch.uint8, torch.int32, E * N * K, x_scales is not None
    p = _args(_current(), (x, T * K // 2 if mx else T * K, u8 if mx else torch.bfloat16, "x"),
              (x_scales, T * K // 32, u8, "x_scales"), (w, m // 2, u8, "w"), (w_scales, m // 32, u8, "w_scales"),
              (w3, m // 2, u8, "w3"), (w3_scales, m // 32, u8, "w3_scales"), (offsets, E + 1, i32, "offsets"),
              (rows, S, i32, "rows"), (out, S * N, torch.bfloat16, "out"))
    _check(load_library().moe_mx_gemm(*p[:8], T, S, K, N, E, flags, p[8], _stream(stream)))


def moe_probe_enable(capacity: int):
    _check(load_library().moe_probe_enable(capacity))


def moe_probe_disable():
    load_library().moe_probe_disable()


def moe_probe_count() -> int:
    return load_library().moe_probe_count()


def moe_probe_dropped() -> int:
    return load_library().moe_probe_dropped()


def moe_probe_get(index: int):
    """Returns (kernel name, milliseconds) of kernel record `index`."""
    name = ctypes.c_char_p()
    ms = ctypes.c_float()
    _check(load_library().moe_probe_get(index, ctypes.byref(name), ctypes.byref(ms)))
    return name.value.decode(), ms.value

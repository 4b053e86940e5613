"""Thin Python binding of the operators in ``include/gptq_w4a16_serving.h`` (argument marshalling only).

Every function has the name and the contract of its C counterpart; tensors are torch CUDA(HIP) tensors, shapes are taken
from them, and the work is enqueued on torch's current stream.  Nothing is computed on the host and there is no fallback.
The packed weights of a layer's experts are given as ``(qweight, qzeros, scales)``, stacked along a first axis:
``gate_up`` with the gate projection's columns before the up projection's, and ``down``.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import GptqError, _ptr, _stream, load

EXPORTS = ("gptq_w4a16_moe_route", "gptq_w4a16_moe_experts", "gptq_w4a16_moe", "gptq_w4a16_moe_workspace_bytes",
           "gptq_w4a16_lora_add", "gptq_w4a16_gemm_lora", "gptq_w4a16_lora_workspace_bytes")

_LOGITS_TYPE = {torch.float16: 0, torch.float32: 1}


class Experts(ctypes.Structure):
    """Mirror of gptq_w4a16_experts_t."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("gate_up_qweight", "gate_up_qzeros", "gate_up_scales", "down_qweight",
                                               "down_qzeros", "down_scales")] + \
               [(n, ctypes.c_int) for n in ("experts", "hidden", "inter", "group_size")]


_lib = None
_addresses = {}  # of the entry points that the extension module calls


def _load():
    """The library with the argument types of this module's functions."""
    global _lib
    if _lib is None:
        lib = load()
        vp, ci, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        experts = ctypes.POINTER(Experts)
        for name, restype, argtypes in [
                ("gptq_w4a16_moe_route", ci, [vp, ci, vp, vp, ci, ci, ci, ci, vp]),
                ("gptq_w4a16_moe_experts", ci, [vp, vp, vp, experts, vp, ci, ci, vp]),
                ("gptq_w4a16_moe", ci, [vp, vp, ci, experts, vp, ci, ci, ci, vp]),
                ("gptq_w4a16_moe_workspace_bytes", size, [ci] * 6),
                ("gptq_w4a16_lora_add", ci, [vp] * 7 + [ci] * 8 + [vp]),
                ("gptq_w4a16_gemm_lora", ci, [vp] * 9 + [ci] * 6 + [vp]),
                ("gptq_w4a16_lora_workspace_bytes", size, [ci] * 5)]:
            getattr(lib, name).restype = restype
            getattr(lib, name).argtypes = argtypes
            _addresses[name] = ctypes.cast(getattr(lib, name), vp).value
        _lib = lib
    return _lib


def _native(function, name, *args):
    """Whether the extension module (csrc/native_call.cpp) has made the call; it leaves to the code below what is not plain."""
    if _lib is None:
        _load()
    module = binding._native_module
    rc = None if module is None else getattr(module, function)(_addresses[name], *args)
    if rc:
        raise GptqError(rc, name)
    return rc == 0


def _shape(t, shape, name):
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _logits(logits):
    if logits.dtype not in _LOGITS_TYPE:
        raise TypeError(f"logits must be torch.float16 or torch.float32, got {logits.dtype}")
    return _ptr(logits, logits.dtype, "logits"), _LOGITS_TYPE[logits.dtype]


def _matrices(packed, name, experts, K, N, group_size):
    """Pointers of stacked packed matrices [K, N]."""
    qweight, qzeros, scales = packed
    if group_size <= 0 or K % group_size or K % 8 or N % 8:
        raise ValueError(f"{name}: group_size must divide {K}, and {K} and {N} be multiples of 8")
    _shape(qweight, (experts, K // 8, N), f"{name} qweight")
    _shape(qzeros, (experts, K // group_size, N // 8), f"{name} qzeros")
    _shape(scales, (experts, K // group_size, N), f"{name} scales")
    return (_ptr(qweight, torch.int32, f"{name} qweight"), _ptr(qzeros, torch.int32, f"{name} qzeros"),
            _ptr(scales, torch.float16, f"{name} scales"))


def _experts(x, gate_up, down, out, group_size):
    """The layer's description and M."""
    if x.dim() != 2 or gate_up[0].dim() != 3:
        raise ValueError("x must be [M, hidden] and the packed weights [experts, ...]")
    M, hidden = x.shape
    experts, inter = gate_up[0].shape[0], gate_up[0].shape[2] // 2
    _shape(out, (M, hidden), "out")
    group_size = int(group_size)
    return Experts(*_matrices(gate_up, "gate_up", experts, hidden, 2 * inter, group_size),
                   *_matrices(down, "down", experts, inter, hidden, group_size), experts, hidden, inter, group_size), M


def gptq_w4a16_moe_route(logits, ids, weights, renormalize: bool = True):
    """The top_k experts of every token and their softmax weights: fills ids [M, top_k] (int32) and weights (float32)."""
    if _native("route", "gptq_w4a16_moe_route", logits, ids, weights, renormalize):
        return ids, weights
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits must be [M, experts] and ids [M, top_k]")
    M, experts = logits.shape
    top_k = ids.shape[1]
    _shape(ids, (M, top_k), "ids")
    _shape(weights, (M, top_k), "weights")
    rc = _load().gptq_w4a16_moe_route(*_logits(logits), _ptr(ids, torch.int32, "ids"),
                                      _ptr(weights, torch.float32, "weights"), M, experts, top_k, int(bool(renormalize)),
                                      _stream())
    if rc != 0:
        raise GptqError(rc, "gptq_w4a16_moe_route")
    return ids, weights


def gptq_w4a16_moe_experts(x, ids, weights, gate_up, down, out, group_size: int):
    """out[M, hidden] = the weighted sum of every token's experts; an id outside [0, experts) adds nothing."""
    if _native("moe_experts", "gptq_w4a16_moe_experts", x, ids, weights, gate_up, down, out, group_size):
        return out
    layer, M = _experts(x, gate_up, down, out, group_size)
    if ids.dim() != 2:
        raise ValueError("ids must be [M, top_k]")
    top_k = ids.shape[1]
    _shape(ids, (M, top_k), "ids")
    _shape(weights, (M, top_k), "weights")
    rc = _load().gptq_w4a16_moe_experts(_ptr(x, torch.float16, "x"), _ptr(ids, torch.int32, "ids"),
                                        _ptr(weights, torch.float32, "weights"), ctypes.byref(layer),
                                        _ptr(out, torch.float16, "out"), M, top_k, _stream())
    if rc != 0:
        raise GptqError(rc, "gptq_w4a16_moe_experts")
    return out


def gptq_w4a16_moe(x, logits, gate_up, down, out, top_k: int, group_size: int, renormalize: bool = True):
    """The whole layer: routing by `logits` [M, experts], then the experts."""
    if _native("moe", "gptq_w4a16_moe", x, logits, gate_up, down, out, top_k, group_size, renormalize):
        return out
    layer, M = _experts(x, gate_up, down, out, group_size)
    _shape(logits, (M, layer.experts), "logits")
    pointer, kind = _logits(logits)
    rc = _load().gptq_w4a16_moe(_ptr(x, torch.float16, "x"), pointer, kind, ctypes.byref(layer),
                                _ptr(out, torch.float16, "out"), M, int(top_k), int(bool(renormalize)), _stream())
    if rc != 0:
        raise GptqError(rc, "gptq_w4a16_moe")
    return out


def gptq_w4a16_moe_workspace_bytes(M: int, hidden: int, inter: int, experts: int, top_k: int, group_size: int) -> int:
    return int(_load().gptq_w4a16_moe_workspace_bytes(int(M), int(hidden), int(inter), int(experts), int(top_k),
                                                      int(group_size)))


def _rows(t, name):
    """Pointer and row stride of a matrix whose rows may stand apart (columns of a wider one)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if t.dtype != torch.float16:
        raise TypeError(f"{name} must be torch.float16, got {t.dtype}")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError(f"the rows of {name} overlap")
    if ld > 2 ** 31 - 1:
        raise ValueError(f"the rows of {name} stand too far apart")
    return t.data_ptr(), ld


def _adapters(x, a, b, scaling, adapter, out):
    if x.dim() != 2 or a.dim() != 3 or out.dim() != 2:
        raise ValueError("x must be [M, K], a [adapters, rank, K] and out [M, N]")
    M, K = x.shape
    N = out.shape[1]
    adapters, rank = a.shape[:2]
    _shape(a, (adapters, rank, K), "a")
    _shape(b, (adapters, N, rank), "b")
    _shape(scaling, (adapters,), "scaling")
    _shape(adapter, (M,), "adapter")
    _shape(out, (M, N), "out")
    pointers = (_ptr(a, torch.float16, "a"), _ptr(b, torch.float16, "b"), _ptr(scaling, torch.float32, "scaling"),
                _ptr(adapter, torch.int32, "adapter"))
    return pointers, M, K, N, rank, adapters


def gptq_w4a16_lora_add(x, a, b, scaling, adapter, base, out):
    """out[m] = base[m] + scaling[l] * (x[m] @ a[l].T) @ b[l].T with l = adapter[m], or base[m] where l is no adapter.
    The rows of x, base and out may be strided; out may be base."""
    if _native("lora_add", "gptq_w4a16_lora_add", x, a, b, scaling, adapter, base, out):
        return out
    pointers, M, K, N, rank, adapters = _adapters(x, a, b, scaling, adapter, out)
    _shape(base, (M, N), "base")
    px, ldx = _rows(x, "x")
    pb, ld_base = _rows(base, "base")
    po, ld_out = _rows(out, "out")
    rc = _load().gptq_w4a16_lora_add(px, *pointers, pb, po, M, K, N, rank, adapters, ldx, ld_base, ld_out, _stream())
    if rc != 0:
        raise GptqError(rc, "gptq_w4a16_lora_add")
    return out


def gptq_w4a16_gemm_lora(x, qweight, qzeros, scales, a, b, scaling, adapter, out, group_size: int):
    """out = x @ W (gptq_w4a16_gemm) with every row's adapter on top."""
    if _native("gemm_lora", "gptq_w4a16_gemm_lora", x, qweight, qzeros, scales, a, b, scaling, adapter, out, group_size):
        return out
    pointers, M, K, N, rank, adapters = _adapters(x, a, b, scaling, adapter, out)
    group_size = int(group_size)
    if group_size <= 0 or K % group_size or K % 8 or N % 8:
        raise ValueError(f"group_size must divide {K}, and {K} and {N} be multiples of 8")
    _shape(qweight, (K // 8, N), "qweight")
    _shape(qzeros, (K // group_size, N // 8), "qzeros")
    _shape(scales, (K // group_size, N), "scales")
    rc = _load().gptq_w4a16_gemm_lora(_ptr(x, torch.float16, "x"), _ptr(qweight, torch.int32, "qweight"),
                                      _ptr(qzeros, torch.int32, "qzeros"), _ptr(scales, torch.float16, "scales"),
                                      *pointers, _ptr(out, torch.float16, "out"), M, K, N, group_size, rank, adapters,
                                      _stream())
    if rc != 0:
        raise GptqError(rc, "gptq_w4a16_gemm_lora")
    return out


def gptq_w4a16_lora_workspace_bytes(M: int, K: int, N: int, rank: int, group_size: int = 0) -> int:
    return int(_load().gptq_w4a16_lora_workspace_bytes(int(M), int(K), int(N), int(rank), int(group_size)))

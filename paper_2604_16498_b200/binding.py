"""Python binding of the C ABI in ``include/forge.h`` (argument marshalling only).

Every function takes torch tensors (used purely as owners of device or pinned host
memory), checks shapes and dtypes, and passes raw pointers, sizes and the current
CUDA stream to ``libforge.so``.  All arithmetic happens inside the library's kernels.
There is no fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

import torch

from .build import host_calls_stamp

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libforge.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
MASK_NONE, MASK_CAUSAL, MASK_PADDING, MASK_CAUSAL_PADDING = range(4)

# name -> (restype, argtypes); mirrors include/forge.h
_vp, _i, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_ATTN = [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _f]
_DEC = [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _i, _f]
SIGNATURES = {
    "forge_attn_fused": (_i, _ATTN + [_vp]),
    "forge_attn_fused_f32": (_i, _ATTN + [_vp]),
    "forge_attn_fused_f16": (_i, _ATTN + [_vp]),
    "forge_attn_fused_strided": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp, _f, _vp]),
    "forge_attn_fused_bias": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _i, _f, _vp]),
    "forge_attn_decode_splitkv": (_i, _DEC + [_vp, _sz, _vp]),
    "forge_attn_decode_splitkv_f16": (_i, _DEC + [_vp, _sz, _vp]),
    "forge_attn_decode_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "forge_attn_decode_workspace_init": (_i, [_vp, _sz, _vp]),
    "forge_attn_decode_splitkv_static": (_i, _DEC + [_vp]),
    "forge_linear_bias_gelu": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _vp]),
    "forge_linear_act": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "forge_linear_act_f16": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp]),
    "forge_linear_act_w8a16": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "forge_linear_swiglu": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp]),
    "forge_attn_host_scratch_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "forge_attn_fused_host": (_i, _ATTN + [_vp, _sz, _vp]),
    "forge_attn_fused_f32_host": (_i, _ATTN + [_vp, _sz, _vp]),
    "forge_attn_decode_host_scratch_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "forge_attn_decode_splitkv_host": (_i, _DEC + [_vp, _sz, _vp]),
    "forge_linear_host_scratch_bytes": (_sz, [_i, _i, _i]),
    "forge_linear_bias_gelu_host": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _vp, _sz, _vp]),
    "forge_check_status": (_i, [_vp]),
    "forge_activation_f32": (_i, [_vp, _vp, _sz, _i, _i, _vp]),
    "forge_debug_wait_timeout": (_i, [ctypes.c_longlong, _vp]),
    "forge_status_string": (ctypes.c_char_p, [_i]),
    "forge_last_cuda_error": (_i, []),
    "forge_launch_count": (ctypes.c_ulonglong, []),
}



class LayerDesc(ctypes.Structure):
    """forge_decoder_layer_desc"""
    _fields_ = [("B", _i), ("S", _i), ("Hq", _i), ("Hkv", _i), ("D", _i), ("F", _i), ("mlp_kind", _i),
                ("w_layout", _i), ("mask_kind", _i), ("scale", _f), ("lens", _vp),
                ("w_qkv", _vp), ("b_qkv", _vp), ("w_o", _vp), ("b_o", _vp), ("w_gate", _vp), ("w_up", _vp),
                ("b_up", _vp), ("w_down", _vp), ("b_down", _vp)]


class LayerPlan(ctypes.Structure):
    """forge_layer_plan"""
    _fields_ = [("num_regs", _i), ("num_bufs", _i), ("rho_buf", _f), ("buf_of", _i * 4), ("reg_start", _i * 4),
                ("reg_end", _i * 4), ("reg_bytes", _sz * 4), ("buf_bytes", _sz * 4), ("buf_offset", _sz * 4),
                ("workspace_bytes", _sz), ("unplanned_bytes", _sz)]


SIGNATURES.update({
    "forge_plan_liveness": (_i, [_i, _vp, _vp, _vp, _i, _vp, _vp]),
    "forge_plan_linear_scan": (_i, [_i, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "forge_decoder_layer_plan": (_i, [ctypes.POINTER(LayerDesc), ctypes.POINTER(LayerPlan)]),
    "forge_decoder_layer_workspace_bytes": (_sz, [ctypes.POINTER(LayerDesc)]),
    "forge_decoder_layer": (_i, [ctypes.POINTER(LayerDesc), _vp, _vp, _vp, _sz, _vp]),
})


class KVCacheDesc(ctypes.Structure):
    """forge_kv_cache"""
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("B", _i), ("Hkv", _i), ("Smax", _i), ("D", _i),
                ("format", _i)]


class RotaryScaling(ctypes.Structure):
    """forge_rotary_scaling: kind ROTARY_SCALE_*, factor, the ramps' bounds fast and slow in turns, original_len."""
    _fields_ = [("kind", _i), ("factor", ctypes.c_double), ("fast", ctypes.c_double), ("slow", ctypes.c_double),
                ("original_len", _i)]


class RotaryDesc(ctypes.Structure):
    """forge_rotary"""
    _fields_ = [("inv_freq", _vp), ("dims", _i), ("layout", _i), ("amplitude", _f)]


_i64x3 = ctypes.c_int64 * 3


class KVAppendDesc(ctypes.Structure):
    """forge_kv_append_desc"""
    _fields_ = [("k", _vp), ("v", _vp), ("q", _vp), ("q_out", _vp),
                ("k_strides", ctypes.POINTER(ctypes.c_int64)), ("v_strides", ctypes.POINTER(ctypes.c_int64)),
                ("q_strides", ctypes.POINTER(ctypes.c_int64)), ("q_out_strides", ctypes.POINTER(ctypes.c_int64)),
                ("lens", _vp), ("counts", _vp), ("positions", _vp), ("rows", _vp), ("rotary", ctypes.POINTER(RotaryDesc)),
                ("dtype", _i), ("Hq", _i), ("S", _i), ("S_src", _i)]


SIGNATURES.update({
    "forge_rotary_frequencies": (_i, [_i, ctypes.c_double, ctypes.POINTER(RotaryScaling), _vp, _vp]),
    "forge_rotary_apply": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, ctypes.POINTER(RotaryDesc), _i, _vp]),
    "forge_kv_append": (_i, [ctypes.POINTER(KVCacheDesc), ctypes.POINTER(KVAppendDesc), _vp]),
    "forge_kv_read": (_i, [ctypes.POINTER(KVCacheDesc), _vp, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp]),
    "forge_attn_kv_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "forge_attn_kv_workspace_init": (_i, [_vp, _sz, _vp]),
    "forge_attn_decode_kv": (_i, [ctypes.POINTER(KVCacheDesc), _vp, _vp, _i, _i, _vp, _f, _vp, _sz, _vp]),
    "forge_attn_tree": (_i, [ctypes.POINTER(KVCacheDesc), _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _f, _vp, _sz, _vp]),
})

class KVPagesDesc(ctypes.Structure):
    """forge_kv_pages"""
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("num_pages", _i), ("Hkv", _i), ("page_size", _i), ("D", _i),
                ("format", _i)]


class PageTablesDesc(ctypes.Structure):
    """forge_kv_page_tables"""
    _fields_ = [("table", _vp), ("free_pages", _vp), ("free_count", _vp), ("B", _i), ("max_pages", _i), ("page_size", _i),
                ("num_pages", _i)]


class PageSlotsDesc(ctypes.Structure):
    """forge_kv_page_slots"""
    _fields_ = [("new_lens", _vp), ("starts", _vp), ("slots", _vp), ("positions", _vp), ("requests", _vp), ("T", _i)]


class KVAppendPagesDesc(ctypes.Structure):
    """forge_kv_append_pages_desc"""
    _fields_ = [("k", _vp), ("v", _vp), ("q", _vp), ("q_out", _vp),
                ("k_strides", ctypes.POINTER(ctypes.c_int64)), ("v_strides", ctypes.POINTER(ctypes.c_int64)),
                ("q_strides", ctypes.POINTER(ctypes.c_int64)), ("q_out_strides", ctypes.POINTER(ctypes.c_int64)),
                ("slots", _vp), ("positions", _vp), ("rotary", ctypes.POINTER(RotaryDesc)), ("dtype", _i), ("Hq", _i), ("T", _i)]


class AdaptersDesc(ctypes.Structure):
    """forge_adapters"""
    _fields_ = [("a", _vp), ("b", _vp), ("scales", _vp), ("n", _i), ("rank", _i), ("K", _i), ("N", _i), ("dtype", _i)]


_i64 = ctypes.c_int64
SIGNATURES.update({
    "forge_kv_assign_pages": (_i, [ctypes.POINTER(PageTablesDesc), _vp, _vp, ctypes.POINTER(PageSlotsDesc), _vp, _vp]),
    "forge_kv_release_pages": (_i, [ctypes.POINTER(PageTablesDesc), _vp, _vp, _vp, _vp]),
    "forge_kv_append_pages": (_i, [ctypes.POINTER(KVPagesDesc), ctypes.POINTER(KVAppendPagesDesc), _vp]),
    "forge_kv_read_pages": (_i, [ctypes.POINTER(KVPagesDesc), _vp, _i, _i, _vp, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp]),
    "forge_attn_decode_pages": (_i, [ctypes.POINTER(KVPagesDesc), _vp, _i, _i, _vp, _vp, _i, _i, _vp, _f, _vp, _sz, _vp]),
    "forge_attn_tree_pages": (_i, [ctypes.POINTER(KVPagesDesc), _vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _f, _vp, _sz,
                                   _vp]),
    "forge_linear_adapters": (_i, [ctypes.POINTER(AdaptersDesc), _vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i, _vp, _sz, _vp]),
    "forge_linear_adapters_workspace_bytes": (_sz, [_i, _i]),
})

_lib = None
# host_calls.cpp: the frequent calls' marshalling in native code.  Its functions return -1 where a call is not plain (anything but
# dense, contiguous CUDA tensors of matching shapes with the output given); then the Python below does it, with every check.
_host_calls = None
_HOST_CALLS_ENTRIES = ("forge_attn_fused", "forge_attn_fused_f16", "forge_attn_fused_f32", "forge_attn_decode_splitkv",
                       "forge_attn_decode_splitkv_f16", "forge_linear_act", "forge_linear_act_f16", "forge_linear_act_w8a16",
                       "forge_linear_swiglu")
_HOST_CALLS_KV_ENTRIES = ("forge_rotary_apply", "forge_kv_append", "forge_kv_read", "forge_attn_decode_kv", "forge_attn_tree")

_HOST_CALLS_PAGES_ENTRIES = ("forge_kv_assign_pages", "forge_kv_append_pages", "forge_kv_read_pages", "forge_attn_decode_pages",
                             "forge_attn_tree_pages", "forge_linear_adapters", "forge_linear_adapters_workspace_bytes")


class ForgeError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        lib = load()
        name = lib.forge_status_string(status).decode()
        extra = f" (cudaError {lib.forge_last_cuda_error()})" if status == ERR_CUDA else ""
        super().__init__(f"{fn} failed: {name}{extra}")


def load() -> ctypes.CDLL:
    """Loads ``libforge.so`` (built by ``paper_2604_16498_b200.build``).  Raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2604_16498_b200.build` "
                               "(there is no fallback implementation)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        _bind_host_calls(lib)
    return _lib


def _bind_host_calls(lib) -> None:
    global _host_calls
    try:
        from . import host_calls
    except ImportError:  # not built, or for another Python: the general way
        return
    # Its symbols may resolve in another torch too, whose tensors it would read wrongly: the general way.
    if getattr(host_calls, "built_for", None) != host_calls_stamp():
        return
    host_calls.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _HOST_CALLS_ENTRIES))
    host_calls.bind_pages(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _HOST_CALLS_PAGES_ENTRIES))
    host_calls.bind_kv(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _HOST_CALLS_KV_ENTRIES))
    _host_calls = host_calls


def _find_raw_stream():
    """torch.cuda.current_stream() builds a Stream object around the stream's number, which takes 3.2 us, a third of the host
    time of a small call; these two lookups take a tenth of that.  They are not part of torch's public interface: a torch
    without them gets the public way."""
    get, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if get is None or dev is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: get(dev())


_raw_stream = _find_raw_stream()


def _stream() -> int:
    """The calling thread's current stream on its current device, as a number."""
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return _raw_stream()


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of {dtype}")
    return t.data_ptr()


def _host(t: torch.Tensor, dtype, name: str) -> int:
    if t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous host tensor of {dtype}")
    return t.data_ptr()


def _check(fn: str, status: int) -> None:
    if status != OK:
        raise ForgeError(fn, status)


def _attn_dims(q, k, v):
    B, Hq, Sq, D = q.shape
    Bk, Hkv, Skv, Dk = k.shape
    if (Bk, Dk) != (B, D) or tuple(v.shape) != tuple(k.shape):
        raise ValueError("q [B,Hq,Sq,D], k/v [B,Hkv,Skv,D] expected")
    return B, Hq, Hkv, Sq, Skv, D


def attn_fused(q, k, v, mask_kind=MASK_NONE, lens=None, scale=None, out=None):
    """forge_attn_fused: bf16 tensors q [B,Hq,Sq,D], k/v [B,Hkv,Skv,D] on the GPU."""
    if _host_calls is not None:
        st = _host_calls.attn(0, q, k, v, mask_kind, lens, scale, out)
        if st >= 0:
            _check("forge_attn_fused", st)
            return out
    B, Hq, Hkv, Sq, Skv, D = _attn_dims(q, k, v)
    out = torch.empty_like(q) if out is None else out
    scale = D ** -0.5 if scale is None else scale
    lp = None if lens is None else _dev(lens, torch.int32, "lens")
    _check("forge_attn_fused", load().forge_attn_fused(
        _dev(q, torch.bfloat16, "q"), _dev(k, torch.bfloat16, "k"), _dev(v, torch.bfloat16, "v"),
        _dev(out, torch.bfloat16, "out"), B, Hq, Hkv, Sq, Skv, D, int(mask_kind), lp, float(scale), _stream()))
    return out


def attn_fused_strided(q, k, v, out, mask_kind=MASK_NONE, lens=None, scale=None):
    """forge_attn_fused_strided: q/out [B,Hq,Sq,D] and k/v [B,Hkv,Skv,D] bf16 VIEWS (any strides with a
    contiguous last dimension, e.g. slices of a fused QKV projection permuted to head-major)."""
    B, Hq, Sq, D = q.shape
    _, Hkv, Skv, _ = k.shape
    if tuple(k.shape) != (B, Hkv, Skv, D) or tuple(v.shape) != (B, Hkv, Skv, D) or tuple(out.shape) != (B, Hq, Sq, D):
        raise ValueError("q/out [B,Hq,Sq,D], k/v [B,Hkv,Skv,D] expected")
    scale = D ** -0.5 if scale is None else scale
    arrs = []
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.stride(3) == 1):
            raise ValueError(f"{name}: expected a CUDA bf16 tensor whose last dimension is contiguous")
        arrs.append((ctypes.c_int64 * 3)(t.stride(0), t.stride(1), t.stride(2)))
    lp = None if lens is None else _dev(lens, torch.int32, "lens")
    _check("forge_attn_fused_strided", load().forge_attn_fused_strided(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, Hq, Hkv, Sq, Skv, D,
        arrs[0], arrs[1], arrs[2], arrs[3], int(mask_kind), lp, float(scale), _stream()))
    return out


def attn_fused_f16(q, k, v, mask_kind=MASK_NONE, lens=None, scale=None, out=None):
    """forge_attn_fused_f16: the same operator on fp16 tensors."""
    if _host_calls is not None:
        st = _host_calls.attn(1, q, k, v, mask_kind, lens, scale, out)
        if st >= 0:
            _check("forge_attn_fused_f16", st)
            return out
    B, Hq, Hkv, Sq, Skv, D = _attn_dims(q, k, v)
    out = torch.empty_like(q) if out is None else out
    scale = D ** -0.5 if scale is None else scale
    lp = None if lens is None else _dev(lens, torch.int32, "lens")
    _check("forge_attn_fused_f16", load().forge_attn_fused_f16(
        _dev(q, torch.float16, "q"), _dev(k, torch.float16, "k"), _dev(v, torch.float16, "v"),
        _dev(out, torch.float16, "out"), B, Hq, Hkv, Sq, Skv, D, int(mask_kind), lp, float(scale), _stream()))
    return out


def attn_fused_bias(q, k, v, bias, mask_kind=MASK_NONE, lens=None, scale=None, out=None):
    """forge_attn_fused_bias: bf16 q/k/v and an fp32 additive bias [B, 1 or Hq, Sq, Skv] on the scaled scores."""
    B, Hq, Hkv, Sq, Skv, D = _attn_dims(q, k, v)
    if bias.dim() != 4 or bias.shape[0] != B or bias.shape[2] != Sq or bias.shape[3] != Skv:
        raise ValueError("bias [B, 1 or Hq, Sq, Skv] expected")
    out = torch.empty_like(q) if out is None else out
    scale = D ** -0.5 if scale is None else scale
    lp = None if lens is None else _dev(lens, torch.int32, "lens")
    _check("forge_attn_fused_bias", load().forge_attn_fused_bias(
        _dev(q, torch.bfloat16, "q"), _dev(k, torch.bfloat16, "k"), _dev(v, torch.bfloat16, "v"),
        _dev(out, torch.bfloat16, "out"), B, Hq, Hkv, Sq, Skv, D, int(mask_kind), lp,
        _dev(bias, torch.float32, "bias"), int(bias.shape[1]), float(scale), _stream()))
    return out


def attn_fused_f32(q, k, v, mask_kind=MASK_NONE, lens=None, scale=None, out=None):
    """forge_attn_fused_f32: the same operator on fp32 tensors."""
    if _host_calls is not None:
        st = _host_calls.attn(2, q, k, v, mask_kind, lens, scale, out)
        if st >= 0:
            _check("forge_attn_fused_f32", st)
            return out
    B, Hq, Hkv, Sq, Skv, D = _attn_dims(q, k, v)
    out = torch.empty_like(q) if out is None else out
    scale = D ** -0.5 if scale is None else scale
    lp = None if lens is None else _dev(lens, torch.int32, "lens")
    _check("forge_attn_fused_f32", load().forge_attn_fused_f32(
        _dev(q, torch.float32, "q"), _dev(k, torch.float32, "k"), _dev(v, torch.float32, "v"),
        _dev(out, torch.float32, "out"), B, Hq, Hkv, Sq, Skv, D, int(mask_kind), lp, float(scale), _stream()))
    return out


def attn_decode_workspace_bytes(B, Hq, D, num_splits) -> int:
    return int(load().forge_attn_decode_workspace_bytes(B, Hq, D, num_splits))


def attn_decode_workspace_init(workspace) -> None:
    """forge_attn_decode_workspace_init: clears a new decode workspace (its arrival counters must start at zero)."""
    _check("forge_attn_decode_workspace_init", load().forge_attn_decode_workspace_init(
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))


def attn_decode_splitkv(q, k_cache, v_cache, lens, num_splits, scale=None, out=None, workspace=None):
    """forge_attn_decode_splitkv (bf16 tensors) or forge_attn_decode_splitkv_f16 (fp16 tensors), chosen by
    q.dtype: q [B,Hq,D], caches [B,Hkv,Smax,D], lens int32 [B].  A workspace passed in must have been
    cleared once (attn_decode_workspace_init); without one, a fresh cleared workspace is allocated."""
    if _host_calls is not None:
        f16 = q.dtype == torch.float16
        st = _host_calls.decode(1 if f16 else 0, q, k_cache, v_cache, lens, num_splits, scale, out, workspace)
        if st >= 0:
            _check("forge_attn_decode_splitkv_f16" if f16 else "forge_attn_decode_splitkv", st)
            return out
    B, Hq, D = q.shape
    Bk, Hkv, Smax, Dk = k_cache.shape
    if (Bk, Dk) != (B, D) or tuple(v_cache.shape) != tuple(k_cache.shape):
        raise ValueError("q [B,Hq,D], caches [B,Hkv,Smax,D] expected")
    out = torch.empty_like(q) if out is None else out
    scale = D ** -0.5 if scale is None else scale
    if workspace is None:
        need = attn_decode_workspace_bytes(B, Hq, D, num_splits)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
        attn_decode_workspace_init(workspace)
    dt = torch.float16 if q.dtype == torch.float16 else torch.bfloat16
    name = "forge_attn_decode_splitkv_f16" if dt == torch.float16 else "forge_attn_decode_splitkv"
    _check(name, getattr(load(), name)(
        _dev(q, dt, "q"), _dev(k_cache, dt, "k_cache"),
        _dev(v_cache, dt, "v_cache"), _dev(out, dt, "out"),
        B, Hq, Hkv, Smax, D, _dev(lens, torch.int32, "lens"), int(num_splits), float(scale),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


DECODE_STATIC_SCRATCH_BYTES = 8 << 20


def attn_decode_splitkv_static(q, k_cache, v_cache, lens, num_splits, out, scale=None):
    """forge_attn_decode_splitkv_static: the decode step for callers that cannot allocate a
    workspace.  The partials go to a fixed 8 MiB array inside the library (shared by all calls on
    the device, so calls must not overlap); larger problems raise ForgeError(ERR_WORKSPACE).
    `out` is the caller's buffer: nothing is allocated here either."""
    B, Hq, D = q.shape
    Bk, Hkv, Smax, Dk = k_cache.shape
    if (Bk, Dk) != (B, D) or tuple(v_cache.shape) != tuple(k_cache.shape):
        raise ValueError("q [B,Hq,D], caches [B,Hkv,Smax,D] expected")
    scale = D ** -0.5 if scale is None else scale
    _check("forge_attn_decode_splitkv_static", load().forge_attn_decode_splitkv_static(
        _dev(q, torch.bfloat16, "q"), _dev(k_cache, torch.bfloat16, "k_cache"),
        _dev(v_cache, torch.bfloat16, "v_cache"), _dev(out, torch.bfloat16, "out"),
        B, Hq, Hkv, Smax, D, _dev(lens, torch.int32, "lens"), int(num_splits), float(scale), _stream()))
    return out


def linear_bias_gelu(x, w, b, out=None):
    """forge_linear_bias_gelu: x [M,K], w [K,N], b [N] (bf16) -> gelu_tanh(x @ w + b) [M,N]."""
    M, K = x.shape
    K2, N = w.shape
    if K2 != K or tuple(b.shape) != (N,):
        raise ValueError("x [M,K], w [K,N], b [N] expected")
    out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device) if out is None else out
    _check("forge_linear_bias_gelu", load().forge_linear_bias_gelu(
        _dev(x, torch.bfloat16, "x"), _dev(w, torch.bfloat16, "w"), _dev(b, torch.bfloat16, "b"),
        _dev(out, torch.bfloat16, "out"), M, N, K, _stream()))
    return out


ACT_GELU_TANH, ACT_GELU_ERF, ACT_RELU, ACT_SILU, ACT_NONE = range(5)
W_KN, W_NK = 0, 1


def linear_act(x, w, b=None, residual=None, act=ACT_GELU_TANH, w_layout=W_KN, out=None):
    """forge_linear_act (bf16 tensors) or forge_linear_act_f16 (fp16 tensors), chosen by x.dtype:
    act(x @ W + b) + residual with W given as [K,N] (W_KN) or [N,K] (W_NK)."""
    if _host_calls is not None:
        f16 = x.dtype == torch.float16
        st = _host_calls.linear(1 if f16 else 0, x, w, b, residual, act, w_layout, out)
        if st >= 0:
            _check("forge_linear_act_f16" if f16 else "forge_linear_act", st)
            return out
    M, K = x.shape
    N = w.shape[1] if w_layout == W_KN else w.shape[0]
    if tuple(w.shape) != ((K, N) if w_layout == W_KN else (N, K)):
        raise ValueError("w must be [K,N] for W_KN and [N,K] for W_NK")
    if b is not None and tuple(b.shape) != (N,):
        raise ValueError("b [N] expected")
    if residual is not None and tuple(residual.shape) != (M, N):
        raise ValueError("residual [M,N] expected")
    out = torch.empty((M, N), dtype=x.dtype, device=x.device) if out is None else out
    bf = torch.float16 if x.dtype == torch.float16 else torch.bfloat16
    name = "forge_linear_act_f16" if bf == torch.float16 else "forge_linear_act"
    _check(name, getattr(load(), name)(
        _dev(x, bf, "x"), _dev(w, bf, "w"), None if b is None else _dev(b, bf, "b"),
        None if residual is None else _dev(residual, bf, "residual"), _dev(out, bf, "out"),
        M, N, K, int(act), int(w_layout), _stream()))
    return out


def linear_act_w8a16(x, w_int8, scale, b=None, residual=None, act=ACT_GELU_TANH, out=None):
    """forge_linear_act_w8a16: fp16 x [M,K], int8 weights [N,K], fp32 per-channel scale [N]."""
    if _host_calls is not None:
        st = _host_calls.linear_w8(x, w_int8, scale, b, residual, act, out)
        if st >= 0:
            _check("forge_linear_act_w8a16", st)
            return out
    M, K = x.shape
    N = w_int8.shape[0]
    if tuple(w_int8.shape) != (N, K) or tuple(scale.shape) != (N,):
        raise ValueError("w_int8 [N,K] and scale [N] expected")
    out = torch.empty((M, N), dtype=torch.float16, device=x.device) if out is None else out
    h = torch.float16
    _check("forge_linear_act_w8a16", load().forge_linear_act_w8a16(
        _dev(x, h, "x"), _dev(w_int8, torch.int8, "w_int8"), _dev(scale, torch.float32, "scale"),
        None if b is None else _dev(b, h, "b"), None if residual is None else _dev(residual, h, "residual"),
        _dev(out, h, "out"), M, N, K, int(act), _stream()))
    return out


def linear_swiglu(x, w_gate, w_up, w_layout=W_KN, out=None):
    """forge_linear_swiglu: silu(x @ Wg) * (x @ Wu); both weights [K,N] (W_KN) or [N,K] (W_NK)."""
    if _host_calls is not None:
        st = _host_calls.swiglu(x, w_gate, w_up, w_layout, out)
        if st >= 0:
            _check("forge_linear_swiglu", st)
            return out
    M, K = x.shape
    N = w_gate.shape[1] if w_layout == W_KN else w_gate.shape[0]
    want = (K, N) if w_layout == W_KN else (N, K)
    if tuple(w_gate.shape) != want or tuple(w_up.shape) != want:
        raise ValueError("w_gate and w_up must both be [K,N] for W_KN or [N,K] for W_NK")
    out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device) if out is None else out
    bf = torch.bfloat16
    _check("forge_linear_swiglu", load().forge_linear_swiglu(
        _dev(x, bf, "x"), _dev(w_gate, bf, "w_gate"), _dev(w_up, bf, "w_up"), _dev(out, bf, "out"),
        M, N, K, int(w_layout), _stream()))
    return out


# ---- the serving step around the KV cache ----
DTYPE_BF16, DTYPE_F16, DTYPE_F32 = range(3)
KV_BF16, KV_F16, KV_INT8, KV_E4M3 = range(4)
ROTARY_HALF, ROTARY_INTERLEAVED = range(2)
(ROTARY_SCALE_NONE, ROTARY_SCALE_LINEAR, ROTARY_SCALE_BASE, ROTARY_SCALE_RAMP_ROTATIONS, ROTARY_SCALE_RAMP_WAVELENGTH) = range(5)
_DTYPES = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16, torch.float32: DTYPE_F32}
_KV_TYPES = (torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn)


def _find_current_device():
    return getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_current_device = _find_current_device()


def _on_current(*tensors) -> None:
    """The library launches on the current device: a tensor of another one is refused."""
    dev = _current_device()
    for t in tensors:
        if t is not None and t.device.index != dev:
            raise ValueError(f"tensors on the current device (cuda:{dev}) expected, got one on {t.device}")


def _dev_or_none(t, dtype, name: str, shape):
    if t is None:
        return None
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: shape {list(shape)} expected")
    return _dev(t, dtype, name)


def _view(t: torch.Tensor, dtype, name: str, shape):
    """Address and {batch, head, token} strides of a [B, H, S, D] view with contiguous rows; a dimension of size 1 has no
    stride of its own and gets one that the library takes."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 4 and tuple(t.shape) == tuple(shape)):
        raise ValueError(f"{name}: expected a CUDA tensor {list(shape)} of {dtype}")
    B, H, S, D = shape
    st = t.stride()
    if st[3] != 1 and D != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), _i64x3(st[0] if B > 1 else 8, st[1] if H > 1 else 8, st[2] if S > 1 else 8)


def rotary_frequencies(dims, base=10000.0, scaling=None):
    """forge_rotary_frequencies: (inverse frequencies as an fp32 host tensor [dims / 2], amplitude); scaling: a RotaryScaling."""
    inv_freq = torch.empty((max(int(dims), 2) // 2,), dtype=torch.float32)
    amplitude = ctypes.c_float(1.0)
    _check("forge_rotary_frequencies", load().forge_rotary_frequencies(
        int(dims), float(base), None if scaling is None else ctypes.byref(scaling), inv_freq.data_ptr(), ctypes.byref(amplitude)))
    return inv_freq, amplitude.value


class Rotary:
    """forge_rotary: inv_freq, an fp32 CUDA tensor [dims / 2] (kept), the layout of the pairs and the amplitude."""

    def __init__(self, inv_freq, layout=ROTARY_HALF, amplitude=1.0):
        if inv_freq.dim() != 1:
            raise ValueError("inv_freq [dims / 2] expected")
        self.inv_freq = inv_freq
        self.desc = RotaryDesc(inv_freq=_dev(inv_freq, torch.float32, "inv_freq"), dims=2 * inv_freq.numel(), layout=int(layout),
                               amplitude=float(amplitude))
        self.address, self.device = ctypes.addressof(self.desc), inv_freq.device.index


class KVCache:
    """forge_kv_cache: k, v [B, Hkv, Smax, D] in bf16, fp16, int8 or float8_e4m3fn; 8-bit ones with k_scale, v_scale
    [B, Hkv, Smax] in fp32.  The tensors are kept and belong to the caller."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4 or tuple(v.shape) != tuple(k.shape):
            raise ValueError("k, v [B,Hkv,Smax,D] expected")
        if k.dtype not in _KV_TYPES:
            raise ValueError(f"k: expected one of {_KV_TYPES}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.format = _KV_TYPES.index(k.dtype)
        self.B, self.Hkv, self.Smax, self.D = k.shape
        eight = self.format in (KV_INT8, KV_E4M3)
        if eight != (k_scale is not None) or eight != (v_scale is not None):
            raise ValueError("k_scale and v_scale [B,Hkv,Smax] belong to 8-bit caches, and to no others")
        kp, vp = _dev(k, k.dtype, "k"), _dev(v, k.dtype, "v")
        shape = (self.B, self.Hkv, self.Smax)
        self.desc = KVCacheDesc(k=kp, v=vp, k_scale=_dev_or_none(k_scale, torch.float32, "k_scale", shape),
                                v_scale=_dev_or_none(v_scale, torch.float32, "v_scale", shape),
                                B=self.B, Hkv=self.Hkv, Smax=self.Smax, D=self.D, format=self.format)
        if len({t.device for t in (k, v, k_scale, v_scale) if t is not None}) != 1:
            raise ValueError("the tensors of a cache must be on one device")
        self.address, self.device = ctypes.addressof(self.desc), k.device.index

    @classmethod
    def empty(cls, B, Hkv, Smax, D, format=KV_BF16, device="cuda"):
        """A new cache (of zeros: 8-bit rows that were never written stand for zeros)."""
        kv = [torch.zeros((B, Hkv, Smax, D), dtype=_KV_TYPES[format], device=device) for _ in range(2)]
        scales = [torch.zeros((B, Hkv, Smax), dtype=torch.float32, device=device) for _ in range(2)] if format in (KV_INT8, KV_E4M3) else []
        return cls(*kv, *scales)


def rotary_apply(x, rotary, positions=None, first=None, inverse=False, out=None):
    """forge_rotary_apply: x [B,H,S,D] view (bf16, fp16 or fp32) rotated at positions int32 [B,S], or first int32 [B] + s, or s;
    inverse: rotated back.  out may be x itself."""
    if _host_calls is not None:
        st = _host_calls.rotary(x, rotary.address, rotary.device, positions, first, 1 if inverse else 0, out)
        if st >= 0:
            _check("forge_rotary_apply", st)
            return out
    B, H, S, D = x.shape
    if x.dtype not in _DTYPES:
        raise ValueError("x: bf16, fp16 or fp32 expected")
    out = torch.empty_like(x) if out is None else out
    xp, xs = _view(x, x.dtype, "x", (B, H, S, D))
    op, os_ = _view(out, x.dtype, "out", (B, H, S, D))
    pp, fp = _dev_or_none(positions, torch.int32, "positions", (B, S)), _dev_or_none(first, torch.int32, "first", (B,))
    _on_current(x, out, rotary.inv_freq, positions, first)
    _check("forge_rotary_apply", load().forge_rotary_apply(
        xp, op, _DTYPES[x.dtype], B, H, S, D, xs, os_, pp, fp, rotary.desc, int(bool(inverse)), _stream()))
    return out


def kv_append(cache, k, v, lens, counts=None, positions=None, rows=None, rotary=None, q=None, q_out=None):
    """forge_kv_append: k, v [B,Hkv,S,D] views (bf16 or fp16) become rows lens[b] .. of the cache, k rotated first if `rotary` is
    given; q [B,Hq,S,D] is rotated into q_out in the same launch.  counts int32 [B]: how many tokens of each sequence; positions
    int32 [B,S]; rows int32 [B,n]: which tokens of k and v, and in which order.  Returns q_out (None without q)."""
    if _host_calls is not None:
        st = _host_calls.append(cache.address, cache.device, k, v, lens, counts, positions, rows, None if rotary is None else rotary.address,
                                None if rotary is None else rotary.device, q, q_out)
        if st >= 0:
            _check("forge_kv_append", st)
            return q_out
    B, H, S_src, D = k.shape
    if (B, H, D) != (cache.B, cache.Hkv, cache.D):
        raise ValueError("k, v [B,Hkv,S,D] of the cache's B, Hkv and D expected")
    if k.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("k: bf16 or fp16 expected")
    if rows is not None and rows.dim() != 2:
        raise ValueError("rows [B,n] expected")
    S = S_src if rows is None else rows.shape[1]
    d = KVAppendDesc(dtype=_DTYPES[k.dtype], S=S, S_src=S_src)
    d.k, ks = _view(k, k.dtype, "k", (B, H, S_src, D))
    d.v, vs = _view(v, k.dtype, "v", (B, H, S_src, D))
    d.k_strides, d.v_strides = ks, vs
    if q is not None:
        q_out = torch.empty_like(q) if q_out is None else q_out
        d.Hq = q.shape[1]
        d.q, qs = _view(q, k.dtype, "q", (B, d.Hq, S, D))
        d.q_out, qos = _view(q_out, k.dtype, "q_out", (B, d.Hq, S, D))
        d.q_strides, d.q_out_strides = qs, qos
    elif q_out is not None:
        raise ValueError("q_out without q")
    d.lens = _dev_or_none(lens, torch.int32, "lens", (B,))
    d.counts = _dev_or_none(counts, torch.int32, "counts", (B,))
    d.positions = _dev_or_none(positions, torch.int32, "positions", (B, S_src))
    d.rows = _dev_or_none(rows, torch.int32, "rows", (B, S))
    if rotary is not None:
        d.rotary = ctypes.pointer(rotary.desc)
    _on_current(cache.k, k, v, q, q_out, lens, counts, positions, rows, None if rotary is None else rotary.inv_freq)
    _check("forge_kv_append", load().forge_kv_append(cache.desc, d, _stream()))
    return q_out


def kv_read(cache, k_out, v_out, first=None, counts=None):
    """forge_kv_read: rows first[b] + i (first int32 [B] or None: 0) of the cache, for i < counts[b] (None: all), into
    k_out, v_out [B,Hkv,S,D] views (bf16 or fp16); other rows of these are left as they were.  Returns (k_out, v_out)."""
    if _host_calls is not None:
        st = _host_calls.read(cache.address, cache.device, k_out, v_out, first, counts)
        if st >= 0:
            _check("forge_kv_read", st)
            return k_out, v_out
    if k_out.dim() != 4 or k_out.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("k_out [B,Hkv,S,D] in bf16 or fp16 expected")
    shape = (cache.B, cache.Hkv, k_out.shape[2], cache.D)
    kp, ks = _view(k_out, k_out.dtype, "k_out", shape)
    vp, vs = _view(v_out, k_out.dtype, "v_out", shape)
    fp, cp = _dev_or_none(first, torch.int32, "first", (cache.B,)), _dev_or_none(counts, torch.int32, "counts", (cache.B,))
    _on_current(cache.k, k_out, v_out, first, counts)
    _check("forge_kv_read", load().forge_kv_read(cache.desc, kp, vp, _DTYPES[k_out.dtype], shape[2], ks, vs, fp, cp, _stream()))
    return k_out, v_out


def attn_kv_workspace_bytes(B, Hq, Hkv, T=1, D=128) -> int:
    return int(load().forge_attn_kv_workspace_bytes(B, Hq, Hkv, T, D))


def attn_kv_workspace_init(workspace) -> None:
    """forge_attn_kv_workspace_init: clears a new workspace (its arrival counters must start at zero)."""
    _check("forge_attn_kv_workspace_init", load().forge_attn_kv_workspace_init(
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))


def _kv_workspace(workspace, cache, Hq, T, device):
    if workspace is None:
        need = attn_kv_workspace_bytes(cache.B, Hq, cache.Hkv, T, cache.D)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        attn_kv_workspace_init(workspace)
    return workspace


def attn_decode_kv(q, cache, lens, scale=None, out=None, workspace=None):
    """forge_attn_decode_kv: q [B,Hq,D] (bf16 or fp16) over the first lens[b] rows of a KVCache.  A workspace passed in must have
    been cleared once (attn_kv_workspace_init) and may serve calls of any shapes, one after the other; without one, a fresh cleared
    workspace is allocated."""
    if _host_calls is not None:
        st = _host_calls.decode_kv(cache.address, cache.device, q, lens, scale, out, workspace)
        if st >= 0:
            _check("forge_attn_decode_kv", st)
            return out
    B, Hq, D = q.shape
    if (B, D) != (cache.B, cache.D):
        raise ValueError("q [B,Hq,D] of the cache's B and D expected")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("q: bf16 or fp16 expected")
    out = torch.empty_like(q) if out is None else out
    if tuple(out.shape) != tuple(q.shape):
        raise ValueError("out: the shape of q expected")
    qp, op, lp = _dev(q, q.dtype, "q"), _dev(out, q.dtype, "out"), _dev_or_none(lens, torch.int32, "lens", (B,))
    _on_current(cache.k, q, out, lens, workspace)
    workspace = _kv_workspace(workspace, cache, Hq, 1, q.device)
    _check("forge_attn_decode_kv", load().forge_attn_decode_kv(
        cache.desc, qp, op, _DTYPES[q.dtype], Hq, lp, float(D ** -0.5 if scale is None else scale),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


def attn_tree(q, cache, lens, tree=None, scale=None, out=None, workspace=None):
    """forge_attn_tree: q [B,Hq,T,D] view (bf16 or fp16), T tokens whose own rows are rows lens[b] .. lens[b] + T - 1 of the cache; tree
    int64 [B or 1, T]: bit u of tree[b, t] says whether token t sees token u (None: those up to itself).  Workspace as in
    attn_decode_kv."""
    if _host_calls is not None:
        st = _host_calls.tree(cache.address, cache.device, q, lens, tree, scale, out, workspace)
        if st >= 0:
            _check("forge_attn_tree", st)
            return out
    B, Hq, T, D = q.shape
    if (B, D) != (cache.B, cache.D):
        raise ValueError("q [B,Hq,T,D] of the cache's B and D expected")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("q: bf16 or fp16 expected")
    if tree is not None and (tree.dim() != 2 or tree.shape[0] not in (1, B)):
        raise ValueError("tree [B or 1, T] expected")
    out = torch.empty_like(q) if out is None else out
    qp, qs = _view(q, q.dtype, "q", (B, Hq, T, D))
    op, os_ = _view(out, q.dtype, "out", (B, Hq, T, D))
    tree_B = 1 if tree is None else tree.shape[0]
    lp, tp = _dev_or_none(lens, torch.int32, "lens", (B,)), _dev_or_none(tree, torch.int64, "tree", (tree_B, T))
    _on_current(cache.k, q, out, lens, tree, workspace)
    workspace = _kv_workspace(workspace, cache, Hq, T, q.device)
    _check("forge_attn_tree", load().forge_attn_tree(
        cache.desc, qp, op, _DTYPES[q.dtype], Hq, T, qs, os_, lp, tp, tree_B, float(D ** -0.5 if scale is None else scale),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


# ---- a step of many requests: a KV cache in pages, adapters of their own ----
class KVPages:
    """forge_kv_pages: k, v [num_pages, Hkv, page_size, D] in bf16, fp16, int8 or float8_e4m3fn; 8-bit ones with k_scale, v_scale
    [num_pages, Hkv, page_size] in fp32.  The tensors are kept and belong to the caller."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4 or tuple(v.shape) != tuple(k.shape):
            raise ValueError("k, v [num_pages,Hkv,page_size,D] expected")
        if k.dtype not in _KV_TYPES:
            raise ValueError(f"k: expected one of {_KV_TYPES}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.format = _KV_TYPES.index(k.dtype)
        self.num_pages, self.Hkv, self.page_size, self.D = k.shape
        eight = self.format in (KV_INT8, KV_E4M3)
        if eight != (k_scale is not None) or eight != (v_scale is not None):
            raise ValueError("k_scale and v_scale [num_pages,Hkv,page_size] belong to 8-bit caches, and to no others")
        kp, vp = _dev(k, k.dtype, "k"), _dev(v, k.dtype, "v")
        shape = (self.num_pages, self.Hkv, self.page_size)
        self.desc = KVPagesDesc(k=kp, v=vp, k_scale=_dev_or_none(k_scale, torch.float32, "k_scale", shape),
                                v_scale=_dev_or_none(v_scale, torch.float32, "v_scale", shape),
                                num_pages=self.num_pages, Hkv=self.Hkv, page_size=self.page_size, D=self.D, format=self.format)
        if len({t.device for t in (k, v, k_scale, v_scale) if t is not None}) != 1:
            raise ValueError("the tensors of a cache must be on one device")
        self.address, self.device = ctypes.addressof(self.desc), k.device.index

    @classmethod
    def empty(cls, num_pages, Hkv, page_size, D, format=KV_BF16, device="cuda"):
        """A new cache (of zeros: 8-bit rows that were never written stand for zeros)."""
        kv = [torch.zeros((num_pages, Hkv, page_size, D), dtype=_KV_TYPES[format], device=device) for _ in range(2)]
        scales = [torch.zeros((num_pages, Hkv, page_size), dtype=torch.float32, device=device) for _ in range(2)] if format in (KV_INT8, KV_E4M3) else []
        return cls(*kv, *scales)


class PageTables:
    """forge_kv_page_tables: table int32 [B, max_pages], free_pages int32 [num_pages], free_count int32 [1].  The tensors are kept and belong
    to the caller."""

    def __init__(self, table, free_pages, free_count, page_size):
        if table.dim() != 2 or free_pages.dim() != 1 or tuple(free_count.shape) != (1,):
            raise ValueError("table [B,max_pages], free_pages [num_pages] and free_count [1] expected")
        self.table, self.free_pages, self.free_count, self.page_size = table, free_pages, free_count, int(page_size)
        self.B, self.max_pages = table.shape
        self.desc = PageTablesDesc(table=_dev(table, torch.int32, "table"), free_pages=_dev(free_pages, torch.int32, "free_pages"),
                                   free_count=_dev(free_count, torch.int32, "free_count"), B=self.B, max_pages=self.max_pages,
                                   page_size=self.page_size, num_pages=free_pages.numel())
        if len({t.device for t in (table, free_pages, free_count)}) != 1:
            raise ValueError("the tensors of the tables must be on one device")
        self.address, self.device = ctypes.addressof(self.desc), table.device.index

    @classmethod
    def empty(cls, B, max_pages, num_pages, page_size, device="cuda"):
        """Tables of no pages (-1), all of num_pages free; page 0 is handed out first."""
        free = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device)
        count = torch.full((1,), num_pages, dtype=torch.int32, device=device)
        return cls(torch.full((B, max_pages), -1, dtype=torch.int32, device=device), free, count, page_size)


class PageSlots:
    """What assign_pages says of a step: lens int32 [B], starts [B + 1], slots, positions and requests [T] (starts, positions and
    requests may be None).  The tensors are kept."""

    def __init__(self, lens, starts, slots, positions=None, requests=None):
        B, T = lens.numel(), slots.numel()
        self.lens, self.starts, self.slots, self.positions, self.requests, self.B, self.T = lens, starts, slots, positions, requests, B, T
        i32 = torch.int32
        self.desc = PageSlotsDesc(new_lens=_dev_or_none(lens, i32, "lens", (B,)), starts=_dev_or_none(starts, i32, "starts", (B + 1,)),
                                  slots=_dev_or_none(slots, i32, "slots", (T,)), positions=_dev_or_none(positions, i32, "positions", (T,)),
                                  requests=_dev_or_none(requests, i32, "requests", (T,)), T=T)
        if len({t.device for t in (lens, starts, slots, positions, requests) if t is not None}) != 1:
            raise ValueError("the tensors of a step must be on one device")
        self.address, self.device = ctypes.addressof(self.desc), lens.device.index

    @classmethod
    def empty(cls, B, T, device="cuda"):
        return cls(*(torch.zeros(n, dtype=torch.int32, device=device) for n in (B, B + 1, T, T, T)))


def assign_pages(tables, lens, out, counts=None, free_left=None):
    """forge_kv_assign_pages: room for counts[b] (int32 [B]; None: one) more rows behind the lens[b] (int32 [B]) rows of each request.  What
    they got goes into `out`, a PageSlots whose T is the tokens that there is room for; out.lens may be lens.  free_left int32 [1]: where the
    number of pages left goes (None: into tables.free_count).  Returns out."""
    if _host_calls is not None:
        st = _host_calls.assign_pages(tables.address, tables.device, lens, counts, out.address, out.device, out.B, free_left)
        if st >= 0:
            _check("forge_kv_assign_pages", st)
            return out
    if out.B != tables.B:
        raise ValueError("out: a PageSlots of the tables' B expected")
    i32 = torch.int32
    lp, cp = _dev_or_none(lens, i32, "lens", (tables.B,)), _dev_or_none(counts, i32, "counts", (tables.B,))
    fp = _dev_or_none(free_left, i32, "free_left", (1,))
    _on_current(tables.table, out.lens, lens, counts, free_left)
    _check("forge_kv_assign_pages", load().forge_kv_assign_pages(tables.desc, lp, cp, out.desc, fp, _stream()))
    return out


def release_pages(tables, lens, done, free_left=None):
    """forge_kv_release_pages: the pages of the first lens[b] rows of requests with done[b] != 0 (int32 [B]) are free again."""
    i32 = torch.int32
    lp, dp = _dev_or_none(lens, i32, "lens", (tables.B,)), _dev_or_none(done, i32, "done", (tables.B,))
    fp = _dev_or_none(free_left, i32, "free_left", (1,))
    _on_current(tables.table, lens, done, free_left)
    _check("forge_kv_release_pages", load().forge_kv_release_pages(tables.desc, lp, dp, fp, _stream()))


def _token_view(t: torch.Tensor, dtype, name: str, shape):
    """Address and {token, head} strides of a [T, H, D] view with contiguous rows."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 3 and tuple(t.shape) == tuple(shape)):
        raise ValueError(f"{name}: expected a CUDA tensor {list(shape)} of {dtype}")
    T, H, D = shape
    st = t.stride()
    if st[2] != 1 and D != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), (ctypes.c_int64 * 2)(st[0] if T > 1 else 8, st[1] if H > 1 else 8)


def kv_append_pages(cache, k, v, slots, positions=None, rotary=None, q=None, q_out=None):
    """forge_kv_append_pages: k, v [T,Hkv,D] views (bf16 or fp16) of packed tokens become rows slots[t] (int32 [T]) of a KVPages, k rotated
    first by positions[t] (int32 [T]) if `rotary` is given; q [T,Hq,D] is rotated into q_out in the same launch.  Returns q_out
    (None without q)."""
    if _host_calls is not None:
        st = _host_calls.append_pages(cache.address, cache.device, k, v, slots, positions, None if rotary is None else rotary.address,
                                      None if rotary is None else rotary.device, q, q_out)
        if st >= 0:
            _check("forge_kv_append_pages", st)
            return q_out
    if k.dim() != 3 or k.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("k [T,Hkv,D] in bf16 or fp16 expected")
    T, H, D = k.shape
    if (H, D) != (cache.Hkv, cache.D):
        raise ValueError("k, v [T,Hkv,D] of the cache's Hkv and D expected")
    d = KVAppendPagesDesc(dtype=_DTYPES[k.dtype], T=T)
    d.k, ks = _token_view(k, k.dtype, "k", (T, H, D))
    d.v, vs = _token_view(v, k.dtype, "v", (T, H, D))
    d.k_strides, d.v_strides = ks, vs
    if q is not None:
        q_out = torch.empty_like(q) if q_out is None else q_out
        d.Hq = q.shape[1]
        d.q, qs = _token_view(q, k.dtype, "q", (T, d.Hq, D))
        d.q_out, qos = _token_view(q_out, k.dtype, "q_out", (T, d.Hq, D))
        d.q_strides, d.q_out_strides = qs, qos
    elif q_out is not None:
        raise ValueError("q_out without q")
    d.slots = _dev_or_none(slots, torch.int32, "slots", (T,))
    d.positions = _dev_or_none(positions, torch.int32, "positions", (T,))
    if rotary is not None:
        d.rotary = ctypes.pointer(rotary.desc)
    _on_current(cache.k, k, v, q, q_out, slots, positions, None if rotary is None else rotary.inv_freq)
    _check("forge_kv_append_pages", load().forge_kv_append_pages(cache.desc, d, _stream()))
    return q_out


def _table(table):
    if table.dim() != 2:
        raise ValueError("table [B,max_pages] expected")
    return _dev(table, torch.int32, "table"), table.shape[0], table.shape[1]


def kv_read_pages(cache, table, k_out, v_out, first=None, counts=None):
    """forge_kv_read_pages: kv_read of a KVPages through table int32 [B,max_pages]."""
    if _host_calls is not None:
        st = _host_calls.read_pages(cache.address, cache.device, table, k_out, v_out, first, counts)
        if st >= 0:
            _check("forge_kv_read_pages", st)
            return k_out, v_out
    tp, B, max_pages = _table(table)
    if k_out.dim() != 4 or k_out.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("k_out [B,Hkv,S,D] in bf16 or fp16 expected")
    shape = (B, cache.Hkv, k_out.shape[2], cache.D)
    kp, ks = _view(k_out, k_out.dtype, "k_out", shape)
    vp, vs = _view(v_out, k_out.dtype, "v_out", shape)
    fp, cp = _dev_or_none(first, torch.int32, "first", (B,)), _dev_or_none(counts, torch.int32, "counts", (B,))
    _on_current(cache.k, table, k_out, v_out, first, counts)
    _check("forge_kv_read_pages", load().forge_kv_read_pages(cache.desc, tp, B, max_pages, kp, vp, _DTYPES[k_out.dtype], shape[2], ks, vs, fp, cp,
                                                             _stream()))
    return k_out, v_out


def _pages_workspace(workspace, cache, B, Hq, T, device):
    if workspace is None:
        workspace = torch.empty(max(attn_kv_workspace_bytes(B, Hq, cache.Hkv, T, cache.D), 16), dtype=torch.uint8, device=device)
        attn_kv_workspace_init(workspace)
    return workspace


def attn_decode_pages(q, cache, table, lens, scale=None, out=None, workspace=None):
    """forge_attn_decode_pages: attn_decode_kv over a KVPages, the rows of request b in the pages of table[b] (int32 [B,max_pages])."""
    if _host_calls is not None:
        st = _host_calls.decode_pages(cache.address, cache.device, q, table, lens, scale, out, workspace)
        if st >= 0:
            _check("forge_attn_decode_pages", st)
            return out
    tp, B, max_pages = _table(table)
    if q.dim() != 3 or (q.shape[0], q.shape[2]) != (B, cache.D):
        raise ValueError("q [B,Hq,D] of the table's B and the cache's D expected")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("q: bf16 or fp16 expected")
    Hq, D = q.shape[1:]
    out = torch.empty_like(q) if out is None else out
    if tuple(out.shape) != tuple(q.shape):
        raise ValueError("out: the shape of q expected")
    qp, op, lp = _dev(q, q.dtype, "q"), _dev(out, q.dtype, "out"), _dev_or_none(lens, torch.int32, "lens", (B,))
    _on_current(cache.k, table, q, out, lens, workspace)
    workspace = _pages_workspace(workspace, cache, B, Hq, 1, q.device)
    _check("forge_attn_decode_pages", load().forge_attn_decode_pages(
        cache.desc, tp, B, max_pages, qp, op, _DTYPES[q.dtype], Hq, lp, float(D ** -0.5 if scale is None else scale),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


def attn_tree_pages(q, cache, table, lens, tree=None, scale=None, out=None, workspace=None):
    """forge_attn_tree_pages: attn_tree over a KVPages, the rows of request b in the pages of table[b] (int32 [B,max_pages])."""
    if _host_calls is not None:
        st = _host_calls.tree_pages(cache.address, cache.device, q, table, lens, tree, scale, out, workspace)
        if st >= 0:
            _check("forge_attn_tree_pages", st)
            return out
    tp, B, max_pages = _table(table)
    if q.dim() != 4 or (q.shape[0], q.shape[3]) != (B, cache.D):
        raise ValueError("q [B,Hq,T,D] of the table's B and the cache's D expected")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("q: bf16 or fp16 expected")
    _, Hq, T, D = q.shape
    if tree is not None and (tree.dim() != 2 or tree.shape[0] not in (1, B)):
        raise ValueError("tree [B or 1, T] expected")
    out = torch.empty_like(q) if out is None else out
    qp, qs = _view(q, q.dtype, "q", (B, Hq, T, D))
    op, os_ = _view(out, q.dtype, "out", (B, Hq, T, D))
    tree_B = 1 if tree is None else tree.shape[0]
    lp, trp = _dev_or_none(lens, torch.int32, "lens", (B,)), _dev_or_none(tree, torch.int64, "tree", (tree_B, T))
    _on_current(cache.k, table, q, out, lens, tree, workspace)
    workspace = _pages_workspace(workspace, cache, B, Hq, T, q.device)
    _check("forge_attn_tree_pages", load().forge_attn_tree_pages(
        cache.desc, tp, B, max_pages, qp, op, _DTYPES[q.dtype], Hq, T, qs, os_, lp, trp, tree_B, float(D ** -0.5 if scale is None else scale),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


def _rows(t: torch.Tensor, dtype, name: str, shape):
    """Address and row stride of a [T, n] view with contiguous rows."""
    if not (t.is_cuda and t.dtype == dtype and tuple(t.shape) == tuple(shape)):
        raise ValueError(f"{name}: expected a CUDA tensor {list(shape)} of {dtype}")
    if t.stride(1) != 1 and shape[1] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if shape[0] > 1 and t.stride(0) < shape[1]:  # 0, of a broadcast row, would say dense
        raise ValueError(f"{name}: rows that do not overlap expected")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else 0


def linear_adapters_workspace_bytes(T, rank) -> int:
    return int(load().forge_linear_adapters_workspace_bytes(T, rank))


def linear_adapters(x, y, a, b, adapters, requests=None, scales=None, out=None, workspace=None):
    """forge_linear_adapters: y + scales[i] * (x A_i^T) B_i^T with i = adapters[requests[t]] (requests None: adapters[t]); x [T,K] and
    y, out [T,N] views with contiguous rows that do not overlap, a [n,rank,K], b [n,N,rank], all bf16 or fp16; adapters int32 [R], requests int32 [T], scales
    fp32 [n] or None.  Tokens without an adapter (-1) keep y.  out may be y itself.  workspace: uint8, of any contents; without one,
    a fresh one is allocated where the call needs it."""
    if _host_calls is not None:
        st = _host_calls.adapters(x, y, a, b, adapters, requests, scales, out, workspace)
        if st >= 0:
            _check("forge_linear_adapters", st)
            return out
    if x.dim() != 2 or y.dim() != 2 or a.dim() != 3 or b.dim() != 3 or adapters.dim() != 1:
        raise ValueError("x [T,K], y [T,N], a [n,rank,K], b [n,N,rank], adapters [R] expected")
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("x: bf16 or fp16 expected")
    (T, K), N, (n, rank) = x.shape, y.shape[1], a.shape[:2]
    if tuple(a.shape) != (n, rank, K) or tuple(b.shape) != (n, N, rank):
        raise ValueError("a [n,rank,K], b [n,N,rank] expected")
    out = torch.empty((T, N), dtype=x.dtype, device=x.device) if out is None else out
    t = x.dtype
    xp, xs = _rows(x, t, "x", (T, K))
    yp, ys = _rows(y, t, "y", (T, N))
    op, os_ = _rows(out, t, "out", (T, N))
    R = adapters.shape[0]
    if requests is None and R != T:
        raise ValueError("adapters [T] expected without requests")
    d = AdaptersDesc(a=_dev(a, t, "a"), b=_dev(b, t, "b"), scales=_dev_or_none(scales, torch.float32, "scales", (n,)), n=n, rank=rank, K=K, N=N,
                     dtype=_DTYPES[t])
    rp, ap = _dev_or_none(requests, torch.int32, "requests", (T,)), _dev(adapters, torch.int32, "adapters")
    _on_current(x, y, out, a, b, scales, requests, adapters, workspace)
    if workspace is None:
        need = linear_adapters_workspace_bytes(T, rank)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    wp, wn = (None, 0) if workspace is None else (_dev(workspace, torch.uint8, "workspace"), workspace.numel())
    _check("forge_linear_adapters", load().forge_linear_adapters(d, xp, yp, op, T, xs, ys, os_, rp, ap, R, wp, wn, _stream()))
    return out


# ---- buffer planning (host only) and the decoder layer ----
MLP_SWIGLU, MLP_GELU = 0, 1


def plan_liveness(out_reg, in_regs_per_op, num_regs):
    """forge_plan_liveness: ops given as (register written or -1, list of registers read).  Returns (start, end)."""
    n = len(out_reg)
    off = [0]
    flat = []
    for regs in in_regs_per_op:
        flat.extend(regs)
        off.append(len(flat))
    c_out = (ctypes.c_int * max(n, 1))(*out_reg)
    c_off = (ctypes.c_int * (n + 1))(*off)
    c_in = (ctypes.c_int * max(len(flat), 1))(*flat)
    start = (ctypes.c_int * max(num_regs, 1))()
    end = (ctypes.c_int * max(num_regs, 1))()
    _check("forge_plan_liveness", load().forge_plan_liveness(n, c_out, c_off, c_in, num_regs, start, end))
    return list(start)[:num_regs], list(end)[:num_regs]


def plan_linear_scan(start, end, nbytes=None, pinned=None):
    """forge_plan_linear_scan.  Returns (buf_of, buf_bytes, num_bufs)."""
    n = len(start)
    c_s = (ctypes.c_int * max(n, 1))(*start)
    c_e = (ctypes.c_int * max(n, 1))(*end)
    c_b = None if nbytes is None else (ctypes.c_size_t * max(n, 1))(*nbytes)
    c_p = None if pinned is None else (ctypes.c_ubyte * max(n, 1))(*[1 if x else 0 for x in pinned])
    buf_of = (ctypes.c_int * max(n, 1))()
    buf_bytes = (ctypes.c_size_t * max(n, 1))()
    m = ctypes.c_int(0)
    _check("forge_plan_linear_scan", load().forge_plan_linear_scan(n, c_s, c_e, c_b, c_p, buf_of, buf_bytes, ctypes.byref(m)))
    return list(buf_of)[:n], list(buf_bytes)[:m.value], m.value


def _layer_desc(B, S, Hq, Hkv, D, F, mlp_kind, w_layout, mask_kind, scale, lens, weights):
    d = LayerDesc(B=B, S=S, Hq=Hq, Hkv=Hkv, D=D, F=F, mlp_kind=mlp_kind, w_layout=w_layout, mask_kind=mask_kind,
                  scale=float(scale), lens=None if lens is None else _dev(lens, torch.int32, "lens"))
    for name in ("w_qkv", "b_qkv", "w_o", "b_o", "w_gate", "w_up", "b_up", "w_down", "b_down"):
        t = weights.get(name)
        setattr(d, name, None if t is None else _dev(t, torch.bfloat16, name))
    return d


def decoder_layer_plan(B, S, Hq, Hkv, D, F, mlp_kind=MLP_SWIGLU):
    """forge_decoder_layer_plan: the buffer plan of a layer of these dimensions (no GPU needed)."""
    d = LayerDesc(B=B, S=S, Hq=Hq, Hkv=Hkv, D=D, F=F, mlp_kind=mlp_kind, w_layout=W_KN, mask_kind=MASK_CAUSAL, scale=1.0)
    plan = LayerPlan()
    _check("forge_decoder_layer_plan", load().forge_decoder_layer_plan(ctypes.byref(d), ctypes.byref(plan)))
    return plan


def decoder_layer(x, weights, B, S, Hq, Hkv, D, F, mlp_kind=MLP_SWIGLU, w_layout=W_KN, mask_kind=MASK_CAUSAL,
                  scale=None, lens=None, out=None, workspace=None):
    """forge_decoder_layer: x [B*S, Hq*D] bf16; weights: dict of bf16 tensors (w_qkv, w_o, w_gate, w_up, w_down
    and optional b_qkv, b_o, b_up, b_down)."""
    scale = D ** -0.5 if scale is None else scale
    d = _layer_desc(B, S, Hq, Hkv, D, F, mlp_kind, w_layout, mask_kind, scale, lens, weights)
    out = torch.empty_like(x) if out is None else out
    if workspace is None:
        need = int(load().forge_decoder_layer_workspace_bytes(ctypes.byref(d)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    _check("forge_decoder_layer", load().forge_decoder_layer(
        ctypes.byref(d), _dev(x, torch.bfloat16, "x"), _dev(out, torch.bfloat16, "out"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()))
    return out


# ---- host-buffer variants: tensors in (pinned) host memory, device scratch from the caller ----
def attn_host_scratch_bytes(B, Hq, Hkv, Sq, Skv, D, elem_bytes) -> int:
    return int(load().forge_attn_host_scratch_bytes(B, Hq, Hkv, Sq, Skv, D, elem_bytes))


def attn_fused_host(q, k, v, out, scratch, mask_kind=MASK_NONE, lens=None, scale=None):
    """forge_attn_fused_host / forge_attn_fused_f32_host, chosen by q.dtype.  Asynchronous."""
    B, Hq, Hkv, Sq, Skv, D = _attn_dims(q, k, v)
    f32 = q.dtype == torch.float32
    dt = torch.float32 if f32 else torch.bfloat16
    scale = D ** -0.5 if scale is None else scale
    lp = None if lens is None else _host(lens, torch.int32, "lens")
    fn = "forge_attn_fused_f32_host" if f32 else "forge_attn_fused_host"
    _check(fn, getattr(load(), fn)(
        _host(q, dt, "q"), _host(k, dt, "k"), _host(v, dt, "v"), _host(out, dt, "out"),
        B, Hq, Hkv, Sq, Skv, D, int(mask_kind), lp, float(scale),
        _dev(scratch, torch.uint8, "scratch"), scratch.numel(), _stream()))
    return out


def attn_decode_host_scratch_bytes(B, Hq, Hkv, Smax, D, num_splits) -> int:
    return int(load().forge_attn_decode_host_scratch_bytes(B, Hq, Hkv, Smax, D, num_splits))


def attn_decode_splitkv_host(q, k_cache, v_cache, lens, num_splits, out, scratch, scale=None):
    B, Hq, D = q.shape
    _, Hkv, Smax, _ = k_cache.shape
    scale = D ** -0.5 if scale is None else scale
    bf = torch.bfloat16
    _check("forge_attn_decode_splitkv_host", load().forge_attn_decode_splitkv_host(
        _host(q, bf, "q"), _host(k_cache, bf, "k_cache"), _host(v_cache, bf, "v_cache"), _host(out, bf, "out"),
        B, Hq, Hkv, Smax, D, _host(lens, torch.int32, "lens"), int(num_splits), float(scale),
        _dev(scratch, torch.uint8, "scratch"), scratch.numel(), _stream()))
    return out


def linear_host_scratch_bytes(M, N, K) -> int:
    return int(load().forge_linear_host_scratch_bytes(M, N, K))


def linear_bias_gelu_host(x, w, b, out, scratch):
    M, K = x.shape
    _, N = w.shape
    bf = torch.bfloat16
    _check("forge_linear_bias_gelu_host", load().forge_linear_bias_gelu_host(
        _host(x, bf, "x"), _host(w, bf, "w"), _host(b, bf, "b"), _host(out, bf, "out"), M, N, K,
        _dev(scratch, torch.uint8, "scratch"), scratch.numel(), _stream()))
    return out


def activation_f32(x, act, exact=False, out=None):
    """forge_activation_f32: the fused linear's epilogue activation, element-wise on an fp32 CUDA tensor."""
    out = torch.empty_like(x) if out is None else out
    _check("forge_activation_f32", load().forge_activation_f32(
        _dev(x, torch.float32, "x"), _dev(out, torch.float32, "out"), x.numel(), int(act), int(bool(exact)), _stream()))
    return out


def debug_wait_timeout(budget_clocks: int = 1_000_000) -> None:
    """forge_debug_wait_timeout: one warp runs the kernels' bounded wait on a barrier nothing completes."""
    _check("forge_debug_wait_timeout", load().forge_debug_wait_timeout(int(budget_clocks), _stream()))


def check_status() -> None:
    """Synchronises the current stream and raises if a kernel gave up on a bounded wait."""
    _check("forge_check_status", load().forge_check_status(_stream()))


def launch_count() -> int:
    return int(load().forge_launch_count())

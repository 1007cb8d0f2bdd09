"""Thin Python binding of libadt (ctypes): argument marshalling only.

Each function has the name of the C entry point it calls and takes torch
tensors in place of raw pointers; every step of the computation runs in the
library's CUDA kernels.  A non-OK status raises AdtError.  The library must
have been built (``python -m paper_2512_21857_gb300.build``); importing a
missing library raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadt.so")
MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")

ADT_OK = 0
STATUS_NAMES = {0: "ADT_OK", 1: "ADT_ERR_INVALID_ARG", 2: "ADT_ERR_UNSUPPORTED", 3: "ADT_ERR_CUDA",
                4: "ADT_ERR_TIMEOUT", 5: "ADT_ERR_WORKSPACE", 6: "ADT_ERR_DEVICE"}
ACCEPT_GREEDY, ACCEPT_SPEC, ACCEPT_SPEC_DET = 0, 1, 2
INIT_HORIZONTAL, INIT_VERTICAL, INIT_RANDOM, INIT_TOKENFLOCK = 0, 1, 2, 3
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
NORM_RMS, NORM_LAYER = 0, 1
ROPE_NONE, ROPE_LINEAR, ROPE_NTK, ROPE_BY_PARTS = 0, 1, 2, 3
DEVERR_BAD_TREE, DEVERR_KV_RANGE, DEVERR_BAD_PATH, DEVERR_TIMEOUT, DEVERR_BAD_INDEX = 1, 2, 4, 8, 16

EXPORTED = [
    "adt_version", "adt_get_device_error", "adt_status_string", "adt_testing_set_wait_limit", "adt_testing_exp_diff",
    "adt_testing_attn_plan", "adt_testing_accept_cluster",
    "adt_tree_attn_workspace_size", "adt_tree_attn", "adt_tree_attn_noalloc",
    "adt_tree_expand_workspace_size", "adt_tree_expand", "adt_tree_expand_cfg",
    "adt_tree_rerank_workspace_size", "adt_tree_rerank",
    "adt_tree_accept_workspace_size", "adt_tree_accept", "adt_tree_accept_cfg",
    "adt_kv_compact", "adt_kv_compact_inplace",
    "adt_rope_freqs", "adt_rope_qkv", "adt_kv_score", "adt_kv_evict",
    "adt_norm_rope_qkv", "adt_kv_compact_q8", "adt_kv_read_q8", "adt_tree_attn_q8_workspace_size", "adt_tree_attn_q8",
    "adt_ctrl_create", "adt_ctrl_destroy", "adt_ctrl_next", "adt_ctrl_update", "adt_ctrl_get",
    "adt_ctrl_state_size", "adt_ctrl_save", "adt_ctrl_load",
]


class AdtError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")
        self.status = status


class CtrlParams(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_double), ("l_d", ctypes.c_int32), ("l_k", ctypes.c_int32),
                ("d_lo", ctypes.c_int32), ("d_hi", ctypes.c_int32), ("k_lo", ctypes.c_int32),
                ("k_hi", ctypes.c_int32), ("init_mode", ctypes.c_int32), ("d0", ctypes.c_int32),
                ("k0", ctypes.c_int32), ("clamp_k_always", ctypes.c_int32), ("k_cap", ctypes.c_int32),
                ("fix_d", ctypes.c_int32), ("fix_k", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("flock_delta", ctypes.c_int32)]


class RopeParams(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_double), ("factor", ctypes.c_double), ("orig_len", ctypes.c_double),
                ("turns_lo", ctypes.c_double), ("turns_hi", ctypes.c_double), ("rotary_dim", ctypes.c_int32),
                ("scaling", ctypes.c_int32)]


_P, _I32, _I64, _F32, _SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_SIGS = {
    "adt_version": ([], _I32),
    "adt_get_device_error": ([_P, ctypes.POINTER(ctypes.c_uint32)], _I32),
    "adt_status_string": ([_I32], ctypes.c_char_p),
    "adt_testing_set_wait_limit": ([ctypes.c_uint32], _I32),
    "adt_testing_exp_diff": ([_P, _P, _I32, _P, _P], _I32),
    "adt_testing_attn_plan": ([_I32] * 6 + [ctypes.POINTER(_I32)], _I32),
    "adt_testing_accept_cluster": ([_I32, _I32, _I32, ctypes.POINTER(_I32)], _I32),
    "adt_tree_attn_workspace_size": ([_I32] * 5, _SZ),
    "adt_tree_attn": ([_P, _P, _P, _P, _I64, _I64, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _F32,
                       _P, _P, _P, _SZ, _P], _I32),
    "adt_tree_attn_noalloc": ([_P, _P, _P, _P, _I64, _I64, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32,
                               _F32, _P, _P, _P], _I32),
    "adt_tree_expand_workspace_size": ([_I32] * 3, _SZ),
    "adt_tree_expand": ([_P, _I64, _P, _P, _I32, _I32, _I32, _I32, _F32, _I32, _P, _P, _P, _P, _P, _P, _P,
                         _P, _SZ, _P], _I32),
    "adt_tree_expand_cfg": ([_P, _P, _I64, _F32, _P, _P, _I32, _I32, _I32, _I32, _F32, _I32, _P, _P, _P, _P, _P,
                             _P, _P, _P, _SZ, _P], _I32),
    "adt_tree_rerank_workspace_size": ([_I32], _SZ),
    "adt_tree_rerank": ([_P, _P, _P, _I32, _P, _I32, _P, _P, _P, _P, _P, _SZ, _P], _I32),
    "adt_tree_accept_workspace_size": ([_I32, _I32], _SZ),
    "adt_tree_accept": ([_P, _I64, _P, _I64, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _F32, _P, _I32,
                         _P, _P, _P, _SZ, _P], _I32),
    "adt_tree_accept_cfg": ([_P, _P, _I64, _P, _P, _I64, _P, _F32, _P, _P, _P, _I32, _I32, _I32, _P, _P, _I32,
                             _F32, _P, _I32, _P, _P, _P, _SZ, _P], _I32),
    "adt_kv_compact": ([_P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I64, _I64,
                        _I64, _I64, _P], _I32),
    "adt_kv_compact_inplace": ([_P, _P, _P, _P, _P, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I64, _I64, _I64,
                                _P], _I32),
    "adt_rope_freqs": ([ctypes.POINTER(RopeParams), _P, ctypes.POINTER(_F32)], _I32),
    "adt_rope_qkv": ([_P, _I64, _P, _I64, _P, _I64, _I32, _P, _P, _F32, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P, _P,
                      _P], _I32),
    "adt_kv_score": ([_P, _P, _P, _P, _P, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I64, _I64, _I64, _I64,
                      _I64, _F32, _F32, _P, _P, _I64, _I64, _I64, _P], _I32),
    "adt_kv_evict": ([_P, _P, _I64, _I64, _I64, _P, _I64, _I64, _I64, _P, _P, _P, _P, _I64, _I64, _I64, _P, _I64, _I64,
                      _I64, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P], _I32),
    "adt_norm_rope_qkv": ([_P, _I64, _P, _I64, _P, _I64, _I32, _I32, _F32, _P, _P, _I32, _P, _P, _I32, _I32, _P, _P, _F32,
                           _I32, _I32, _I32, _I32, _I32, _I32, _P, _P, _P, _P], _I32),
    "adt_kv_compact_q8": ([_P] * 10 + [_I32, _P, _I32, _I32, _I32, _I32, _I32] + [_I64] * 7 + [_P], _I32),
    "adt_kv_read_q8": ([_P] * 7 + [_I32] * 5 + [_I64] * 9 + [_P], _I32),
    "adt_tree_attn_q8_workspace_size": ([_I32] * 6, _SZ),
    "adt_tree_attn_q8": ([_P] * 6 + [_I64] * 4 + [_P] * 4 + [_I32] * 6 + [_F32, _P, _P, _P, _SZ, _P], _I32),
    "adt_ctrl_create": ([ctypes.POINTER(CtrlParams), _I32, _I32, ctypes.POINTER(_P)], _I32),
    "adt_ctrl_destroy": ([_P], None),
    "adt_ctrl_state_size": ([_P], _SZ),
    "adt_ctrl_save": ([_P, _P, _SZ], _I32),
    "adt_ctrl_load": ([_P, _SZ, ctypes.POINTER(_P)], _I32),
    "adt_ctrl_next": ([_P, _I32, ctypes.POINTER(_I32), ctypes.POINTER(_I32)], _I32),
    "adt_ctrl_update": ([_P, _I32, _I32, ctypes.POINTER(_I32)], _I32),
    "adt_ctrl_get": ([_P, _I32, ctypes.POINTER(_I32), ctypes.POINTER(_I32)], _I32),
}

_LIB = None
_MARSHAL = None


def _native():
    """The C++ part that marshals the calls of the later operators (once)."""
    global _MARSHAL
    if _MARSHAL is None:
        lib()
        if not os.path.exists(MARSHAL_PATH):
            raise RuntimeError(f"{MARSHAL_PATH} is missing: build it with `python -m paper_2512_21857_gb300.build`")
        spec = importlib.util.spec_from_file_location("_marshal", MARSHAL_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.load(LIB_PATH)
        _MARSHAL = module
    return _MARSHAL


def lib() -> ctypes.CDLL:
    """Loads libadt.so (once).  Raises if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_21857_gb300.build`")
        so = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGS.items():
            fn = getattr(so, name)
            fn.argtypes = args
            fn.restype = res
        _LIB = so
    return _LIB


def _check(status: int, where: str) -> None:
    if status != ADT_OK:
        raise AdtError(status, where)


# A call's marshalling is on a decode loop's critical path (the launch itself
# takes 2 us): addresses go to ctypes as plain integers, and the current
# stream's handle is read without building a torch.cuda.Stream for it (3.0 ->
# 0.2 us a call).

def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_get_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _nbytes(t):
    return t.numel() * t.element_size()


def _expect(t, dtype, name):
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")


def zeroed_workspace(nbytes: int, device=None) -> torch.Tensor:
    """A zero-filled byte buffer usable as a workspace (counters start at 0)."""
    return torch.zeros(max(int(nbytes), 16), dtype=torch.uint8, device=device or "cuda")


# ----------------------------------------------------------------------------- queries

def adt_version() -> int:
    return lib().adt_version()


def adt_get_device_error(stream=None) -> int:
    bits = ctypes.c_uint32(0)
    lib().adt_get_device_error(_stream(stream), ctypes.byref(bits))
    return int(bits.value)


def adt_testing_set_wait_limit(polls: int) -> None:
    """Testing hook: polls before the waits of adt_tree_attn and of sampling walks give up (0 = defaults)."""
    _check(lib().adt_testing_set_wait_limit(int(polls)), "adt_testing_set_wait_limit")


def adt_testing_attn_plan(B, H, Hkv, D, max_nodes, max_kv):
    """Testing hook: (query rows a thread block, thread blocks that share the keys, prefetching clusters)."""
    plan = (_I32 * 3)()
    _check(lib().adt_testing_attn_plan(B, H, Hkv, D, max_nodes, max_kv, plan), "adt_testing_attn_plan")
    return tuple(plan)


def adt_testing_exp_diff(a, b, out, stream=None) -> None:
    """Testing hook: out = e^(a - b) in the acceptance walk's double-float arithmetic."""
    _check(lib().adt_testing_exp_diff(_ptr(a), _ptr(b), int(a.numel()), _ptr(out), _stream(stream)),
           "adt_testing_exp_diff")


def adt_tree_attn_workspace_size(B, H, D, max_nodes, max_kv) -> int:
    return int(lib().adt_tree_attn_workspace_size(B, H, D, max_nodes, max_kv))


def adt_tree_expand_workspace_size(F, V, k_child) -> int:
    return int(lib().adt_tree_expand_workspace_size(F, V, k_child))


def adt_tree_rerank_workspace_size(C) -> int:
    return int(lib().adt_tree_rerank_workspace_size(C))


def adt_tree_accept_workspace_size(B, V) -> int:
    return int(lib().adt_tree_accept_workspace_size(B, V))


# ----------------------------------------------------------------------------- kernels

def adt_tree_attn(q, k_cache, v_cache, kv_len, k_tree, v_tree, parents, node_offsets, *, B, H, Hkv, D,
                  max_nodes, max_kv, softmax_scale, out, lse=None, workspace, cache_stride_b=None,
                  cache_stride_h=None, stream=None) -> None:
    """q, k_tree, v_tree, out: bf16 [Ntot, *, D]; caches bf16 with (b, g, pos, d) strides."""
    bf16, i32 = torch.bfloat16, torch.int32
    _expect(q, bf16, "q")
    _expect(k_tree, bf16, "k_tree")
    _expect(v_tree, bf16, "v_tree")
    _expect(out, bf16, "out")
    _expect(kv_len, i32, "kv_len")
    _expect(parents, i32, "parents")
    _expect(node_offsets, i32, "node_offsets")
    if k_cache.dtype != bf16 or v_cache.dtype != bf16:
        raise TypeError("caches must be bf16")
    strides = k_cache.stride()
    if strides != v_cache.stride():
        raise ValueError("k_cache and v_cache must share strides")
    sb = strides[0] if cache_stride_b is None else cache_stride_b
    sh = strides[1] if cache_stride_h is None else cache_stride_h
    if lse is not None:
        _expect(lse, torch.float32, "lse")
    st = lib().adt_tree_attn(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len), sb, sh, _ptr(k_tree),
                             _ptr(v_tree), _ptr(parents), _ptr(node_offsets), B, H, Hkv, D, max_nodes, max_kv,
                             float(softmax_scale), _ptr(out), _ptr(lse), _ptr(workspace),
                             _nbytes(workspace), _stream(stream))
    _check(st, "adt_tree_attn")


def adt_tree_expand(logits, frontier_score, frontier_id, *, F, V, k_child, k_keep, temperature=1.0,
                    child_id_base=0, child_token, child_logp, child_score, child_parent, keep_idx,
                    next_score=None, next_id=None, workspace, ld=None, stream=None) -> None:
    _expect(frontier_score, torch.float32, "frontier_score")
    if logits.dtype != torch.float32 or logits.stride(-1) != 1:
        raise TypeError("logits: fp32 rows with unit inner stride")
    if logits.dim() != 2:
        raise ValueError("logits: [F, V] rows")
    ld = logits.stride(0) if ld is None else ld
    st = lib().adt_tree_expand(_ptr(logits), ld, _ptr(frontier_score), _ptr(frontier_id), F, V, k_child, k_keep,
                               float(temperature), int(child_id_base), _ptr(child_token), _ptr(child_logp),
                               _ptr(child_score), _ptr(child_parent), _ptr(keep_idx), _ptr(next_score),
                               _ptr(next_id), _ptr(workspace), _nbytes(workspace),
                               _stream(stream))
    _check(st, "adt_tree_expand")


def adt_tree_expand_cfg(logits_cond, logits_uncond, frontier_score, frontier_id, *, cfg_scale, F, V, k_child,
                        k_keep, temperature=1.0, child_id_base=0, child_token, child_logp, child_score,
                        child_parent, keep_idx, next_score=None, next_id=None, workspace, stream=None) -> None:
    """adt_tree_expand on uncond + cfg_scale * (cond - uncond); both [F, V] rows share one row stride."""
    _expect(frontier_score, torch.float32, "frontier_score")
    for t in (logits_cond, logits_uncond):
        if t.dtype != torch.float32 or t.dim() != 2 or t.stride(-1) != 1:
            raise TypeError("logits: fp32 [F, V] rows with unit inner stride")
    if logits_cond.stride(0) != logits_uncond.stride(0):
        raise ValueError("conditional and unconditional rows must share a row stride")
    st = lib().adt_tree_expand_cfg(_ptr(logits_cond), _ptr(logits_uncond), logits_cond.stride(0), float(cfg_scale),
                                   _ptr(frontier_score), _ptr(frontier_id), F, V, k_child, k_keep,
                                   float(temperature), int(child_id_base), _ptr(child_token), _ptr(child_logp),
                                   _ptr(child_score), _ptr(child_parent), _ptr(keep_idx), _ptr(next_score),
                                   _ptr(next_id), _ptr(workspace), _nbytes(workspace),
                                   _stream(stream))
    _check(st, "adt_tree_expand_cfg")


def adt_tree_rerank(cand_token, cand_score, cand_parent, C, root_token, n_nodes, *, tokens, parents,
                    cand_index=None, depth=None, workspace, stream=None) -> None:
    st = lib().adt_tree_rerank(_ptr(cand_token), _ptr(cand_score), _ptr(cand_parent), int(C), _ptr(root_token),
                               int(n_nodes), _ptr(tokens), _ptr(parents), _ptr(cand_index), _ptr(depth),
                               _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(st, "adt_tree_rerank")


def adt_tree_accept(target_logits, draft_logits, tokens, parents, node_offsets, *, B, V, max_nodes, mode,
                    u_accept=None, u_sample=None, temperature=1.0, path, max_path, accept_len, bonus_token,
                    draft_row=None, workspace=None, stream=None) -> None:
    ldt = target_logits.stride(0)
    ldd = draft_logits.stride(0) if draft_logits is not None else 0
    ws = workspace
    st = lib().adt_tree_accept(_ptr(target_logits), ldt, _ptr(draft_logits), ldd, _ptr(draft_row), _ptr(tokens),
                               _ptr(parents), _ptr(node_offsets), B, V, max_nodes, _ptr(u_accept),
                               _ptr(u_sample), int(mode), float(temperature), _ptr(path), int(max_path),
                               _ptr(accept_len), _ptr(bonus_token), _ptr(ws),
                               0 if ws is None else _nbytes(ws), _stream(stream))
    _check(st, "adt_tree_accept")


def adt_tree_accept_cfg(target_cond, target_uncond, draft_cond, draft_uncond, tokens, parents, node_offsets, *,
                        cfg_scale, B, V, max_nodes, mode, u_accept=None, u_sample=None, temperature=1.0, path,
                        max_path, accept_len, bonus_token, draft_row=None, stream=None) -> None:
    """adt_tree_accept with every target / draft row formed as uncond + cfg_scale * (cond - uncond)."""
    if target_cond.stride(0) != target_uncond.stride(0):
        raise ValueError("conditional and unconditional target rows must share a row stride")
    ldd = draft_cond.stride(0) if draft_cond is not None else 0
    if draft_cond is not None and draft_uncond is not None and draft_uncond.stride(0) != ldd:
        raise ValueError("conditional and unconditional draft rows must share a row stride")
    st = lib().adt_tree_accept_cfg(_ptr(target_cond), _ptr(target_uncond), target_cond.stride(0), _ptr(draft_cond),
                                   _ptr(draft_uncond), ldd, _ptr(draft_row), float(cfg_scale), _ptr(tokens),
                                   _ptr(parents), _ptr(node_offsets), B, V, max_nodes, _ptr(u_accept),
                                   _ptr(u_sample), int(mode), float(temperature), _ptr(path), int(max_path),
                                   _ptr(accept_len), _ptr(bonus_token), None, 0, _stream(stream))
    _check(st, "adt_tree_accept_cfg")


def adt_kv_compact(k_cache, v_cache, kv_len, kv_len_out, k_tree, v_tree, node_offsets, path, max_path,
                   accept_len, *, B, Hkv, D, num_layers, max_kv, cache_layer_stride, cache_stride_b,
                   cache_stride_h, tree_layer_stride, stream=None) -> None:
    st = lib().adt_kv_compact(_ptr(k_cache), _ptr(v_cache), _ptr(kv_len), _ptr(kv_len_out), _ptr(k_tree),
                              _ptr(v_tree), _ptr(node_offsets), _ptr(path), int(max_path), _ptr(accept_len),
                              B, Hkv, D, num_layers, max_kv, cache_layer_stride, cache_stride_b, cache_stride_h,
                              tree_layer_stride, _stream(stream))
    _check(st, "adt_kv_compact")


def adt_kv_compact_inplace(k_cache, v_cache, kv_len, kv_len_out, node_offsets, path, max_path, accept_len, *, B,
                           Hkv, D, num_layers, max_kv, cache_layer_stride, cache_stride_b, cache_stride_h,
                           stream=None) -> None:
    st = lib().adt_kv_compact_inplace(_ptr(k_cache), _ptr(v_cache), _ptr(kv_len), _ptr(kv_len_out),
                                      _ptr(node_offsets), _ptr(path), int(max_path), _ptr(accept_len), B, Hkv, D,
                                      num_layers, max_kv, cache_layer_stride, cache_stride_b, cache_stride_h,
                                      _stream(stream))
    _check(st, "adt_kv_compact_inplace")


# ----------------------------------------------------------------------------- positions and a bounded cache

_TYPES = {torch.bfloat16: 0, torch.float32: 1}

# These calls are made from Python one at a time as often as in a graph, and take 9 to 18 tensors: each is looked at
# once (device, type and address; shape and strides as whole tuples), which halves what a call costs the host.


def _addr(t, dtype, dev, name):
    """The address of a tensor of that type on CUDA device dev, the current one, which the launch goes to; None for None."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError(f"{name}: expected a tensor on the current CUDA device, got one on {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _vec(t, dtype, dev, count, name):
    """The address of a contiguous tensor of at least `count` elements; None for None."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != dev:
        return _addr(t, dtype, dev, name)  # raises
    if t.numel() < count or not t.is_contiguous():
        raise ValueError(f"{name}: expected {count} elements, contiguous")
    return t.data_ptr()


def _launch_on(t, stream, name):
    """(current CUDA device, handle of the stream) of a call whose tensor t has to be on that device."""
    dev = t.get_device()
    if dev < 0 or dev != (_get_device() if _get_device is not None else torch.cuda.current_device()):
        raise ValueError(f"{name}: expected a tensor on the current CUDA device, got one on {t.device}")
    if stream is not None:
        return dev, stream.cuda_stream
    return dev, _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def adt_rope_freqs(rotary_dim, *, theta=10000.0, scaling=ROPE_NONE, factor=1.0, orig_len=0.0, turns_lo=1.0,
                   turns_hi=32.0):
    """(inv_freq, magnitude): fp64 [rotary_dim / 2] on the CPU, radians a position, to be copied to the device once."""
    p = RopeParams(theta, factor, orig_len, turns_lo, turns_hi, rotary_dim, scaling)
    inv = torch.empty(max(rotary_dim // 2, 1), dtype=torch.float64)
    mag = _F32()
    _check(lib().adt_rope_freqs(ctypes.byref(p), inv.data_ptr(), ctypes.byref(mag)), "adt_rope_freqs")
    return inv, mag.value


def _rope_pair(t, out, dtype, dev, heads, D, N, name):
    """(address, row stride, output address) of [N, heads * D] rows or [N, heads, D] heads, contiguous within a row."""
    if t is None or out is None:
        if t is not out:
            raise ValueError(f"{name} and {name}_out: both or neither")
        return None, 0, None
    shape, strides, width = t.shape, t.stride(), heads * D
    if not (shape == (N, width) and strides[1] == 1 or
            shape == (N, heads, D) and strides[2] == 1 and (strides[1] == D or heads == 1)):
        raise ValueError(f"{name}: expected rows [{N}, {width}] or [{N}, {heads}, {D}], contiguous within a row")
    if out.numel() != N * width:
        raise ValueError(f"{name}_out: expected [{N}, {heads}, {D}]")
    return (_addr(t, dtype, dev, name), strides[0] if N > 1 else width,
            _vec(out, torch.bfloat16, dev, 0, name + "_out"))


def adt_rope_qkv(q, k, v, positions, inv_freq, *, H, Hkv, D, layout=ROPE_HALF, magnitude=1.0, q_out=None, k_out=None,
                 v_out=None, stream=None) -> None:
    """q [N, H * D], k and v [N, Hkv * D] rows (bf16 or fp32, any row stride; None: absent) to bf16 [N, heads, D]
    outputs: q and k rotated by positions * inv_freq, v copied.  rotary_dim = 2 * len(inv_freq)."""
    dev, handle = _launch_on(positions, stream, "positions")
    N = positions.numel()
    first = q if q is not None else k if k is not None else v
    if first is None or first.dtype not in _TYPES:
        raise TypeError("q, k, v: bf16 or fp32, all the same")
    dtype = first.dtype
    qa, ldq, qo = _rope_pair(q, q_out, dtype, dev, H, D, N, "q")
    ka, ldk, ko = _rope_pair(k, k_out, dtype, dev, Hkv, D, N, "k")
    va, ldv, vo = _rope_pair(v, v_out, dtype, dev, Hkv, D, N, "v")
    st = lib().adt_rope_qkv(qa, ldq, ka, ldk, va, ldv, _TYPES[dtype], _vec(positions, torch.int32, dev, N, "positions"),
                            _vec(inv_freq, torch.float64, dev, 0, "inv_freq"), magnitude, layout, N, H, Hkv, D,
                            2 * inv_freq.numel(), qo, ko, vo, handle)
    _check(st, "adt_rope_qkv")


def _strides3(t, layers, B, Hkv, rows, D, name):
    """Strides of the first three dimensions of [layers, B, Hkv, rows or more, D] (D = 0: of [layers, B, Hkv, rows or
    more]), those of a dimension of one as 0: they say nothing; the rows are packed."""
    shape, strides = t.shape, t.stride()
    want = 5 if D else 4
    if len(shape) != want or shape[0] != layers or shape[1] != B or shape[2] != Hkv or shape[3] < rows or \
            (D and shape[4] != D):
        raise ValueError(f"{name}: expected {[layers, B, Hkv, rows, D][:want]} or more rows, got {list(shape)}")
    if (strides[3] != (D or 1) and shape[3] > 1) or (D and strides[4] != 1):
        raise ValueError(f"{name}: expected packed rows")
    return strides[0] if layers > 1 else 0, strides[1] if B > 1 else 0, strides[2] if Hkv > 1 else 0


def adt_kv_score(q, lse, k_cache, kv_len, node_offsets, path, max_path, accept_len, score, *, score_out=None, B, H, Hkv,
                 D, num_layers, max_kv, softmax_scale, decay=1.0, stream=None) -> None:
    """q [layers, nodes, H, D] bf16, lse [layers, nodes, H], k_cache [layers, B, Hkv, rows >= max_kv, D] and score
    [layers, B, Hkv, rows >= max_kv] fp32, updated in place unless score_out (the same strides) is given."""
    dev, handle = _launch_on(q, stream, "q")
    f32, i32, bf16 = torch.float32, torch.int32, torch.bfloat16
    qs, ls, nodes = q.stride(), lse.stride(), q.shape[1]
    # (Strides of dimensions of one say nothing: torch's own check where they differ.)
    if q.shape[2:] != (H, D) or q.shape[0] < num_layers or (qs[1:] != (H * D, D, 1) and not q[0].is_contiguous()):
        raise ValueError(f"q: expected [{num_layers}, nodes, {H}, {D}], each layer contiguous")
    if lse.shape[1:] != (nodes, H) or lse.shape[0] < num_layers or (ls[1:] != (H, 1) and not lse[0].is_contiguous()):
        raise ValueError(f"lse: expected [{num_layers}, {nodes}, {H}], each layer contiguous")
    cs = _strides3(k_cache, num_layers, B, Hkv, max_kv, D, "k_cache")
    ss = _strides3(score, num_layers, B, Hkv, max_kv, 0, "score")
    sa = _addr(score, f32, dev, "score")
    if score_out is None:
        so = sa
    else:
        so = _addr(score_out, f32, dev, "score_out")
        if _strides3(score_out, num_layers, B, Hkv, max_kv, 0, "score_out") != ss:
            raise ValueError("score and score_out must share strides")
    st = lib().adt_kv_score(_addr(q, bf16, dev, "q"), _addr(lse, f32, dev, "lse"), _addr(k_cache, bf16, dev, "k_cache"),
                            _vec(kv_len, i32, dev, B, "kv_len"), _vec(node_offsets, i32, dev, B + 1, "node_offsets"),
                            _vec(path, i32, dev, B * max_path, "path"), max_path,
                            _vec(accept_len, i32, dev, B, "accept_len"), B, H, Hkv, D, num_layers, max_kv,
                            qs[0] if num_layers > 1 else 0, ls[0] if num_layers > 1 else 0, *cs,
                            softmax_scale, decay, sa, so, *ss, handle)
    _check(st, "adt_kv_score")


def adt_kv_evict(k_cache, v_cache, score, kv_len, kv_len_out=None, *, k_out=None, v_out=None, score_out=None,
                 move_scores=True, keep_idx=None, B, Hkv, D, num_layers, max_kv, budget, n_sink=0, n_recent=0,
                 stream=None) -> None:
    """Caches [layers, B, Hkv, rows >= max_kv, D] bf16 and score [layers, B, Hkv, rows >= max_kv] fp32 cut down to
    `budget` rows: in place, or into k_out, v_out.  The scores go to score_out, by default to where the rows went (in
    place: the same buffer); with move_scores=False they stay as they are."""
    if (k_out is None) != (v_out is None):
        raise ValueError("k_out and v_out: both or neither")
    if score_out is not None and not move_scores:
        raise ValueError("score_out without moving scores")
    if score_out is None and move_scores and k_out is not None:
        raise ValueError("score_out: needed where the rows go to another cache")
    dev, handle = _launch_on(k_cache, stream, "k_cache")
    f32, i32, bf16 = torch.float32, torch.int32, torch.bfloat16
    ks = _strides3(k_cache, num_layers, B, Hkv, max_kv, D, "k_cache")
    cs = co = _strides3(score, num_layers, B, Hkv, max_kv, 0, "score")
    same = _strides3(v_cache, num_layers, B, Hkv, max_kv, D, "v_cache") == ks
    ka, va, sa = _addr(k_cache, bf16, dev, "k_cache"), _addr(v_cache, bf16, dev, "v_cache"), _addr(score, f32, dev, "score")
    ko, vo, so, to = ka, va, sa if move_scores else None, ks
    rows = min(max_kv, budget)
    if k_out is not None and k_out is not k_cache:
        to = _strides3(k_out, num_layers, B, Hkv, rows, D, "k_out")
        ko = _addr(k_out, bf16, dev, "k_out")
    if v_out is not None and v_out is not v_cache:
        same = same and _strides3(v_out, num_layers, B, Hkv, rows, D, "v_out") == to
        vo = _addr(v_out, bf16, dev, "v_out")
    if not same:
        raise ValueError("K and V must share strides")
    if score_out is not None:
        co, so = _strides3(score_out, num_layers, B, Hkv, rows, 0, "score_out"), _addr(score_out, f32, dev, "score_out")
    st = lib().adt_kv_evict(ka, va, *ks, sa, *cs, _vec(kv_len, i32, dev, B, "kv_len"),
                            _vec(kv_len_out, i32, dev, B, "kv_len_out"), ko, vo, *to, so, *co,
                            _vec(keep_idx, i32, dev, num_layers * B * Hkv * budget, "keep_idx"), B, Hkv, D, num_layers,
                            max_kv, budget, n_sink, n_recent, handle)
    _check(st, "adt_kv_evict")


def adt_norm_rope_qkv(q, k, v, positions, inv_freq, *, H, Hkv, D, norm=NORM_RMS, eps=1e-6, q_weight=None, q_bias=None,
                      k_weight=None, k_bias=None, layout=ROPE_HALF, magnitude=1.0, q_out=None, k_out=None, v_out=None,
                      stream=None) -> None:
    """adt_rope_qkv of heads that are normed first.  Weights and biases (fp32 or bf16, all the same): [D] for all heads,
    or a head's own in [heads, D]; None: ones, zeros."""
    st = (_MARSHAL or _native()).norm_rope_qkv(q, k, v, positions, inv_freq, H, Hkv, D, norm, eps, q_weight, q_bias, k_weight,
                                               k_bias, layout, magnitude, q_out, k_out, v_out, stream)
    if st:
        _check(st, "adt_norm_rope_qkv")


# ----------------------------------------------------------------------------- the 8-bit cache

# (Their checks of tensors: csrc/marshal.cc.)


def adt_kv_compact_q8(k_cache, v_cache, k_scale, v_scale, kv_len, kv_len_out, k_tree, v_tree, node_offsets, path, max_path,
                      accept_len, *, B, Hkv, D, num_layers, max_kv, stream=None) -> None:
    """Caches [layers, B, Hkv, rows >= max_kv, D] float8_e4m3fn, scales [layers, B, Hkv, rows >= max_kv] uint8, k_tree and
    v_tree [layers, nodes, Hkv, D] bf16; kv_len_out may be None."""
    st = (_MARSHAL or _native()).kv_compact_q8(k_cache, v_cache, k_scale, v_scale, kv_len, kv_len_out, k_tree, v_tree,
                                               node_offsets, path, max_path, accept_len, B, Hkv, D, num_layers, max_kv, stream)
    if st:
        _check(st, "adt_kv_compact_q8")


def adt_kv_read_q8(k_cache, v_cache, k_scale, v_scale, kv_len, k_out, v_out, *, B, Hkv, D, num_layers, max_kv,
                   stream=None) -> None:
    """Rows of an 8-bit cache (as for adt_kv_compact_q8) to k_out, v_out [layers, B, Hkv, rows >= max_kv, D] bf16."""
    st = (_MARSHAL or _native()).kv_read_q8(k_cache, v_cache, k_scale, v_scale, kv_len, k_out, v_out, B, Hkv, D, num_layers,
                                            max_kv, stream)
    if st:
        _check(st, "adt_kv_read_q8")


def adt_tree_attn_q8_workspace_size(B, H, Hkv, D, max_nodes, max_kv) -> int:
    return int(lib().adt_tree_attn_q8_workspace_size(B, H, Hkv, D, max_nodes, max_kv))


def adt_tree_attn_q8(q, k_cache, v_cache, k_scale, v_scale, kv_len, k_tree, v_tree, parents, node_offsets, *, B, H, Hkv, D,
                     max_nodes, max_kv, softmax_scale, out, lse=None, workspace, stream=None) -> None:
    """adt_tree_attn of one layer over caches [B, Hkv, rows >= max_kv, D] float8_e4m3fn with scales
    [B, Hkv, rows >= max_kv] uint8; q, k_tree, v_tree, out bf16 [Ntot, *, D], lse fp32 [Ntot, H] or None."""
    st = (_MARSHAL or _native()).tree_attn_q8(q, k_cache, v_cache, k_scale, v_scale, kv_len, k_tree, v_tree, parents,
                                              node_offsets, B, H, Hkv, D, max_nodes, max_kv, softmax_scale, out, lse, workspace,
                                              stream)
    if st:
        _check(st, "adt_tree_attn_q8")


# ----------------------------------------------------------------------------- controller

class Controller:
    """Host depth / width controller (adt_ctrl_*); one per image."""

    def __init__(self, grid_h, grid_w, *, beta=1.0, l_d=1, l_k=3, d_lo=1, d_hi=9, k_lo=4, k_hi=13,
                 init_mode=INIT_HORIZONTAL, d0=5, k0=10, clamp_k_always=True, k_cap=64, fix_d=0, fix_k=0,
                 seed=0, flock_delta=2):
        self._p = CtrlParams(beta, l_d, l_k, d_lo, d_hi, k_lo, k_hi, init_mode, d0, k0, int(bool(clamp_k_always)),
                             k_cap, fix_d, fix_k, seed, flock_delta)
        h = ctypes.c_void_p()
        _check(lib().adt_ctrl_create(ctypes.byref(self._p), grid_h, grid_w, ctypes.byref(h)), "adt_ctrl_create")
        self._h = h

    def next(self, pos):
        d, k = ctypes.c_int32(), ctypes.c_int32()
        _check(lib().adt_ctrl_next(self._h, pos, ctypes.byref(d), ctypes.byref(k)), "adt_ctrl_next")
        return d.value, k.value

    def update(self, pos, accept_len):
        nxt = ctypes.c_int32()
        _check(lib().adt_ctrl_update(self._h, pos, accept_len, ctypes.byref(nxt)), "adt_ctrl_update")
        return nxt.value

    def get(self, pos):
        d, k = ctypes.c_int32(), ctypes.c_int32()
        _check(lib().adt_ctrl_get(self._h, pos, ctypes.byref(d), ctypes.byref(k)), "adt_ctrl_get")
        return d.value, k.value

    def save(self) -> bytes:
        """The controller's state as bytes (checkpoint)."""
        n = int(lib().adt_ctrl_state_size(self._h))
        buf = ctypes.create_string_buffer(n)
        _check(lib().adt_ctrl_save(self._h, buf, n), "adt_ctrl_save")
        return buf.raw

    @classmethod
    def load(cls, state: bytes) -> "Controller":
        """A controller resumed from save()'s bytes."""
        h = ctypes.c_void_p()
        _check(lib().adt_ctrl_load(state, len(state), ctypes.byref(h)), "adt_ctrl_load")
        obj = cls.__new__(cls)
        obj._h = h
        return obj

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and _LIB is not None:
            _LIB.adt_ctrl_destroy(h)
            self._h = None

"""Binding of libcapmoe.so: same names as the C ABI, argument marshalling only (ctypes, and for the calls of a training or
decode step, which come every few microseconds, a compiled one: csrc/bind.cpp).

torch is used for device memory and streams; every step of the layer runs inside the CUDA
library.  If the shared library is missing or cannot be loaded, every call raises: there is
no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.util
import math
import os
from dataclasses import dataclass
from typing import Optional

import torch

from .build import bind_path

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcapmoe.so")
_lib = None

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, ECUDA, ETIMEOUT, EINDEX = range(7)
F32, BF16 = 0, 1
MODE_NODROP, MODE_TOKEN_DROP, MODE_EXPANDED_DROP = 0, 1, 2
MODES = {"nodrop": 0, "token_drop": 1, "expanded_drop": 2, "device_token_drop": 3, "device_expanded_drop": 4}

EXPORTS = ["capmoe_capacity", "capmoe_max_rows", "capmoe_device_max_rows", "capmoe_drop_workspace_bytes", "capmoe_status_str",
           "capmoe_last_cuda_error", "capmoe_launch_count", "capmoe_ffn_uses_tensor_cores", "capmoe_route",
           "capmoe_token_drop", "capmoe_token_drop_static", "capmoe_expanded_drop", "capmoe_device_capacity",
           "capmoe_device_drop", "capmoe_drop_keys", "capmoe_priority_keys", "capmoe_limit_experts",
           "capmoe_rows_from_mask", "capmoe_permute", "capmoe_grouped_ffn",
           "capmoe_combine", "capmoe_layer_forward", "capmoe_layer_forward_host", "capmoe_debug_wait_probe",
           "capmoe_grouped_ffn_segments", "capmoe_debug_ffn_variant", "capmoe_ep_plan", "capmoe_ep_forward_dispatch", "capmoe_ep_forward_experts", "capmoe_ep_forward_combine", "capmoe_ep_segments", "capmoe_ep_dispatch",
           "capmoe_ep_combine", "capmoe_debug_read_probe", "capmoe_debug_check_indices",
           "capmoe_grouped_mm", "capmoe_grouped_mm_dx", "capmoe_grouped_mm_dw_workspace_bytes", "capmoe_grouped_mm_dw",
           "capmoe_dw_split_bytes", "capmoe_ffn_backward_workspace_bytes", "capmoe_grouped_ffn_backward", "capmoe_quantize_rows",
           "capmoe_quantize_weights", "capmoe_grouped_mm_fp8", "capmoe_ffn_fp8_workspace_bytes", "capmoe_grouped_ffn_fp8",
           "capmoe_grouped_ffn_fp8_codes", "capmoe_rms_norm", "capmoe_rms_norm_backward_workspace_bytes", "capmoe_rms_norm_backward",
           "capmoe_permute_fp8", "capmoe_combine_backward", "capmoe_permute_backward", "capmoe_route_backward_workspace_bytes",
           "capmoe_route_backward"]


class CapmoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().capmoe_status_str(status).decode()
        if status == ECUDA:
            msg += " (" + lib().capmoe_last_cuda_error().decode() + ")"
        super().__init__(f"{where}: {msg} [status {status}]")


class _Layer(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int64), ("d", ctypes.c_int), ("E", ctypes.c_int), ("k", ctypes.c_int),
        ("F", ctypes.c_int), ("D", ctypes.c_int), ("dtype", ctypes.c_int),
        ("mode", ctypes.c_int), ("C", ctypes.c_int64), ("straggler", ctypes.c_int),
        ("x", ctypes.c_void_p), ("w_router", ctypes.c_void_p), ("bias", ctypes.c_void_p),
        ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
        ("ws_gate", ctypes.c_void_p), ("ws_up", ctypes.c_void_p), ("ws_down", ctypes.c_void_p),
        ("F_shared", ctypes.c_int),
        ("logits", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("topk_idx", ctypes.c_void_p),
        ("topk_score", ctypes.c_void_p), ("load", ctypes.c_void_p),
        ("keep_mask", ctypes.c_void_p), ("cand", ctypes.c_void_p), ("kept", ctypes.c_void_p),
        ("expert_offsets", ctypes.c_void_p), ("slot_row", ctypes.c_void_p),
        ("x_perm", ctypes.c_void_p), ("perm_token", ctypes.c_void_p), ("perm_weight", ctypes.c_void_p),
        ("h_ws", ctypes.c_void_p), ("y_perm", ctypes.c_void_p), ("A_max", ctypes.c_int64),
        ("hs_ws", ctypes.c_void_p), ("y_shared", ctypes.c_void_p), ("one_segment", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("drop_ws", ctypes.c_void_p), ("drop_ws_bytes", ctypes.c_size_t),
        ("dev_status", ctypes.c_void_p),
        ("stage_events", ctypes.POINTER(ctypes.c_void_p)),
        ("metric", ctypes.c_int), ("metric_seed", ctypes.c_uint64), ("token_class", ctypes.c_void_p),
        ("topk_first", ctypes.c_int), ("max_experts", ctypes.c_int), ("drop_keys", ctypes.c_void_p),
        ("bad", ctypes.c_void_p), ("debug_checks", ctypes.c_int),
    ]

class _EPRank(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int64), ("d", ctypes.c_int), ("E", ctypes.c_int), ("k", ctypes.c_int),
        ("F", ctypes.c_int), ("dtype", ctypes.c_int),
        ("R", ctypes.c_int), ("rank", ctypes.c_int), ("mode", ctypes.c_int),
        ("C_local", ctypes.c_int64), ("C", ctypes.c_int64),
        ("x", ctypes.c_void_p), ("w_router", ctypes.c_void_p), ("bias", ctypes.c_void_p),
        ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
        ("logits", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("topk_idx", ctypes.c_void_p),
        ("topk_score", ctypes.c_void_p), ("load", ctypes.c_void_p),
        ("keep_mask", ctypes.c_void_p), ("cand", ctypes.c_void_p), ("kept", ctypes.c_void_p),
        ("expert_offsets", ctypes.c_void_p), ("slot_row", ctypes.c_void_p),
        ("slot_row_ep", ctypes.c_void_p), ("token_group", ctypes.c_void_p),
        ("perm_token", ctypes.c_void_p), ("perm_weight", ctypes.c_void_p),
        ("x_send", ctypes.c_void_p), ("y_ret", ctypes.c_void_p),
        ("peer_x", ctypes.c_void_p), ("peer_y", ctypes.c_void_p),
        ("x_recv", ctypes.c_void_p), ("h_ws", ctypes.c_void_p), ("y_recv", ctypes.c_void_p),
        ("cnt_recv", ctypes.c_void_p), ("seg_begin", ctypes.c_void_p), ("seg_end", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("drop_ws", ctypes.c_void_p), ("drop_ws_bytes", ctypes.c_size_t),
        ("dev_status", ctypes.c_void_p), ("bad", ctypes.c_void_p),
    ]

N_STAGE_EVENTS = 8
FFN_STATUS_WORDS = 128     # CAPMOE_FFN_STATUS_WORDS: status word + scratch of the FFN's tile schedulers
STAGE_NAMES = ["route", "drop", "permute", "ffn_gate_up", "ffn_down", "shared_ffn", "combine"]


def lib():
    """The loaded CUDA library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_05066_b200.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        L.capmoe_status_str.restype = ctypes.c_char_p
        L.capmoe_last_cuda_error.restype = ctypes.c_char_p
        L.capmoe_launch_count.restype = ctypes.c_uint64
        for name, types in _ARGTYPES.items():
            getattr(L, name).argtypes = types
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return ctypes.c_void_p(0)
    assert t.is_contiguous(), "capmoe tensors must be contiguous"
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dt(t_or_dtype) -> int:
    dt = t_or_dtype.dtype if isinstance(t_or_dtype, torch.Tensor) else t_or_dtype
    if dt == torch.float32:
        return F32
    if dt == torch.bfloat16:
        return BF16
    raise CapmoeError(EUNSUPPORTED, f"dtype {dt}")


def _check(rc: int, where: str):
    if rc != OK:
        raise CapmoeError(rc, where)


def _i64(v):
    return ctypes.c_int64(int(v))


# ----------------------------------------------------------------------------- host helpers
def capacity(N: int, E: int, k: int, gamma: float, round_mode: str = "ceil") -> int:
    out = ctypes.c_int64(0)
    _check(lib().capmoe_capacity(_i64(N), int(E), int(k), ctypes.c_double(gamma),
                                 0 if round_mode == "ceil" else 1, ctypes.byref(out)), "capmoe_capacity")
    return out.value


def max_rows(N: int, E: int, k: int, D: int, C: int, expanded: bool) -> int:
    out = ctypes.c_int64(0)
    _check(lib().capmoe_max_rows(_i64(N), int(E), int(k), int(D), _i64(C), int(bool(expanded)),
                                 ctypes.byref(out)), "capmoe_max_rows")
    return out.value


def device_max_rows(N: int, E: int, k: int, D: int, C_dev: int, expanded: bool) -> int:
    out = ctypes.c_int64(0)
    _check(lib().capmoe_device_max_rows(_i64(N), int(E), int(k), int(D), _i64(C_dev), int(bool(expanded)),
                                        ctypes.byref(out)), "capmoe_device_max_rows")
    return out.value


def drop_workspace_bytes(N: int, E: int, k: int, D: int, expanded: bool) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().capmoe_drop_workspace_bytes(_i64(N), int(E), int(k), int(D), int(bool(expanded)),
                                             ctypes.byref(out)), "capmoe_drop_workspace_bytes")
    return out.value


def launch_count() -> int:
    return int(lib().capmoe_launch_count())


def ffn_uses_tensor_cores(d: int, F: int, dtype) -> bool:
    return bool(lib().capmoe_ffn_uses_tensor_cores(int(d), int(F), _dt(dtype)))


# ----------------------------------------------------------------------------- stages
def route(x, w_router, bias, k: int, logits_in=None, out=None, stream=None):
    """-> dict(logits, scores, topk_idx, topk_score, load); `out` may hand in those buffers to be reused."""
    if logits_in is not None:
        N, E = logits_in.shape
        d, dev, dt = 0, logits_in.device, F32
    else:
        N, d = x.shape
        E = w_router.shape[0]
        dev, dt = x.device, _dt(x)
    f32 = dict(device=dev, dtype=torch.float32)
    i32 = dict(device=dev, dtype=torch.int32)
    if out is None:
        out = dict(logits=torch.empty((N, E), **f32), scores=torch.empty((N, E), **f32),
                   topk_idx=torch.empty((N, k), **i32), topk_score=torch.empty((N, k), **f32),
                   load=torch.empty((E,), **i32))
    _check(lib().capmoe_route(_ptr(x), _ptr(w_router), _ptr(bias), _ptr(logits_in), _i64(N), int(d), int(E),
                              int(k), dt, _ptr(out["logits"]), _ptr(out["scores"]), _ptr(out["topk_idx"]),
                              _ptr(out["topk_score"]), _ptr(out["load"]), _stream(stream)), "capmoe_route")
    return out


def token_drop(topk_score, topk_idx, E: int, C: int, ws=None, stream=None):
    """-> dict(keep_mask, kept, offsets, slot_row)"""
    N, k = topk_idx.shape
    dev = topk_idx.device
    W = (E + 63) // 64
    if ws is None:
        ws = torch.empty((drop_workspace_bytes(N, E, k, 0, False),), device=dev, dtype=torch.uint8)
    out = dict(keep_mask=torch.empty((N, W), device=dev, dtype=torch.int64),
               kept=torch.empty((E,), device=dev, dtype=torch.int32),
               offsets=torch.empty((E + 1,), device=dev, dtype=torch.int32),
               slot_row=torch.empty((N, k), device=dev, dtype=torch.int32))
    _check(lib().capmoe_token_drop(_ptr(topk_score), _ptr(topk_idx), _i64(N), int(E), int(k), _i64(C),
                                   _ptr(out["keep_mask"]), _ptr(out["kept"]), _ptr(out["offsets"]),
                                   _ptr(out["slot_row"]), _ptr(ws), ctypes.c_size_t(ws.numel()),
                                   _stream(stream)), "capmoe_token_drop")
    return out


STATIC_DROP_MAX_PAIRS = 1 << 20


def token_drop_static(topk_score, topk_idx, E: int, C: int, stream=None):
    """Token Drop through the entry point that needs no workspace from the caller (the scratch
    is a fixed array inside the library, shared by all calls on the device: do not overlap calls).
    Limited to N*k <= STATIC_DROP_MAX_PAIRS.  -> dict(keep_mask, kept, offsets, slot_row)"""
    N, k = topk_idx.shape
    dev = topk_idx.device
    W = (E + 63) // 64
    out = dict(keep_mask=torch.empty((N, W), device=dev, dtype=torch.int64),
               kept=torch.empty((E,), device=dev, dtype=torch.int32),
               offsets=torch.empty((E + 1,), device=dev, dtype=torch.int32),
               slot_row=torch.empty((N, k), device=dev, dtype=torch.int32))
    rc = lib().capmoe_token_drop_static(_ptr(topk_score), _ptr(topk_idx), _i64(N), int(E), int(k), _i64(C),
                                        _ptr(out["keep_mask"]), _ptr(out["kept"]), _ptr(out["offsets"]),
                                        _ptr(out["slot_row"]), _stream(stream))
    if rc == EWORKSPACE:
        raise CapmoeError(rc, f"capmoe_token_drop_static: N*k = {N * k} exceeds the built-in scratch "
                              f"({STATIC_DROP_MAX_PAIRS} pairs)")
    _check(rc, "capmoe_token_drop_static")
    return out


def expanded_drop(scores, topk_idx, C: int, D: int, token_group=None, ws=None, stream=None):
    """-> dict(keep_mask, cand, kept, offsets, slot_row)"""
    N, E = scores.shape
    k = topk_idx.shape[1]
    dev = scores.device
    if D < 1 or E % D != 0:
        raise CapmoeError(EINVAL, "capmoe_expanded_drop: E % D != 0")
    m = E // D
    W = (E + 63) // 64
    if ws is None:
        ws = torch.empty((drop_workspace_bytes(N, E, k, D, True),), device=dev, dtype=torch.uint8)
    out = dict(keep_mask=torch.empty((N, W), device=dev, dtype=torch.int64),
               cand=torch.empty((E,), device=dev, dtype=torch.int32),
               kept=torch.empty((E,), device=dev, dtype=torch.int32),
               offsets=torch.empty((E + 1,), device=dev, dtype=torch.int32),
               slot_row=torch.empty((N, k + m), device=dev, dtype=torch.int32))
    _check(lib().capmoe_expanded_drop(_ptr(scores), _ptr(topk_idx), _i64(N), int(E), int(k), _i64(C), int(D),
                                      _ptr(token_group), _ptr(out["keep_mask"]), _ptr(out["cand"]),
                                      _ptr(out["kept"]), _ptr(out["offsets"]), _ptr(out["slot_row"]), _ptr(ws),
                                      ctypes.c_size_t(ws.numel()), _stream(stream)), "capmoe_expanded_drop")
    return out


METRICS = {"score": 0, "order": 1, "reverse_order": 2, "random": 3}


def drop_keys(metric: str, seed: int, scores, idx, E: int, stream=None):
    """32-bit drop keys for every entry of scores [N,cols] (idx [N,cols] expert ids, or None for a
    dense [N,E] matrix).  Returned as a float32-typed tensor holding the key bit patterns, so it
    can be passed straight to token_drop / expanded_drop / device_drop in place of the scores."""
    N, cols = scores.shape
    keys = torch.empty((N, cols), device=scores.device, dtype=torch.float32)
    _check(lib().capmoe_drop_keys(METRICS[metric], ctypes.c_uint64(seed), _ptr(scores), _ptr(idx), _i64(N),
                                  int(cols), int(E), _ptr(keys), _stream(stream)), "capmoe_drop_keys")
    return keys


def priority_keys(base, idx, E: int, exact: bool, token_class=None, topk_idx=None, stream=None):
    """Keys with a priority class above the metric's key: 2 * [pair is one of the token's top-k]
    (when topk_idx is given: Expanded Drop as substitution only) + token_class[t] (uint8, 1 = the
    protected modality).  base: the float32-typed key tensor drop_keys returns; same type back."""
    N, cols = base.shape
    keys = torch.empty_like(base)
    k = 0 if topk_idx is None else topk_idx.shape[1]
    _check(lib().capmoe_priority_keys(_ptr(base), _ptr(idx), _i64(N), int(cols), int(E), int(bool(exact)),
                                      _ptr(token_class), _ptr(topk_idx), int(k), _ptr(keys), _stream(stream)),
           "capmoe_priority_keys")
    return keys


def limit_experts(scores, keep_mask, k_max: int, stream=None):
    """'w/ max': edits keep_mask in place so that no token sits on more than k_max experts."""
    N, E = scores.shape
    _check(lib().capmoe_limit_experts(_ptr(scores), _i64(N), int(E), int(k_max), _ptr(keep_mask), _stream(stream)),
           "capmoe_limit_experts")
    return keep_mask


def rows_from_mask(keep_mask, topk_idx, E: int, slots: int, D: int = 1, token_group=None, ws=None, stream=None):
    """-> dict(kept, offsets, slot_row, bad) for a keep mask whose bits lie on the tokens' slots."""
    N, k = topk_idx.shape
    dev = topk_idx.device
    need = ((N + 255) // 256) * E * 4
    if ws is None:
        ws = torch.empty((max(need, 16),), device=dev, dtype=torch.uint8)
    out = dict(kept=torch.empty((E,), device=dev, dtype=torch.int32),
               offsets=torch.empty((E + 1,), device=dev, dtype=torch.int32),
               slot_row=torch.empty((N, slots), device=dev, dtype=torch.int32),
               bad=torch.zeros((1,), device=dev, dtype=torch.int32))
    _check(lib().capmoe_rows_from_mask(_ptr(keep_mask), _ptr(topk_idx), _i64(N), int(E), int(k), int(slots), int(D),
                                       _ptr(token_group), _ptr(out["kept"]), _ptr(out["offsets"]),
                                       _ptr(out["slot_row"]), _ptr(out["bad"]), _ptr(ws),
                                       ctypes.c_size_t(ws.numel()), _stream(stream)), "capmoe_rows_from_mask")
    return out


def device_capacity(N: int, E: int, k: int, D: int, gamma: float, round_mode: str = "ceil") -> int:
    out = ctypes.c_int64(0)
    _check(lib().capmoe_device_capacity(_i64(N), int(E), int(k), int(D), ctypes.c_double(gamma),
                                        0 if round_mode == "ceil" else 1, ctypes.byref(out)),
           "capmoe_device_capacity")
    return out.value


def device_drop(scores, topk_idx, C_dev: int, D: int, expanded: bool, token_group=None, ws=None, stream=None):
    """Capacity per device instead of per expert.  -> dict(keep_mask, cand, kept, offsets, slot_row)"""
    N, E = scores.shape
    k = topk_idx.shape[1]
    dev = scores.device
    if D < 1 or E % D != 0:
        raise CapmoeError(EINVAL, "capmoe_device_drop: E % D != 0")
    m = E // D
    W = (E + 63) // 64
    slots = k + m if expanded else k
    if ws is None:
        ws = torch.empty((drop_workspace_bytes(N, E, k, D, expanded),), device=dev, dtype=torch.uint8)
    out = dict(keep_mask=torch.empty((N, W), device=dev, dtype=torch.int64),
               cand=torch.empty((E,), device=dev, dtype=torch.int32),
               kept=torch.empty((E,), device=dev, dtype=torch.int32),
               offsets=torch.empty((E + 1,), device=dev, dtype=torch.int32),
               slot_row=torch.empty((N, slots), device=dev, dtype=torch.int32))
    _check(lib().capmoe_device_drop(_ptr(scores), _ptr(topk_idx), _i64(N), int(E), int(k), _i64(C_dev), int(D),
                                    int(bool(expanded)), _ptr(token_group), _ptr(out["keep_mask"]),
                                    _ptr(out["cand"]), _ptr(out["kept"]), _ptr(out["offsets"]),
                                    _ptr(out["slot_row"]), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream(stream)),
           "capmoe_device_drop")
    return out


def permute(x, scores, topk_idx, slot_row, A_max: int, D: int = 0, token_group=None, out=None, stream=None):
    """-> dict(x_perm [A_max,d], perm_token [A_max], perm_weight [A_max]); rows >= A are left unwritten.
    `out` may hand in those three buffers to be reused."""
    N, d = x.shape
    E = scores.shape[1]
    k = topk_idx.shape[1]
    slots = slot_row.shape[1]
    dev = x.device
    if out is None:
        out = dict(x_perm=torch.zeros((A_max, d), device=dev, dtype=x.dtype),
                   perm_token=torch.full((A_max,), -1, device=dev, dtype=torch.int32),
                   perm_weight=torch.zeros((A_max,), device=dev, dtype=torch.float32))
    _check(lib().capmoe_permute(_ptr(x), _i64(N), int(d), int(E), int(k), int(slots), int(D), _dt(x),
                                _ptr(scores), _ptr(topk_idx), _ptr(token_group), _ptr(slot_row),
                                _ptr(out["x_perm"]), _ptr(out["perm_token"]), _ptr(out["perm_weight"]),
                                _stream(stream)), "capmoe_permute")
    return out


def grouped_ffn(x_perm, offsets, w_gate, w_up, w_down, D_straggler: int = 0, h_ws=None, y_perm=None,
                dev_status=None, stream=None):
    """-> y_perm [A_max, d].  dev_status: int32 [FFN_STATUS_WORDS] (word 0 = device status), made here if None."""
    A_max, d = x_perm.shape
    E, F, _ = w_gate.shape
    dev = x_perm.device
    if dev_status is None:
        dev_status = torch.zeros((FFN_STATUS_WORDS,), device=dev, dtype=torch.int32)
    if h_ws is None:
        h_ws = torch.empty((A_max, F), device=dev, dtype=x_perm.dtype)
    if y_perm is None:
        y_perm = torch.zeros((A_max, d), device=dev, dtype=x_perm.dtype)
    _check(lib().capmoe_grouped_ffn(_ptr(x_perm), _ptr(offsets), int(E), int(d), int(F), _dt(x_perm),
                                    _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(h_ws), _ptr(y_perm),
                                    _i64(A_max), int(D_straggler), _ptr(dev_status), _stream(stream)),
           "capmoe_grouped_ffn")
    return y_perm


def grouped_ffn_segments(x_rows, seg_begin, seg_end, w_gate, w_up, w_down, w_mod: int, h_ws=None, y_rows=None,
                         dev_status=None, stream=None):
    """SwiGLU FFN over explicit row segments; segment s uses weight block s % w_mod.  -> y_rows"""
    rows, d = x_rows.shape
    F = w_gate.shape[-2]
    dev = x_rows.device
    if dev_status is None:
        dev_status = torch.zeros((FFN_STATUS_WORDS,), device=dev, dtype=torch.int32)
    if h_ws is None:
        h_ws = torch.empty((rows, F), device=dev, dtype=x_rows.dtype)
    if y_rows is None:
        y_rows = torch.zeros((rows, d), device=dev, dtype=x_rows.dtype)
    _check(lib().capmoe_grouped_ffn_segments(_ptr(x_rows), _ptr(seg_begin), _ptr(seg_end), int(seg_begin.numel()),
                                             int(w_mod), int(d), int(F), _dt(x_rows), _ptr(w_gate), _ptr(w_up),
                                             _ptr(w_down), _ptr(h_ws), _ptr(y_rows), _i64(rows), _ptr(dev_status),
                                             _stream(stream)), "capmoe_grouped_ffn_segments")
    return y_rows


# ----------------------------------------------------------------------------- grouped products
# A decode step makes these calls every few microseconds, so they are written for little time on the host: argument
# types are declared once (ints and addresses then pass without ctypes objects), messages are built only on failure.
# `stream=s` is the call under torch.cuda.stream(s): outputs and workspaces made here then belong to s, so that their
# memory is neither still in use by another stream's kernels when the call writes it nor handed on before it is done.
_V, _I, _L, _S = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_ARGTYPES = {
    "capmoe_grouped_mm": [_V, _V, _V, _I, _I, _I, _I, _V, _L, _V, _V],
    "capmoe_grouped_mm_dx": [_V, _V, _V, _I, _I, _I, _I, _V, _L, _V, _V],
    "capmoe_grouped_mm_dw": [_V, _V, _V, _I, _I, _I, _I, _I, _V, _L, _V, _S, _V, _V],
    "capmoe_grouped_ffn_backward": [_V, _V, _V, _I, _I, _I, _I, _V, _V, _V, _V, _V, _V, _V, _L, _V, _S, _V, _V],
    "capmoe_quantize_rows": [_V, _V, _L, _I, _I, _V, _V, _V],
    "capmoe_quantize_weights": [_V, _I, _I, _I, _I, _V, _V, _V],
    "capmoe_grouped_mm_fp8": [_V, _V, _V, _V, _V, _I, _I, _I, _V, _L, _V, _V],
    "capmoe_grouped_ffn_fp8": [_V, _V, _I, _I, _I, _V, _V, _V, _V, _V, _V, _V, _L, _V, _S, _V, _V],
    "capmoe_grouped_ffn_fp8_codes": [_V, _V, _V, _I, _I, _I, _V, _V, _V, _V, _V, _V, _V, _L, _V, _S, _V, _V],
    "capmoe_rms_norm": [_V, _V, _V, _L, _I, _I, ctypes.c_float, _V, _V, _V, _V, _V, _V],
    "capmoe_rms_norm_backward": [_V, _V, _V, _V, _V, _L, _I, _I, _I, _V, _V, _V, _S, _V],
    "capmoe_permute_fp8": [_V, _V, _L, _I, _I, _I, _I, _I, _L, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V],
    "capmoe_combine_backward": [_V, _V, _V, _V, _L, _I, _I, _I, _L, _V, _V, _V],
    "capmoe_permute_backward": [_V, _V, _L, _I, _I, _I, _L, _V, _V, _V, _V],
    "capmoe_route_backward": [_V, _V, _V, _V, _V, _V, _L, _I, _I, _I, _I, _I, _V, _V, _L, _I, _I, _L, _V, _V, _V, _V, _V, _S, _V, _V],
}


def _refuse(where: str, what: str, status: int = EINVAL):
    raise CapmoeError(status, f"{where}: {what}")


_bind = None                # the compiled binding (csrc/bind.cpp), loaded with the library


def _binding():
    """The compiled binding for this interpreter and torch; the operators that match their arguments with it need it."""
    global _bind
    lib()
    path = bind_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2503_05066_b200.build`")
    spec = importlib.util.spec_from_file_location("paper_2503_05066_b200._bind", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    _bind = module
    return _bind


def _run_unbound(name: str, like, *args):
    """The binding's run() by ctypes, for the grouped products where it has not been built for this interpreter and torch."""
    here = like.get_device()
    if any(isinstance(v, torch.Tensor) and (v.get_device() != here or not v.is_contiguous()) for v in args) or here < 0:
        return None
    if here != torch.cuda.current_device():
        return None
    return getattr(lib(), name)(*[v.data_ptr() if isinstance(v, torch.Tensor) else v for v in args], torch.cuda.current_stream(here).cuda_stream)


def _run(name: str, like, *args):
    """Calls entry point `name` with `args` and the current stream; tensors among the arguments pass as their addresses."""
    if _bind is None and not os.path.exists(bind_path()):
        rc = _run_unbound(name, like, *args)
    else:
        rc = (_bind or _binding()).run(name, like, *args)
    if rc:
        raise CapmoeError(rc, name)
    if rc is None:                         # nothing was called
        here = like.get_device()
        for v in args:
            if isinstance(v, torch.Tensor):
                if v.get_device() != here or here < 0:
                    _refuse(name, f"CUDA tensors on one device expected, got {v.device} next to {like.device}")
                assert v.is_contiguous(), "capmoe tensors must be contiguous"
        for sizes in (_dw_bytes, _ffn_backward_bytes, _norm_backward_bytes, _route_backward_bytes):
            sizes.cache_clear()            # the library sized a workspace for the current device, but it is remembered for `here`
        _refuse(name, f"tensors on cuda:{here}, but cuda:{torch.cuda.current_device()} is the current device")


def _bytes(fn, *args) -> int:
    out = ctypes.c_size_t(0)
    _check(getattr(lib(), fn)(*args, ctypes.byref(out)), fn)
    return out.value


def _fits(where: str, *sizes):
    """Sizes that the library takes as C ints, which ctypes would cut to 32 bits."""
    if max(sizes) > 0x7fffffff:
        _refuse(where, f"sizes {sizes} pass 32 bits", EUNSUPPORTED)


def _experts(where: str, offsets) -> int:
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() < 2:
        _refuse(where, "offsets must be int32 [E+1]")
    return offsets.numel() - 1


def _out(where: str, t, shape, dtype, like):
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    if t.shape != shape or t.dtype != dtype:
        _refuse(where, f"output must be {dtype} {tuple(shape)}")
    return t


def _status(where: str, dev_status):
    if dev_status is not None and (dev_status.dtype != torch.int32 or dev_status.numel() < FFN_STATUS_WORDS):
        _refuse(where, f"dev_status must be int32 [{FFN_STATUS_WORDS}]")
    return dev_status


def grouped_mm(x_rows, offsets, w, y=None, dev_status=None, stream=None):
    """y[r] = W[e] x[r] for the rows r of every expert e.  x_rows [rows,d], w [E,n,d] -> y [rows,n]; rows behind
    offsets[E] are left as they are (undefined in a y made here)."""
    where = "capmoe_grouped_mm"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_mm(x_rows, offsets, w, y, dev_status)
    E = _experts(where, offsets)
    if x_rows.dim() != 2 or w.dim() != 3 or w.shape[0] != E or w.shape[2] != x_rows.shape[1] or w.dtype != x_rows.dtype:
        _refuse(where, "x_rows [rows,d] and w [E,n,d] of one dtype expected")
    rows, d = x_rows.shape
    n = w.shape[1]
    _fits(where, E, d, n)
    y = _out(where, y, (rows, n), x_rows.dtype, x_rows)
    _run(where, x_rows, x_rows, offsets, w, E, d, n, _dt(x_rows), y, rows, _status(where, dev_status))
    return y


def grouped_mm_dx(dy_rows, offsets, w, dx=None, dev_status=None, stream=None):
    """Gradient of grouped_mm's rows: dx[r] = W[e]^T dy[r].  dy_rows [rows,n], w [E,n,d] -> dx [rows,d]."""
    where = "capmoe_grouped_mm_dx"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_mm_dx(dy_rows, offsets, w, dx, dev_status)
    E = _experts(where, offsets)
    if dy_rows.dim() != 2 or w.dim() != 3 or w.shape[0] != E or w.shape[1] != dy_rows.shape[1] or w.dtype != dy_rows.dtype:
        _refuse(where, "dy_rows [rows,n] and w [E,n,d] of one dtype expected")
    rows, n = dy_rows.shape
    d = w.shape[2]
    _fits(where, E, d, n)
    dx = _out(where, dx, (rows, d), dy_rows.dtype, dy_rows)
    _run(where, dy_rows, dy_rows, offsets, w, E, d, n, _dt(dy_rows), dx, rows, _status(where, dev_status))
    return dx


def grouped_mm_dw(dy_rows, x_rows, offsets, dw=None, out_dtype=None, ws=None, dev_status=None, stream=None):
    """Gradient of grouped_mm's weights: dW[e] = sum over e's rows of dy[r] x[r]^T, zeros for an expert without rows.
    -> dw [E,n,d] in the rows' dtype, or out_dtype (float32)."""
    where = "capmoe_grouped_mm_dw"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_mm_dw(dy_rows, x_rows, offsets, dw, out_dtype, ws, dev_status)
    E = _experts(where, offsets)
    if (dy_rows.dim() != 2 or x_rows.dim() != 2 or dy_rows.shape[0] != x_rows.shape[0] or dy_rows.dtype != x_rows.dtype):
        _refuse(where, "dy_rows [rows,n] and x_rows [rows,d] of one dtype expected")
    rows, n = dy_rows.shape
    d = x_rows.shape[1]
    _fits(where, E, d, n)
    dw = _out(where, dw, (E, n, d), out_dtype or (dw.dtype if dw is not None else x_rows.dtype), x_rows)
    if ws is None:
        ws = x_rows.new_empty((_dw_bytes(x_rows.get_device(), rows, E, d, n, x_rows.dtype),), dtype=torch.uint8)
    _run(where, x_rows, dy_rows, x_rows, offsets, E, d, n, _dt(x_rows), _dt(dw), dw, rows, ws,
         ws.numel() * ws.element_size(), _status(where, dev_status))
    return dw


def dw_split_bytes(rows: int, E: int, d: int, n: int, dtype, products: int = 1) -> int:
    """What to add to the workspace of grouped_mm_dw (products=1) or grouped_ffn_backward (n=F, products=3) for splitting
    long sums when there are few output tiles; workspaces made inside those calls have it."""
    return _bytes("capmoe_dw_split_bytes", _i64(rows), int(E), int(d), int(n), _dt(dtype), int(products))


def ffn_backward_workspace_bytes(A_max: int, E: int, F: int, dtype) -> int:
    return _bytes("capmoe_ffn_backward_workspace_bytes", _i64(A_max), int(E), int(F), _dt(dtype))


# Sizes of the workspaces that the calls make themselves; the splits depend on the (current) device's SM count.
@functools.lru_cache(maxsize=1024)
def _dw_bytes(device, rows, E, d, n, dtype):
    return _bytes("capmoe_grouped_mm_dw_workspace_bytes", E) + dw_split_bytes(rows, E, d, n, dtype)


@functools.lru_cache(maxsize=1024)
def _ffn_backward_bytes(device, A_max, E, d, F, dtype):
    return ffn_backward_workspace_bytes(A_max, E, F, dtype) + dw_split_bytes(A_max, E, d, F, dtype, 3)


@functools.lru_cache(maxsize=1024)
def _ffn_fp8_bytes(A_max, d, F):
    return ffn_fp8_workspace_bytes(A_max, d, F)


def grouped_ffn_backward(x_perm, dy_perm, offsets, w_gate, w_up, w_down, dx=None, dw=None, ws=None, dev_status=None,
                         stream=None):
    """Gradients of grouped_ffn from its input and the gradient of its output (the hidden activations are recomputed).
    -> (dx [A_max,d], dw_gate [E,F,d], dw_up [E,F,d], dw_down [E,d,F]); `dw` may hand in the last three."""
    where = "capmoe_grouped_ffn_backward"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_ffn_backward(x_perm, dy_perm, offsets, w_gate, w_up, w_down, dx, dw, ws, dev_status)
    E = _experts(where, offsets)
    if (x_perm.dim() != 2 or x_perm.shape != dy_perm.shape or w_gate.dim() != 3 or w_gate.shape[0] != E or
            w_gate.shape[2] != x_perm.shape[1] or w_up.shape != w_gate.shape or
            w_down.shape != (E, w_gate.shape[2], w_gate.shape[1])):
        _refuse(where, "x_perm, dy_perm [A_max,d], w_gate, w_up [E,F,d], w_down [E,d,F] expected")
    dtype = x_perm.dtype
    if dy_perm.dtype != dtype or w_gate.dtype != dtype or w_up.dtype != dtype or w_down.dtype != dtype:
        _refuse(where, "one dtype expected")
    A_max, d = x_perm.shape
    F = w_gate.shape[1]
    _fits(where, E, d, F)
    dx = _out(where, dx, (A_max, d), dtype, x_perm)
    dwg, dwu, dwd = (None, None, None) if dw is None else dw
    dwg = _out(where, dwg, (E, F, d), dtype, x_perm)
    dwu = _out(where, dwu, (E, F, d), dtype, x_perm)
    dwd = _out(where, dwd, (E, d, F), dtype, x_perm)
    if ws is None:
        ws = x_perm.new_empty((_ffn_backward_bytes(x_perm.get_device(), A_max, E, d, F, dtype),), dtype=torch.uint8)
    _run(where, x_perm, x_perm, dy_perm, offsets, E, d, F, _dt(dtype), w_gate, w_up, w_down, dx, dwg, dwu, dwd, A_max, ws,
         ws.numel() * ws.element_size(), _status(where, dev_status))
    return dx, dwg, dwu, dwd


# ----------------------------------------------------------------------------- 8-bit expert products
FP8, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
QBLOCK = 128                # columns of a row (rows and columns of a weight) that share one power-of-two scale


def _blocks(v: int) -> int:
    return (v + QBLOCK - 1) // QBLOCK


def quantize_rows(x, offsets=None, out=None, stream=None):
    """x [rows,d] (float32 or bfloat16) -> (q [rows,d] float8_e4m3fn, scale [rows, ceil(d/128)] float8_e8m0fnu), one
    power-of-two scale per 128 columns.  With offsets [E+1] only the rows below offsets[E] are quantised."""
    where = "capmoe_quantize_rows"
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantize_rows(x, offsets, out)
    if x.dim() != 2:
        _refuse(where, "x [rows,d] expected")
    rows, d = x.shape
    _fits(where, d)
    q, scale = (None, None) if out is None else out
    q = torch.empty_like(x, dtype=FP8) if q is None else _out(where, q, (rows, d), FP8, x)
    scale = _out(where, scale, (rows, _blocks(d)), SCALE, x)
    n_rows = None
    if offsets is not None:
        n_rows = offsets.data_ptr() + 4 * _experts(where, offsets)
        if offsets.get_device() != x.get_device():
            _refuse(where, "offsets must be on x's device")
        assert offsets.is_contiguous(), "capmoe tensors must be contiguous"
    _run(where, x, x, n_rows, rows, d, _dt(x), q, scale)
    return q, scale


def quantize_weights(w, out=None, stream=None):
    """w [E,n,d] -> (q [E,n,d] float8_e4m3fn, scale [E, ceil(n/128), ceil(d/128)] float8_e8m0fnu), one scale per
    128 x 128 block."""
    where = "capmoe_quantize_weights"
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantize_weights(w, out)
    if w.dim() != 3:
        _refuse(where, "w [E,n,d] expected")
    E, n, d = w.shape
    _fits(where, E, n, d)
    q, scale = (None, None) if out is None else out
    q = _out(where, q, (E, n, d), FP8, w)
    scale = _out(where, scale, (E, _blocks(n), _blocks(d)), SCALE, w)
    _run(where, w, w, E, n, d, _dt(w), q, scale)
    return q, scale


def _coded(where: str, q, scale, shape, tall: int):
    want = (*shape[:-2], _blocks(shape[-2]) if tall > 1 else shape[-2], _blocks(shape[-1]))
    if q.dtype != FP8 or q.shape != shape or scale.dtype != SCALE or scale.shape != want:
        _refuse(where, f"float8_e4m3fn {tuple(shape)} with float8_e8m0fnu scales {want} expected")


def grouped_mm_fp8(x_q, x_scale, offsets, w_q, w_scale, y=None, dev_status=None, stream=None):
    """grouped_mm from 8-bit rows (quantize_rows) and weights (quantize_weights) -> y [rows,n] bfloat16."""
    where = "capmoe_grouped_mm_fp8"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_mm_fp8(x_q, x_scale, offsets, w_q, w_scale, y, dev_status)
    E = _experts(where, offsets)
    if x_q.dim() != 2 or w_q.dim() != 3:
        _refuse(where, "x_q [rows,d], w_q [E,n,d] expected")
    rows, d = x_q.shape
    n = w_q.shape[1]
    _fits(where, E, d, n)
    _coded(where, x_q, x_scale, (rows, d), 1)
    _coded(where, w_q, w_scale, (E, n, d), QBLOCK)
    y = _out(where, y, (rows, n), torch.bfloat16, x_q)
    _run(where, x_q, x_q, x_scale, offsets, w_q, w_scale, E, d, n, y, rows, _status(where, dev_status))
    return y


def ffn_fp8_workspace_bytes(A_max: int, d: int, F: int) -> int:
    return _bytes("capmoe_ffn_fp8_workspace_bytes", _i64(A_max), int(d), int(F))


def grouped_ffn_fp8(x_perm, offsets, w_gate, w_up, w_down, y_perm=None, ws=None, dev_status=None, stream=None):
    """grouped_ffn with 8-bit weights, each a (q, scale) pair of quantize_weights; x_perm [A_max,d] bfloat16 and the
    hidden rows are quantised on the way -> y_perm [A_max,d] bfloat16.  x_perm may be a (q, scale) pair itself, as
    quantize_rows or permute_fp8 leave it."""
    where = "capmoe_grouped_ffn_fp8"
    if stream is not None:
        with torch.cuda.stream(stream):
            return grouped_ffn_fp8(x_perm, offsets, w_gate, w_up, w_down, y_perm, ws, dev_status)
    E = _experts(where, offsets)
    x_scale = None
    if isinstance(x_perm, (tuple, list)):
        where = "capmoe_grouped_ffn_fp8_codes"
        x_perm, x_scale = x_perm
    if x_perm.dim() != 2 or (x_scale is None and x_perm.dtype != torch.bfloat16) or w_gate[0].dim() != 3:
        _refuse(where, "x_perm [A_max,d] bfloat16 (or codes and scales) and (q, scale) weights expected")
    A_max, d = x_perm.shape
    F = w_gate[0].shape[1]
    _fits(where, E, d, F)
    rows = (x_perm,)
    if x_scale is not None:
        _coded(where, x_perm, x_scale, (A_max, d), 1)
        rows = (x_perm, x_scale)
    _coded(where, *w_gate, (E, F, d), QBLOCK)
    _coded(where, *w_up, (E, F, d), QBLOCK)
    _coded(where, *w_down, (E, d, F), QBLOCK)
    y_perm = _out(where, y_perm, (A_max, d), torch.bfloat16, x_perm)
    if ws is None:
        ws = x_perm.new_empty((_ffn_fp8_bytes(A_max, d, F),), dtype=torch.uint8)
    _run(where, x_perm, *rows, offsets, E, d, F, *w_gate, *w_up, *w_down, y_perm, A_max, ws,
         ws.numel() * ws.element_size(), _status(where, dev_status))
    return y_perm


# ----------------------------------------------------------------------------- the norm in front of the layer
def _want(where: str, name: str, t, shape, dtype):
    if t is not None and (t.shape != shape or t.dtype != dtype):
        _refuse(where, f"{name} must be {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t


def _no_fit(where: str, x):
    """The last refusal of arguments that do not fit together: the rows' type, or else the sizes."""
    _dt(x.dtype)
    _refuse(where, "types or sizes of the arguments do not fit together")


def rms_norm(x, w, residual=None, eps: float = 1e-6, fp8: bool = False, out=None, stream=None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * w by rows.  x, residual [N,d], w [d] -> dict(y, h, rstd [N] float32), h
    being x itself without a residual; with fp8 also q, scale: the codes that quantize_rows makes of y.  `out` may hand in any
    of these buffers (h may be x's or residual's)."""
    where = "capmoe_rms_norm"
    if stream is not None:
        with torch.cuda.stream(stream):
            return rms_norm(x, w, residual, eps, fp8, out)
    bind = _bind or _binding()
    fit = bind.match("T[N,d] T[d] T?[N,d]", x, w, residual)
    if fit is None:
        if x.dim() != 2 or w.dim() != 1 or w.shape[0] != x.shape[1] or w.dtype != x.dtype:
            _refuse(where, "x [N,d] and w [d] of one dtype expected")
        _want(where, "residual", residual, x.shape, x.dtype)
        _no_fit(where, x)
    code, N, d = fit
    r = dict(h=x)
    if out is None:                           # (allocations are most of the call's time: the cheapest form of each)
        new = bind.new
        r["y"] = y = new(x, None)
        r["rstd"] = rstd = new(x, torch.float32, N)
        if residual is not None:
            r["h"] = new(x, None)
        if fp8:
            r["q"], r["scale"] = new(x, FP8), new(x, SCALE, N, _blocks(d))
    else:
        shape, dtype = x.shape, x.dtype
        r["y"] = y = _out(where, out.get("y"), shape, dtype, x)
        r["rstd"] = rstd = _out(where, out.get("rstd"), (N,), torch.float32, x)
        if residual is not None:
            r["h"] = _out(where, out.get("h"), shape, dtype, x)
        if fp8:
            r["q"], r["scale"] = _out(where, out.get("q"), shape, FP8, x), _out(where, out.get("scale"), (N, _blocks(d)), SCALE, x)
    _run(where, x, x, residual, w, N, d, code, eps, None if residual is None else r["h"], y, rstd, r.get("q"), r.get("scale"))
    return r


@functools.lru_cache(maxsize=1024)
def _norm_backward_bytes(device, N, d, code):
    _fits("capmoe_rms_norm_backward", d)
    return _bytes("capmoe_rms_norm_backward_workspace_bytes", _i64(N), d, code)


def rms_norm_backward_workspace_bytes(N: int, d: int, dtype) -> int:
    return _bytes("capmoe_rms_norm_backward_workspace_bytes", _i64(N), int(d), _dt(dtype))


def rms_norm_backward(dy, h, w, rstd, dh=None, dx=None, dw=None, out_dtype=None, ws=None, stream=None):
    """Gradients of rms_norm from dy, the h and rstd that it returned and dh, what reaches h from behind (or None).
    -> (dx [N,d], the gradient of x and of the residual alike, dw [d] in the rows' dtype, or out_dtype (float32))."""
    where = "capmoe_rms_norm_backward"
    if stream is not None:
        with torch.cuda.stream(stream):
            return rms_norm_backward(dy, h, w, rstd, dh, dx, dw, out_dtype, ws)
    bind = _bind or _binding()
    fit = bind.match("T[N,d] T[d] T[N,d] f[N] T?[N,d]", h, w, dy, rstd, dh)
    if fit is None:
        if h.dim() != 2 or w.dim() != 1 or w.shape[0] != h.shape[1] or w.dtype != h.dtype:
            _refuse(where, "h [N,d] and w [d] of one dtype expected")
        _want(where, "dy", dy, h.shape, h.dtype)
        _want(where, "dh", dh, h.shape, h.dtype)
        _want(where, "rstd", rstd, h.shape[:1], torch.float32)
        _no_fit(where, h)
    code, N, d = fit
    dx = bind.new(h, None) if dx is None else _out(where, dx, h.shape, h.dtype, h)
    if dw is None:
        dw = bind.new(w, out_dtype)
    else:
        _out(where, dw, (d,), out_dtype or dw.dtype, h)
    if ws is None:
        size = _norm_backward_bytes(h.get_device(), N, d, code)
        ws = bind.new(h, torch.uint8, size)
    else:
        size = ws.numel() * ws.element_size()
    _run(where, h, dy, h, w, rstd, dh, N, d, code, _dt(dw) if out_dtype or dw.dtype != h.dtype else code, dx, dw, ws, size)
    return dx, dw


# ----------------------------------------------------------------------------- permute in 8 bits; gradients of combine, permute, route
def _slot_rows(where: str, slot_row, N: int):
    if slot_row.dtype != torch.int32 or slot_row.dim() != 2 or slot_row.shape[0] != N:
        _refuse(where, "slot_row must be int32 [N,slots]")


def _route_lists(where: str, scores, topk_idx, slot_row, token_group):
    """Refuses what the route and drop stages do not leave; -> N."""
    if scores.dim() != 2 or scores.dtype != torch.float32 or topk_idx.dim() != 2 or topk_idx.dtype != torch.int32:
        _refuse(where, "scores [N,E] float32 and topk_idx [N,k] int32 expected")
    N = scores.shape[0]
    if topk_idx.shape[0] != N:
        _refuse(where, "scores and topk_idx of one number of tokens expected")
    _want(where, "token_group", token_group, (N,), torch.int32)
    _slot_rows(where, slot_row, N)
    return N


def permute_fp8(x_q, x_scale, scores, topk_idx, slot_row, A_max: int, D: int = 0, token_group=None, out=None, dev_status=None, stream=None):
    """permute of 8-bit rows (rms_norm(fp8=True), quantize_rows).  -> dict(x_q [A_max,d], x_scale [A_max, ceil(d/128)],
    perm_token [A_max], perm_weight [A_max]); rows >= A are left unwritten.  `out` may hand in those buffers."""
    where = "capmoe_permute_fp8"
    if stream is not None:
        with torch.cuda.stream(stream):
            return permute_fp8(x_q, x_scale, scores, topk_idx, slot_row, A_max, D, token_group, out, dev_status)
    bind = _bind or _binding()
    fit = bind.match("q[N,d] s[N,B] f[N,E] i[N,k] i[N,s] i?[N]", x_q, x_scale, scores, topk_idx, slot_row, token_group)
    if fit is None:
        N = _route_lists(where, scores, topk_idx, slot_row, token_group)
        if x_q.dim() != 2 or x_q.shape[0] != N:
            _refuse(where, "x_q [N,d] expected")
        _refuse(where, f"float8_e4m3fn [N,d] with float8_e8m0fnu scales {(N, _blocks(x_q.shape[1]))} expected")
    _, N, d, E, k, slots = fit
    nb = _blocks(d)
    if out is None:
        new = bind.new
        r = dict(x_q=new(x_q, FP8, A_max, d), x_scale=new(x_q, SCALE, A_max, nb), perm_token=new(x_q, torch.int32, A_max),
                 perm_weight=new(x_q, torch.float32, A_max))
    else:
        r = dict(x_q=_out(where, out.get("x_q"), (A_max, d), FP8, x_q), x_scale=_out(where, out.get("x_scale"), (A_max, nb), SCALE, x_q),
                 perm_token=_out(where, out.get("perm_token"), (A_max,), torch.int32, x_q),
                 perm_weight=_out(where, out.get("perm_weight"), (A_max,), torch.float32, x_q))
    _run(where, x_q, x_q, x_scale, N, d, E, k, slots, D, A_max, scores, topk_idx, token_group, slot_row, r["x_q"], r["x_scale"],
         r["perm_token"], r["perm_weight"], _status(where, dev_status))
    return r


def combine_backward(dy, y_perm, slot_row, perm_weight, dy_perm=None, dweight=None, stream=None):
    """Gradients of combine: dy_perm[r] = perm_weight[r] dy[t], dweight[r] = dy[t] . y_perm[r] for the row r of a slot of t.
    dy [N,d], y_perm [A_max,d] -> (dy_perm [A_max,d], dweight [A_max] float32); rows that no slot names are left as they are
    (undefined in buffers made here).  The gradient of y_shared is dy."""
    where = "capmoe_combine_backward"
    if stream is not None:
        with torch.cuda.stream(stream):
            return combine_backward(dy, y_perm, slot_row, perm_weight, dy_perm, dweight)
    bind = _bind or _binding()
    fit = bind.match("T[N,d] T[A,d] i[N,s] f[A]", dy, y_perm, slot_row, perm_weight)
    if fit is None:
        if dy.dim() != 2 or y_perm.dim() != 2 or y_perm.shape[1] != dy.shape[1] or y_perm.dtype != dy.dtype:
            _refuse(where, "dy [N,d] and y_perm [A_max,d] of one dtype expected")
        _slot_rows(where, slot_row, dy.shape[0])
        _want(where, "perm_weight", perm_weight, y_perm.shape[:1], torch.float32)
        _no_fit(where, dy)
    code, N, d, A_max, slots = fit
    dy_perm = bind.new(y_perm, None) if dy_perm is None else _out(where, dy_perm, y_perm.shape, dy.dtype, dy)
    dweight = bind.new(perm_weight, None) if dweight is None else _out(where, dweight, (A_max,), torch.float32, dy)
    _run(where, dy, dy, y_perm, slot_row, perm_weight, N, d, slots, code, A_max, dy_perm, dweight)
    return dy_perm, dweight


def permute_backward(dx_perm, slot_row, add=None, dx=None, stream=None):
    """Gradient of permute: dx[t] = sum of dx_perm over t's rows, plus `add`, a tensor [N,d] or up to two of them (what reaches
    x through the router or a shared expert).  dx_perm [A_max,d] -> dx [N,d], which may be one of `add`."""
    where = "capmoe_permute_backward"
    if stream is not None:
        with torch.cuda.stream(stream):
            return permute_backward(dx_perm, slot_row, add, dx)
    bind = _bind or _binding()
    add0 = add1 = None
    if add is not None:
        add = (add,) if isinstance(add, torch.Tensor) else tuple(add)
        if len(add) > 2:
            _refuse(where, "at most two tensors to add", EUNSUPPORTED)
        add0, add1 = (add + (None, None))[:2]
    fit = bind.match("T[A,d] i[N,s] T?[N,d] T?[N,d]", dx_perm, slot_row, add0, add1)
    if fit is None:
        if dx_perm.dim() != 2:
            _refuse(where, "dx_perm [A_max,d] expected")
        N = slot_row.shape[0] if slot_row.dim() else 0
        _slot_rows(where, slot_row, N)
        for t in (add0, add1):
            _want(where, "add", t, (N, dx_perm.shape[1]), dx_perm.dtype)
        _no_fit(where, dx_perm)
    code, A_max, d, N, slots = fit
    dx = bind.new(dx_perm, None, N, d) if dx is None else _out(where, dx, (N, d), dx_perm.dtype, dx_perm)
    _run(where, dx_perm, dx_perm, slot_row, N, d, slots, code, A_max, add0, add1, dx)
    return dx


@functools.lru_cache(maxsize=1024)
def _route_backward_bytes(device, N, d, E, code):
    _fits("capmoe_route_backward", d, E)
    return _bytes("capmoe_route_backward_workspace_bytes", _i64(N), d, E, code)


def route_backward_workspace_bytes(N: int, d: int, E: int, dtype) -> int:
    return _bytes("capmoe_route_backward_workspace_bytes", _i64(N), int(d), int(E), _dt(dtype))


def route_backward(x, w_router, scores, topk_idx, slot_row, dweight, D: int = 0, token_group=None, dscores=None, out=None, out_dtype=None,
                   ws=None, dev_status=None, stream=None):
    """Gradients of route from dweight [A_max], the gradient of the kept pairs' weights (combine_backward), and dscores, what
    the scores get besides: [N,E], or [E] for all tokens (a balance loss), or None.  -> dict(dlogits [N,E] float32, dx [N,d],
    dw [E,d] in the rows' dtype, or out_dtype (float32), dbias [E] float32); `out` may hand in any of them."""
    where = "capmoe_route_backward"
    if stream is not None:
        with torch.cuda.stream(stream):
            return route_backward(x, w_router, scores, topk_idx, slot_row, dweight, D, token_group, dscores, out, out_dtype, ws, dev_status)
    bind = _bind or _binding()
    fit = bind.match("T[N,d] T[E,d] f[N,E] i[N,k] i[N,s] f[A] i?[N]", x, w_router, scores, topk_idx, slot_row, dweight, token_group)
    if fit is None:
        N = _route_lists(where, scores, topk_idx, slot_row, token_group)
        if x.dim() != 2 or x.shape[0] != N or w_router.shape != (scores.shape[1], x.shape[1]) or w_router.dtype != x.dtype:
            _refuse(where, "x [N,d] and w_router [E,d] of one dtype expected")
        if dweight.dtype != torch.float32 or dweight.dim() != 1:
            _refuse(where, "dweight must be float32 [A_max]")
        _no_fit(where, x)
    code, N, d, E, k, slots, A_max = fit
    ld = 0
    if dscores is not None:
        if dscores.dim() == 2:
            ld = E
        _want(where, "dscores", dscores, (N, E) if ld else (E,), torch.float32)
    new = bind.new
    if out is None:
        r = dict(dlogits=new(scores, None), dx=new(x, None), dw=new(w_router, out_dtype), dbias=new(x, torch.float32, E))
    else:
        dw, dtype = out.get("dw"), x.dtype
        r = dict(dlogits=_out(where, out.get("dlogits"), (N, E), torch.float32, x), dx=_out(where, out.get("dx"), (N, d), dtype, x),
                 dw=_out(where, dw, (E, d), out_dtype or (dw.dtype if dw is not None else dtype), x),
                 dbias=_out(where, out.get("dbias"), (E,), torch.float32, x))
    if ws is None:
        size = _route_backward_bytes(x.get_device(), N, d, E, code)
        ws = new(x, torch.uint8, size)
    else:
        size = ws.numel() * ws.element_size()
    _run(where, x, x, w_router, scores, topk_idx, slot_row, dweight, N, d, E, k, slots, D, token_group, dscores, ld, code, code if out_dtype is None and out is None else _dt(r["dw"]),
         A_max, r["dlogits"], r["dx"], r["dw"], r["dbias"], ws, size, _status(where, dev_status))
    return r


# ----------------------------------------------------------------------------- expert parallelism
def ep_plan(slot_row, topk_idx, offsets, E: int, C_local: int, D: int = 1, token_group=None, stream=None):
    """-> (slot_row_ep [N,slots], bad [1]): rows of the [E][C_local] space of an expert-parallel rank."""
    N, slots = slot_row.shape
    k = topk_idx.shape[1]
    out = torch.empty_like(slot_row)
    bad = torch.zeros((1,), device=slot_row.device, dtype=torch.int32)
    _check(lib().capmoe_ep_plan(_ptr(slot_row), _ptr(topk_idx), _ptr(offsets), _i64(N), int(E), int(k), int(slots),
                                int(D), _ptr(token_group), _i64(C_local), _ptr(out), _ptr(bad), _stream(stream)),
           "capmoe_ep_plan")
    return out, bad


def ep_segments(counts, C_local: int, stream=None):
    """counts [S] int32 -> (seg_begin, seg_end) of the S fixed-place segments of C_local rows each."""
    S = counts.numel()
    b, e = torch.empty_like(counts), torch.empty_like(counts)
    _check(lib().capmoe_ep_segments(_ptr(counts), int(S), _i64(C_local), _ptr(b), _ptr(e), _stream(stream)),
           "capmoe_ep_segments")
    return b, e


def ep_dispatch(x, scores, topk_idx, slot_row_ep, peer_rows, R: int, rank: int, C_local: int, D: int = 0,
                token_group=None, out=None, stream=None):
    """Permute with every kept row stored into its owner's buffer (peer_rows: int64 tensor of R base
    addresses on the device).  -> dict(perm_token, perm_weight) of the local [E*C_local] row space."""
    N, d = x.shape
    E = scores.shape[1]
    k = topk_idx.shape[1]
    slots = slot_row_ep.shape[1]
    if out is None:
        out = dict(perm_token=torch.full((max(E * C_local, 1),), -1, device=x.device, dtype=torch.int32),
                   perm_weight=torch.zeros((max(E * C_local, 1),), device=x.device, dtype=torch.float32))
    _check(lib().capmoe_ep_dispatch(_ptr(x), _i64(N), int(d), int(E), int(k), int(slots), int(D), _dt(x), _ptr(scores),
                                    _ptr(topk_idx), _ptr(token_group), _ptr(slot_row_ep), _ptr(peer_rows), int(R),
                                    int(rank), _i64(C_local), _ptr(out["perm_token"]), _ptr(out["perm_weight"]),
                                    _stream(stream)), "capmoe_ep_dispatch")
    return out


def ep_combine(peer_rows, R: int, rank: int, E: int, C_local: int, slot_row_ep, perm_weight, d: int, dtype,
               y_shared=None, y=None, stream=None):
    """Combine with every kept row's result read from its owner's buffer (peer_rows as in ep_dispatch)."""
    N, slots = slot_row_ep.shape
    if y is None:
        y = torch.empty((N, d), device=slot_row_ep.device, dtype=dtype)
    _check(lib().capmoe_ep_combine(_ptr(peer_rows), int(R), int(rank), int(E), _i64(C_local), _ptr(slot_row_ep),
                                   _ptr(perm_weight), _i64(N), int(d), int(slots), _dt(dtype), _ptr(y_shared), _ptr(y),
                                   _stream(stream)), "capmoe_ep_combine")
    return y


EP_MODES = {"nodrop": 0, "token_drop": 1, "expanded_drop": 2}


def ep_rank_struct(**fields) -> _EPRank:
    """capmoe_ep_rank from tensors (device pointers taken), ints and None."""
    P = _EPRank()
    for name, v in fields.items():
        if isinstance(v, torch.Tensor):
            assert v.is_contiguous()
            v = v.data_ptr()
        elif v is None:
            v = 0
        setattr(P, name, v)
    return P


def ep_forward_dispatch(P: _EPRank, stream=None):
    _check(lib().capmoe_ep_forward_dispatch(ctypes.byref(P), _stream(stream)), "ep_forward_dispatch")


def ep_forward_experts(P: _EPRank, stream=None):
    _check(lib().capmoe_ep_forward_experts(ctypes.byref(P), _stream(stream)), "ep_forward_experts")


def ep_forward_combine(P: _EPRank, stream=None):
    _check(lib().capmoe_ep_forward_combine(ctypes.byref(P), _stream(stream)), "ep_forward_combine")


def combine(y_perm, slot_row, perm_weight, y_shared=None, y=None, stream=None):
    """-> y [N, d]"""
    N, slots = slot_row.shape
    d = y_perm.shape[1]
    if y is None:
        y = torch.empty((N, d), device=slot_row.device, dtype=y_perm.dtype)
    _check(lib().capmoe_combine(_ptr(y_perm), _ptr(slot_row), _ptr(perm_weight), _i64(N), int(d), int(slots),
                                _dt(y_perm), _ptr(y_shared), _ptr(y), _stream(stream)), "capmoe_combine")
    return y


def debug_check_indices(slot_row, topk_idx, offsets, E: int, A_max: int, D: int = 1, token_group=None, stream=None):
    """Runs the index check; returns the device status it produced (OK or EINDEX)."""
    N, slots = slot_row.shape
    k = topk_idx.shape[1]
    st = torch.zeros((1,), device=slot_row.device, dtype=torch.int32)
    _check(lib().capmoe_debug_check_indices(_ptr(slot_row), _ptr(topk_idx), _ptr(offsets), _i64(N), int(E), int(k),
                                            int(slots), int(D), _ptr(token_group), _i64(A_max), _ptr(st), _stream(stream)),
           "capmoe_debug_check_indices")
    return int(st.item())


FFN_VARIANTS = {"auto": 0, "pair": 1, "single": 2, "short": 3, "short_down": 4}


def debug_ffn_variant(name: str):
    """Forces one tensor-core FFN kernel for the whole process ("auto" restores the choice by shape)."""
    _check(lib().capmoe_debug_ffn_variant(FFN_VARIANTS[name]), "debug_ffn_variant")


def debug_read_probe(t: torch.Tensor, stream=None):
    """One plain pass of loads over the tensor's bytes (the one-shot read floor of that size)."""
    _check(lib().capmoe_debug_read_probe(_ptr(t), ctypes.c_size_t(t.numel() * t.element_size()), ctypes.c_void_p(0),
                                         _stream(stream)), "capmoe_debug_read_probe")


def debug_wait_probe(limit_cycles: int = 50_000_000, stream=None) -> int:
    """Runs the bounded-wait self-test; returns the device status it produced (ETIMEOUT expected)."""
    st = torch.zeros((1,), device="cuda", dtype=torch.int32)
    _check(lib().capmoe_debug_wait_probe(_i64(limit_cycles), _ptr(st), _stream(stream)), "capmoe_debug_wait_probe")
    torch.cuda.synchronize()
    return int(st.item())


# ----------------------------------------------------------------------------- whole layer
class MoELayer:
    """Device buffers for one layer plus the C struct that names them.  `forward()` enqueues
    capmoe_layer_forward; `forward_host()` enqueues the host-buffer variant."""

    def __init__(self, x, w_router, bias, w_gate, w_up, w_down, k: int, D: int, mode: str, gamma: float = 1.0,
                 straggler: bool = False, shared=None, round_mode: str = "ceil", C: Optional[int] = None,
                 metric: str = "score", seed: int = 0, token_class=None, topk_first: bool = False,
                 max_experts: int = 0, debug_checks: bool = False):
        """Variants of the drop (token_drop / expanded_drop modes): `metric` ranks candidates by Score, Order,
        Reverse Order or Random; `token_class` (uint8 [N], 1 = protected modality) drops the other modality
        first; `topk_first` lets the expansion only fill spare capacity; `max_experts` > 0 is 'w/ max'."""
        dev = x.device
        N, d = x.shape
        E, F, _ = w_gate.shape
        self.N, self.d, self.E, self.k, self.F, self.D = N, d, E, k, F, D
        self.mode = mode
        m = E // D
        expanded = mode in ("expanded_drop", "device_expanded_drop")
        device_level = mode.startswith("device_")
        if C is None:
            if mode == "nodrop":
                C = N
            elif device_level:
                C = device_capacity(N, E, k, D, gamma, round_mode)
            else:
                C = capacity(N, E, k, gamma, round_mode)
        self.C = C
        self.slots = k + m if expanded else k
        A_max = device_max_rows(N, E, k, D, C, expanded) if device_level else max_rows(N, E, k, D, C, expanded)
        self.A_max = A_max
        W = (E + 63) // 64
        f32 = dict(device=dev, dtype=torch.float32)
        i32 = dict(device=dev, dtype=torch.int32)
        act = dict(device=dev, dtype=x.dtype)
        t = self.t = {}
        t["x"], t["w_router"], t["bias"] = x, w_router, bias
        t["w_gate"], t["w_up"], t["w_down"] = w_gate, w_up, w_down
        t["logits"] = torch.empty((N, E), **f32)
        t["scores"] = torch.empty((N, E), **f32)
        t["topk_idx"] = torch.empty((N, k), **i32)
        t["topk_score"] = torch.empty((N, k), **f32)
        t["load"] = torch.empty((E,), **i32)
        t["keep_mask"] = torch.empty((N, W), device=dev, dtype=torch.int64)
        t["cand"] = torch.zeros((E,), **i32)
        t["kept"] = torch.empty((E,), **i32)
        t["expert_offsets"] = torch.empty((E + 1,), **i32)
        t["slot_row"] = torch.empty((N, self.slots), **i32)
        t["x_perm"] = torch.zeros((max(A_max, 1), d), **act)
        t["perm_token"] = torch.full((max(A_max, 1),), -1, **i32)
        t["perm_weight"] = torch.zeros((max(A_max, 1),), **f32)
        t["h_ws"] = torch.empty((max(A_max, 1), F), **act)
        t["y_perm"] = torch.zeros((max(A_max, 1), d), **act)
        t["y"] = torch.empty((N, d), **act)
        t["drop_ws"] = torch.empty((drop_workspace_bytes(N, E, k, D, expanded),), device=dev, dtype=torch.uint8)
        t["dev_status"] = torch.zeros((FFN_STATUS_WORDS,), **i32)
        F_shared = 0
        if shared is not None:
            t["ws_gate"], t["ws_up"], t["ws_down"] = shared
            F_shared = shared[0].shape[-2]
            t["hs_ws"] = torch.empty((N, F_shared), **act)
            t["y_shared"] = torch.empty((N, d), **act)
            t["one_segment"] = torch.tensor([0, N], **i32)
        keyed = metric != "score" or token_class is not None or (topk_first and mode == "expanded_drop")
        if keyed or max_experts > 0:
            if mode not in ("token_drop", "expanded_drop"):
                raise ValueError("drop variants apply to the token_drop and expanded_drop modes")
        if keyed:
            t["drop_keys"] = torch.empty((N, E if expanded else k), **f32)
        if token_class is not None:
            assert token_class.dtype == torch.uint8 and token_class.shape == (N,)
            t["token_class"] = token_class
        if max_experts > 0:
            t["bad"] = torch.zeros((1,), **i32)
        L = self.c = _Layer()
        L.metric, L.metric_seed, L.topk_first, L.max_experts = METRICS[metric], seed, int(bool(topk_first)), max_experts
        L.debug_checks = int(bool(debug_checks))
        L.N, L.d, L.E, L.k, L.F, L.D, L.dtype = N, d, E, k, F, D, _dt(x)
        L.mode, L.C, L.straggler = MODES[mode], C, int(bool(straggler))
        L.F_shared, L.A_max = F_shared, A_max
        L.drop_ws_bytes = t["drop_ws"].numel()
        for name, _typ in _Layer._fields_:
            if name in t:
                assert t[name].is_contiguous()
                setattr(L, name, t[name].data_ptr())

    def set_stage_events(self, events):
        """events: None, or N_STAGE_EVENTS recorded torch.cuda.Event(enable_timing=True) objects."""
        if events is None:
            self.c.stage_events = ctypes.POINTER(ctypes.c_void_p)()
            self._ev = None
            return
        assert len(events) == N_STAGE_EVENTS
        arr = (ctypes.c_void_p * N_STAGE_EVENTS)(*[ctypes.c_void_p(e.cuda_event) for e in events])
        self._ev = (arr, events)
        self.c.stage_events = ctypes.cast(arr, ctypes.POINTER(ctypes.c_void_p))

    def forward(self, stream=None):
        _check(lib().capmoe_layer_forward(ctypes.byref(self.c), _stream(stream)), "capmoe_layer_forward")
        return self.t["y"]

    def capture_graph(self):
        """Records one forward into a CUDA graph (stage events off), so that `replay()` re-issues the
        whole layer with one launch call.  Run `forward()` at least once before: kernels are loaded on
        their first launch, which a capture does not allow.  Buffers and shapes are frozen."""
        self.set_stage_events(None)
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream(device=self.t["x"].device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            self.forward()
        self._graph = graph
        return graph

    def replay(self):
        self._graph.replay()
        return self.t["y"]

    def forward_host(self, x_host: torch.Tensor, y_host: torch.Tensor, stream=None):
        assert x_host.is_pinned() and y_host.is_pinned() and x_host.is_contiguous() and y_host.is_contiguous()
        _check(lib().capmoe_layer_forward_host(ctypes.byref(self.c), ctypes.c_void_p(x_host.data_ptr()),
                                               ctypes.c_void_p(y_host.data_ptr()), _stream(stream)),
               "capmoe_layer_forward_host")
        return y_host

    def backward(self, dy, dscores=None, out_dtype=None, stream=None):
        """Gradients of the layer's last forward() from dy [N,d], the gradient of y, and dscores ([N,E] or [E]), what the router's
        scores get besides (a balance loss).  The forward's buffers must be as it left them.  -> dict(dx [N,d], dw_router, dbias,
        dw_gate, dw_up, dw_down, dlogits, and for a shared expert dws_gate, dws_up, dws_down); the router's weights' gradient in
        out_dtype (float32) or the activations' dtype.  The parts of dx that come through the router and the shared expert are rounded to
        the activations' dtype before they are added up with the experts' (in fp32): half a step of each part."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dy, dscores, out_dtype)
        t = self.t
        status = t["dev_status"]
        dy_perm, dweight = combine_backward(dy, t["y_perm"], t["slot_row"], t["perm_weight"])
        dx_perm, dwg, dwu, dwd = grouped_ffn_backward(t["x_perm"], dy_perm, t["expert_offsets"], t["w_gate"], t["w_up"], t["w_down"],
                                                      dev_status=status)
        r = route_backward(t["x"], t["w_router"], t["scores"], t["topk_idx"], t["slot_row"], dweight,
                           D=self.D if self.slots > self.k else 0, dscores=dscores, out_dtype=out_dtype, dev_status=status)
        g = dict(dw_router=r["dw"], dbias=r["dbias"], dw_gate=dwg, dw_up=dwu, dw_down=dwd, dlogits=r["dlogits"])
        add = (r["dx"],)
        if "ws_gate" in t:
            d = t["x"].shape[1]
            wg, wu, wd = t["ws_gate"].view(1, -1, d), t["ws_up"].view(1, -1, d), t["ws_down"].view(1, d, -1)
            dxs, dsg, dsu, dsd = grouped_ffn_backward(t["x"], dy, t["one_segment"], wg, wu, wd, dev_status=status)
            g.update(dws_gate=dsg.view_as(t["ws_gate"]), dws_up=dsu.view_as(t["ws_up"]), dws_down=dsd.view_as(t["ws_down"]))
            add += (dxs,)
        g["dx"] = permute_backward(dx_perm, t["slot_row"], add=add, dx=r["dx"])
        return g

    def check_device_status(self):
        s = int(self.t["dev_status"][0].item())
        if s != OK:
            raise CapmoeError(s, "device status")

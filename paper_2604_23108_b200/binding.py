"""ctypes binding of libmohge.so: same names and argument order as include/mohge.h.

Only argument marshalling happens here (tensor -> device pointer); every step
of the layer runs in the CUDA library.  There is no fallback: if the shared
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import math
import operator
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

MAX_GROUPS = 8
BF16, F32 = 0, 1
_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmohge.so")


class MohgeError(RuntimeError):
    pass


class mohge_config(C.Structure):
    _fields_ = [
        ("d_model", C.c_int32), ("n_groups", C.c_int32), ("experts_per_group", C.c_int32),
        ("k_groups", C.c_int32), ("k_experts", C.c_int32),
        ("group_width", C.c_int32 * MAX_GROUPS), ("dtype", C.c_int32),
        ("alpha_g", C.c_float), ("alpha_e", C.c_float), ("eps", C.c_float),
        ("f_norm_by_T", C.c_int32), ("fe_mode", C.c_int32), ("row_align", C.c_int32),
    ]


_lib = None

_P = C.c_void_p
_SIGS = {
    "mohge_launch_count": (C.c_int64, []),
    "mohge_workspace_bytes": (C.c_int64, [C.POINTER(mohge_config), C.c_int64]),
    "mohge_perm_rows": (C.c_int64, [C.POINTER(mohge_config), C.c_int64]),
    "mohge_workspace_init": (C.c_int32, [C.POINTER(mohge_config), C.c_int64, _P, C.c_int64, _P]),
    "mohge_get_switch": (C.c_int32, [C.c_char_p]),
    "mohge_set_switch": (C.c_int32, [C.c_char_p, C.c_int32]),
    "mohge_map_cache_stats": (None, [C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "mohge_get_device_status": (C.c_int32, [_P, C.POINTER(C.c_int32), _P]),
    "mohge_route": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 12),
    "mohge_aux_stats": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 12),
    "mohge_aux_stats_static": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 11),
    "mohge_dispatch": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 11),
    "mohge_expert_fwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 10),
    "mohge_combine": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 6),
    "mohge_combine_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 9),
    "mohge_expert_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 12
                         + [C.c_int32, _P, _P]),
    "mohge_expert_bwd_dgate": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 12
                               + [C.c_int32] + [_P] * 7),
    "mohge_dispatch_indices": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 10),
    "mohge_expert_fwd_gather": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 11),
    "mohge_expert_bwd_gather": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 13
                                + [C.c_int32] + [_P] * 7),
    "mohge_row_tokens": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 6),
    "mohge_expert_bwd_dy": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 13
                            + [C.c_int32] + [_P] * 8),
    "mohge_dispatch_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 5),
    "mohge_shared_fwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64, C.c_int32] + [_P] * 8),
    "mohge_shared_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64, C.c_int32] + [_P] * 10
                         + [C.c_int32, _P, _P]),
    "mohge_route_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 14),
    "mohge_mx8_pitch": (C.c_int64, [C.c_int64]),
    "mohge_mx8_tiled_bytes": (C.c_int64, [C.c_int64] * 3),
    "mohge_norm_fwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 3 + [C.c_float] + [_P] * 6),
    "mohge_w4_packed_bytes": (C.c_int64, [C.c_int64, C.c_int64, C.c_int32, C.c_int32]),
    "mohge_quantize_w4": (C.c_int32, [C.c_int64] + [C.c_int32] * 3 + [_P] * 4),
    "mohge_pack_w4": (C.c_int32, [C.c_int64, C.c_int64] + [C.c_int32] * 3 + [_P] * 4),
    "mohge_w4_scratch_bytes": (C.c_int64, [C.POINTER(mohge_config), C.c_int64]),
    "mohge_expert_fwd_w4": (C.c_int32, [C.POINTER(mohge_config), C.c_int64, C.c_int32] + [_P] * 10),
    "mohge_quantize_mx8": (C.c_int32, [C.c_int64, C.c_int64, C.c_int32, C.c_int32] + [_P] * 4),
    "mohge_permute_mx8": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 6),
    "mohge_expert_fwd_mx8": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 13),
    "mohge_norm_bwd": (C.c_int32, [C.POINTER(mohge_config), C.c_int64] + [_P] * 7 + [C.c_int32, _P, _P]),
}


def lib():
    """Loads libmohge.so (built by paper_2604_23108_b200.build); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MohgeError("libmohge.so is not built: run `python -m paper_2604_23108_b200.build`")
        L = C.CDLL(LIB_PATH)
        L.mohge_last_error.restype = C.c_char_p
        L.mohge_last_error.argtypes = []
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def exported_symbols() -> List[str]:
    return ["mohge_last_error"] + list(_SIGS)


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise MohgeError("%s failed (%d): %s" % (what, rc, lib().mohge_last_error().decode()))


def _require(cond: bool, fmt: str, *args) -> None:
    if not cond:
        raise MohgeError(fmt % args)


def _require_bytes(what: str, t: torch.Tensor, n: int) -> None:
    have = t.numel() * t.element_size()
    _require(have >= n, "%s holds %d bytes, %d are written or read", what, have, n)


def _dtype_code(t: torch.Tensor, what: str) -> int:
    """The library's number of t's type: a type it has no kernels for is refused, never read as another one."""
    _require(t.dtype in (torch.bfloat16, torch.float32), "%s: %s, expected torch.bfloat16 or torch.float32", what, t.dtype)
    return BF16 if t.dtype == torch.bfloat16 else F32


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()          # an int: ctypes converts it for a c_void_p parameter


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    """The caller's current stream as a raw handle (every call is enqueued on it)."""
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _ptr_array(ts: Sequence[torch.Tensor]):
    arr = (C.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        assert t.is_cuda and t.is_contiguous()
        arr[i] = t.data_ptr()
    return arr


@dataclass
class Config:
    d_model: int
    n_groups: int
    experts_per_group: int
    k_groups: int
    k_experts: int
    group_width: Sequence[int]
    dtype: str = "bf16"
    alpha_g: float = 1e-4
    alpha_e: float = 2.5e-3
    eps: float = 1e-20
    f_norm_by_T: int = 1
    fe_mode: int = 0
    row_align: int = 128

    def __setattr__(self, name, value):
        self.__dict__.pop("_c_cache", None)
        self.__dict__[name] = value

    def c(self) -> mohge_config:
        """The POD of the C ABI; rebuilt only when a field has changed since the last call."""
        # any sequence of whole numbers (list, tuple, range, array, tensor), which may be changed in place
        widths = [operator.index(w) for w in self.group_width]
        cached = self.__dict__.get("_c_cache")
        if cached is not None and cached[0] == widths:
            return cached[1]
        s = mohge_config()
        s.d_model, s.n_groups, s.experts_per_group = self.d_model, self.n_groups, self.experts_per_group
        s.k_groups, s.k_experts = self.k_groups, self.k_experts
        for g in range(MAX_GROUPS):
            s.group_width[g] = widths[g] if g < len(widths) else 0
        s.dtype = BF16 if self.dtype == "bf16" else F32
        s.alpha_g, s.alpha_e, s.eps = self.alpha_g, self.alpha_e, self.eps
        s.f_norm_by_T, s.fe_mode, s.row_align = self.f_norm_by_T, self.fe_mode, self.row_align
        # what weights laid out for a layer depend on
        s.layer = (self.d_model, self.n_groups, self.experts_per_group, tuple(s.group_width[:self.n_groups]))
        self.__dict__["_c_cache"] = (widths, s)
        return s

    @property
    def n_experts(self):
        return self.n_groups * self.experts_per_group

    @property
    def n_logits(self):
        return self.n_groups + self.n_experts

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


def mohge_launch_count() -> int:
    return int(lib().mohge_launch_count())


def mohge_workspace_bytes(cfg: Config, T: int) -> int:
    n = lib().mohge_workspace_bytes(C.byref(cfg.c()), T)
    if n <= 0:
        raise MohgeError("mohge_workspace_bytes: %s" % lib().mohge_last_error().decode())
    return n


def mohge_perm_rows(cfg: Config, T: int) -> int:
    n = lib().mohge_perm_rows(C.byref(cfg.c()), T)
    if n <= 0 and T > 0:
        raise MohgeError("mohge_perm_rows: %s" % lib().mohge_last_error().decode())
    return n


def mohge_workspace_init(cfg, T, ws):
    _check(lib().mohge_workspace_init(C.byref(cfg.c()), T, _ptr(ws), ws.numel() * ws.element_size(),
                                      _stream()), "mohge_workspace_init")


MOHGE_ERR_TIMEOUT, MOHGE_ERR_DEVICE_CHECK = -5, -6


def mohge_get_device_status_rc(ws):
    """(return code, status word): the code is 0, MOHGE_ERR_TIMEOUT or MOHGE_ERR_DEVICE_CHECK as
    decoded from the word by the library."""
    out = C.c_int32(0)
    rc = lib().mohge_get_device_status(_ptr(ws), C.byref(out), _stream())
    if rc not in (0, MOHGE_ERR_TIMEOUT, MOHGE_ERR_DEVICE_CHECK):
        _check(rc, "mohge_get_device_status")
    return rc, out.value


def mohge_get_device_status(ws) -> int:
    """The device status word (0 = nothing reported)."""
    return mohge_get_device_status_rc(ws)[1]


def mohge_get_switch(name: str) -> int:
    return int(lib().mohge_get_switch(name.encode()))


def mohge_set_switch(name: str, value: int) -> None:
    _check(lib().mohge_set_switch(name.encode(), int(value)), "mohge_set_switch")


def mohge_map_cache_stats():
    h, m = C.c_int64(0), C.c_int64(0)
    lib().mohge_map_cache_stats(C.byref(h), C.byref(m))
    return h.value, m.value


def mohge_route(cfg, T, x, w_router, logit_bias, logits_in, logits_out, group_idx, expert_idx,
                gate_w, gs_saved, esp_saved, ws):
    _check(lib().mohge_route(C.byref(cfg.c()), T, _ptr(x), _ptr(w_router), _ptr(logit_bias),
                             _ptr(logits_in), _ptr(logits_out), _ptr(group_idx), _ptr(expert_idx),
                             _ptr(gate_w), _ptr(gs_saved), _ptr(esp_saved), _ptr(ws), _stream()),
           "mohge_route")


def mohge_aux_stats(cfg, T, gs_saved, esp_saved, group_idx, expert_idx, group_count, group_psum,
                    expert_count_routed, expert_count_lit, expert_psum, loss_out, ws):
    _check(lib().mohge_aux_stats(C.byref(cfg.c()), T, _ptr(gs_saved), _ptr(esp_saved),
                                 _ptr(group_idx), _ptr(expert_idx), _ptr(group_count),
                                 _ptr(group_psum), _ptr(expert_count_routed),
                                 _ptr(expert_count_lit), _ptr(expert_psum), _ptr(loss_out),
                                 _ptr(ws), _stream()), "mohge_aux_stats")


def mohge_aux_stats_static(cfg, T, gs_saved, esp_saved, group_idx, expert_idx, group_count,
                           group_psum, expert_count_routed, expert_count_lit, expert_psum, loss_out):
    """mohge_aux_stats without a workspace: for callers that cannot allocate one (see mohge.h)."""
    _check(lib().mohge_aux_stats_static(C.byref(cfg.c()), T, _ptr(gs_saved), _ptr(esp_saved),
                                        _ptr(group_idx), _ptr(expert_idx), _ptr(group_count),
                                        _ptr(group_psum), _ptr(expert_count_routed),
                                        _ptr(expert_count_lit), _ptr(expert_psum), _ptr(loss_out),
                                        _stream()), "mohge_aux_stats_static")


def mohge_dispatch(cfg, T, x, expert_idx, counts, offsets, aligned_offsets, row_of, prow_of,
                   src_of, x_perm, ws):
    _check(lib().mohge_dispatch(C.byref(cfg.c()), T, _ptr(x), _ptr(expert_idx), _ptr(counts),
                                _ptr(offsets), _ptr(aligned_offsets), _ptr(row_of), _ptr(prow_of),
                                _ptr(src_of), _ptr(x_perm), _ptr(ws), _stream()), "mohge_dispatch")


def mohge_expert_fwd(cfg, T, x_perm, counts, aligned_offsets, w13, w2, au_saved, h_saved, y_perm, ws):
    a13, a2 = _ptr_array(w13), _ptr_array(w2)
    _check(lib().mohge_expert_fwd(C.byref(cfg.c()), T, _ptr(x_perm), _ptr(counts),
                                  _ptr(aligned_offsets), C.cast(a13, _P), C.cast(a2, _P),
                                  _ptr(au_saved), _ptr(h_saved), _ptr(y_perm), _ptr(ws), _stream()),
           "mohge_expert_fwd")


def mohge_combine(cfg, T, y_perm, prow_of, gate_w, y, y_add=None):
    _check(lib().mohge_combine(C.byref(cfg.c()), T, _ptr(y_perm), _ptr(prow_of), _ptr(gate_w),
                               _ptr(y_add), _ptr(y), _stream()), "mohge_combine")


def mohge_combine_bwd(cfg, T, dy, y_perm, prow_of, gate_w, counts, aligned_offsets, dy_perm, dgate_w):
    _check(lib().mohge_combine_bwd(C.byref(cfg.c()), T, _ptr(dy), _ptr(y_perm), _ptr(prow_of),
                                   _ptr(gate_w), _ptr(counts), _ptr(aligned_offsets), _ptr(dy_perm),
                                   _ptr(dgate_w), _stream()), "mohge_combine_bwd")


def mohge_expert_bwd(cfg, T, dy_perm, x_perm, au_saved, h_saved, counts, aligned_offsets, w13, w2,
                     dau, dx_perm, dw13, dw2, accumulate, ws):
    a13, a2, d13, d2 = _ptr_array(w13), _ptr_array(w2), _ptr_array(dw13), _ptr_array(dw2)
    _check(lib().mohge_expert_bwd(C.byref(cfg.c()), T, _ptr(dy_perm), _ptr(x_perm), _ptr(au_saved),
                                  _ptr(h_saved), _ptr(counts), _ptr(aligned_offsets),
                                  C.cast(a13, _P), C.cast(a2, _P), _ptr(dau), _ptr(dx_perm),
                                  C.cast(d13, _P), C.cast(d2, _P), int(accumulate), _ptr(ws),
                                  _stream()), "mohge_expert_bwd")


def mohge_expert_bwd_dgate(cfg, T, dy_perm, x_perm, au_saved, h_saved, counts, aligned_offsets, w13, w2,
                           dau, dx_perm, dw13, dw2, accumulate, dy, y_perm, prow_of, gate_w, dgate_w, ws):
    a13, a2, d13, d2 = _ptr_array(w13), _ptr_array(w2), _ptr_array(dw13), _ptr_array(dw2)
    _check(lib().mohge_expert_bwd_dgate(C.byref(cfg.c()), T, _ptr(dy_perm), _ptr(x_perm), _ptr(au_saved),
                                        _ptr(h_saved), _ptr(counts), _ptr(aligned_offsets),
                                        C.cast(a13, _P), C.cast(a2, _P), _ptr(dau), _ptr(dx_perm),
                                        C.cast(d13, _P), C.cast(d2, _P), int(accumulate), _ptr(dy),
                                        _ptr(y_perm), _ptr(prow_of), _ptr(gate_w), _ptr(dgate_w),
                                        _ptr(ws), _stream()), "mohge_expert_bwd_dgate")


def mohge_dispatch_indices(cfg, T, expert_idx, counts, offsets, aligned_offsets, row_of, prow_of,
                           src_of, tok_of_prow, ws):
    _check(lib().mohge_dispatch_indices(C.byref(cfg.c()), T, _ptr(expert_idx), _ptr(counts),
                                        _ptr(offsets), _ptr(aligned_offsets), _ptr(row_of),
                                        _ptr(prow_of), _ptr(src_of), _ptr(tok_of_prow), _ptr(ws),
                                        _stream()), "mohge_dispatch_indices")


def mohge_expert_fwd_gather(cfg, T, x, tok_of_prow, counts, aligned_offsets, w13, w2, au_saved, h_saved,
                            y_perm, ws):
    a13, a2 = _ptr_array(w13), _ptr_array(w2)
    _check(lib().mohge_expert_fwd_gather(C.byref(cfg.c()), T, _ptr(x), _ptr(tok_of_prow), _ptr(counts),
                                         _ptr(aligned_offsets), C.cast(a13, _P), C.cast(a2, _P),
                                         _ptr(au_saved), _ptr(h_saved), _ptr(y_perm), _ptr(ws), _stream()),
           "mohge_expert_fwd_gather")


def mohge_expert_bwd_gather(cfg, T, dy_perm, x, tok_of_prow, au_saved, h_saved, counts, aligned_offsets,
                            w13, w2, dau, dx_perm, dw13, dw2, accumulate, dy, y_perm, prow_of, gate_w,
                            dgate_w, ws):
    a13, a2, d13, d2 = _ptr_array(w13), _ptr_array(w2), _ptr_array(dw13), _ptr_array(dw2)
    _check(lib().mohge_expert_bwd_gather(C.byref(cfg.c()), T, _ptr(dy_perm), _ptr(x), _ptr(tok_of_prow),
                                         _ptr(au_saved), _ptr(h_saved), _ptr(counts),
                                         _ptr(aligned_offsets), C.cast(a13, _P), C.cast(a2, _P),
                                         _ptr(dau), _ptr(dx_perm), C.cast(d13, _P), C.cast(d2, _P),
                                         int(accumulate), _ptr(dy), _ptr(y_perm), _ptr(prow_of),
                                         _ptr(gate_w), _ptr(dgate_w), _ptr(ws), _stream()),
           "mohge_expert_bwd_gather")


def mohge_row_tokens(cfg, T, counts, offsets, aligned_offsets, src_of, tok_of_prow):
    _check(lib().mohge_row_tokens(C.byref(cfg.c()), T, _ptr(counts), _ptr(offsets), _ptr(aligned_offsets),
                                  _ptr(src_of), _ptr(tok_of_prow), _stream()), "mohge_row_tokens")


def mohge_expert_bwd_dy(cfg, T, dy, tok_of_prow, x_perm, au_saved, h_saved, counts, aligned_offsets, w13, w2,
                        dau, dx_perm, dw13, dw2, accumulate, y_perm, prow_of, gate_w, dgate_w, hs, row_gate,
                        ws):
    a13, a2, d13, d2 = _ptr_array(w13), _ptr_array(w2), _ptr_array(dw13), _ptr_array(dw2)
    _check(lib().mohge_expert_bwd_dy(C.byref(cfg.c()), T, _ptr(dy), _ptr(tok_of_prow), _ptr(x_perm),
                                     _ptr(au_saved), _ptr(h_saved), _ptr(counts), _ptr(aligned_offsets),
                                     C.cast(a13, _P), C.cast(a2, _P), _ptr(dau), _ptr(dx_perm),
                                     C.cast(d13, _P), C.cast(d2, _P), int(accumulate), _ptr(y_perm),
                                     _ptr(prow_of), _ptr(gate_w), _ptr(dgate_w), _ptr(hs), _ptr(row_gate),
                                     _ptr(ws), _stream()), "mohge_expert_bwd_dy")


def mohge_dispatch_bwd(cfg, T, dx_perm, prow_of, dx, dx_add=None):
    _check(lib().mohge_dispatch_bwd(C.byref(cfg.c()), T, _ptr(dx_perm), _ptr(prow_of),
                                    _ptr(dx_add), _ptr(dx), _stream()), "mohge_dispatch_bwd")


def mohge_shared_fwd(cfg, T, shared_width, x, w13_shared, w2_shared, au_shared, h_shared, y_shared, ws):
    _check(lib().mohge_shared_fwd(C.byref(cfg.c()), T, int(shared_width), _ptr(x), _ptr(w13_shared),
                                  _ptr(w2_shared), _ptr(au_shared), _ptr(h_shared), _ptr(y_shared),
                                  _ptr(ws), _stream()), "mohge_shared_fwd")


def mohge_shared_bwd(cfg, T, shared_width, dy, x, au_shared, h_shared, w13_shared, w2_shared,
                     dau_shared, dx_shared, dw13_shared, dw2_shared, accumulate, ws):
    _check(lib().mohge_shared_bwd(C.byref(cfg.c()), T, int(shared_width), _ptr(dy), _ptr(x),
                                  _ptr(au_shared), _ptr(h_shared), _ptr(w13_shared),
                                  _ptr(w2_shared), _ptr(dau_shared), _ptr(dx_shared),
                                  _ptr(dw13_shared), _ptr(dw2_shared), int(accumulate), _ptr(ws),
                                  _stream()), "mohge_shared_bwd")


def mohge_route_bwd(cfg, T, x, w_router, dgate_w, gs_saved, esp_saved, group_idx, expert_idx,
                    group_count, expert_count, dlogits, dx, dw_router, ws):
    _check(lib().mohge_route_bwd(C.byref(cfg.c()), T, _ptr(x), _ptr(w_router), _ptr(dgate_w),
                                 _ptr(gs_saved), _ptr(esp_saved), _ptr(group_idx), _ptr(expert_idx),
                                 _ptr(group_count), _ptr(expert_count), _ptr(dlogits), _ptr(dx),
                                 _ptr(dw_router), _ptr(ws), _stream()), "mohge_route_bwd")


def mohge_mx8_pitch(K: int) -> int:
    return int(lib().mohge_mx8_pitch(K))


def mohge_mx8_tiled_bytes(batch: int, rows: int, K: int) -> int:
    return int(lib().mohge_mx8_tiled_bytes(batch, rows, K))


def mohge_norm_fwd(cfg, T, x, residual, weight, norm_eps, h, y, y8, y8_scale, rstd):
    _check(lib().mohge_norm_fwd(C.byref(cfg.c()), T, _ptr(x), _ptr(residual), _ptr(weight), norm_eps, _ptr(h),
                                _ptr(y), _ptr(y8), _ptr(y8_scale), _ptr(rstd), _stream()), "mohge_norm_fwd")


def mohge_norm_bwd(cfg, T, dy, dh, h, weight, rstd, dx, dweight, accumulate, ws):
    _check(lib().mohge_norm_bwd(C.byref(cfg.c()), T, _ptr(dy), _ptr(dh), _ptr(h), _ptr(weight), _ptr(rstd),
                                _ptr(dx), _ptr(dweight), int(accumulate), _ptr(ws), _stream()), "mohge_norm_bwd")


def mx8_scale_pitch(K: int) -> int:
    """Bytes per row of the scales in the mx8 rows layout."""
    return 4 * ((K + 127) // 128)


def mx8_empty(rows: int, K: int, device="cuda"):
    """Uninitialised (elements, scales) of the mx8 rows layout."""
    return (torch.empty(rows, mohge_mx8_pitch(K), dtype=torch.uint8, device=device),
            torch.empty(rows, mx8_scale_pitch(K), dtype=torch.uint8, device=device))


def new_workspace(cfg: Config, T: int, device="cuda") -> torch.Tensor:
    """A workspace for T tokens, its status word cleared."""
    ws = torch.empty(mohge_workspace_bytes(cfg, T), dtype=torch.uint8, device=device)
    mohge_workspace_init(cfg, T, ws)
    return ws


def mohge_w4_packed_bytes(batch: int, rows: int, K: int, group_size: int) -> int:
    n = lib().mohge_w4_packed_bytes(batch, rows, K, group_size)
    if n <= 0 and batch * rows > 0:
        raise MohgeError("mohge_w4_packed_bytes: %s" % lib().mohge_last_error().decode())
    return int(n)


def mohge_quantize_w4(w, group_size, q, scale):
    """w [.., K] BF16 or FP32 -> q [.., K / 2] uint8, scale [.., ceil(K / group_size)] BF16."""
    *lead, K = w.shape
    code = _dtype_code(w, "mohge_quantize_w4: w")
    rows = math.prod(lead)
    _require_bytes("mohge_quantize_w4: q", q, rows * (K // 2))
    _require_bytes("mohge_quantize_w4: scale", scale, 2 * rows * -(-K // group_size))
    _check(lib().mohge_quantize_w4(rows, K, group_size, code, _ptr(w), _ptr(q), _ptr(scale), _stream()),
           "mohge_quantize_w4")


def quantize_w4(w, group_size: int):
    """(codes, scales) of the plain 4-bit form of w [.., K]."""
    *lead, K = w.shape
    q = torch.empty(*lead, K // 2, dtype=torch.uint8, device=w.device)
    scale = torch.empty(*lead, -(-K // group_size), dtype=torch.bfloat16, device=w.device)
    mohge_quantize_w4(w, group_size, q, scale)
    return q, scale


def mohge_pack_w4(q, scale, group_size, gate_up, packed):
    """q [batch, rows, K / 2] uint8 and its scales -> packed (mohge_w4_packed_bytes bytes)."""
    batch, rows, half = q.shape
    _require_form("mohge_pack_w4: q", q, (batch, rows, half), torch.uint8)
    _require_form("mohge_pack_w4: scale", scale, (batch, rows, -(-2 * half // group_size)), torch.bfloat16)
    _require_bytes("mohge_pack_w4: packed", packed, mohge_w4_packed_bytes(batch, rows, 2 * half, group_size))
    _check(lib().mohge_pack_w4(batch, rows, 2 * half, group_size, int(gate_up), _ptr(q), _ptr(scale), _ptr(packed),
                               _stream()), "mohge_pack_w4")


def _require_form(what: str, t: torch.Tensor, shape, dtype=None) -> None:
    """shape, and dtype where one is given (1: any type of one byte)."""
    fits = dtype is None or (t.element_size() == 1 if dtype == 1 else t.dtype == dtype)
    _require(tuple(t.shape) == tuple(shape) and fits, "%s is %s %s, expected %s %s", what, t.dtype, tuple(t.shape),
             {None: "any type", 1: "one byte each"}.get(dtype, dtype), tuple(shape))


def _require_weights(cfg: Config, what: str, w13, w2, k13=lambda d: d, k2=lambda w: w, dtype=None) -> None:
    """One w13[g] [N, 2 W_g, k13(d)] and w2[g] [N, d, k2(W_g)] per group of the layer: the library walks as many host
    pointers, and as many rows and columns behind each, as the config says."""
    d, Ng, N, W = cfg.c().layer
    for name, ws, shape in (("w13", w13, lambda w: (N, 2 * w, k13(d))), ("w2", w2, lambda w: (N, d, k2(w)))):
        _require(len(ws) == Ng, "%s: %d %s for %d groups", what, len(ws), name, Ng)
        for g in range(Ng):
            _require_form("%s: %s[%d]" % (what, name, g), ws[g], shape(W[g]), dtype)


def _layer_of(cfg: Config, weights) -> mohge_config:
    """The POD of cfg, which has to be of the layer that `weights` were laid out for."""
    c = cfg.c()
    _require(c.layer == weights.layer, "weights of a layer (d, groups, experts per group, widths) = %s with a config of %s",
             weights.layer, c.layer)
    return c


class W4Weights:
    """The experts' weights in packed 4-bit form, made once: per group g, codes w13_q[g] [N, 2 W_g, d / 2] and
    w2_q[g] [N, d, W_g / 2] with their scales (mohge_quantize_w4's layout)."""

    def __init__(self, cfg: Config, group_size: int, w13_q, w13_scale, w2_q, w2_scale):
        groups = lambda k: -(-k // group_size)  # noqa: E731
        _require_weights(cfg, "W4Weights: codes", w13_q, w2_q, lambda d: d // 2, lambda w: w // 2, torch.uint8)
        _require_weights(cfg, "W4Weights: scales", w13_scale, w2_scale, groups, groups, torch.bfloat16)

        def pack(q, s, gate_up):
            out = torch.empty(mohge_w4_packed_bytes(q.shape[0], q.shape[1], 2 * q.shape[2], group_size), dtype=torch.uint8,
                              device=q.device)
            mohge_pack_w4(q, s, group_size, gate_up, out)
            return out

        self.group_size, self.layer = group_size, cfg.c().layer
        self.w13 = [pack(q, s, True) for q, s in zip(w13_q, w13_scale)]
        self.w2 = [pack(q, s, False) for q, s in zip(w2_q, w2_scale)]
        self._a13, self._a2 = _ptr_array(self.w13), _ptr_array(self.w2)
        self.p13, self.p2 = C.cast(self._a13, _P), C.cast(self._a2, _P)

    @classmethod
    def quantize(cls, cfg: Config, group_size: int, w13, w2):
        """From the layer's own weights w13[g] [N, 2 W_g, d] and w2[g] [N, d, W_g]."""
        _require_weights(cfg, "W4Weights.quantize", w13, w2)
        a, b = [quantize_w4(w, group_size) for w in w13], [quantize_w4(w, group_size) for w in w2]
        return cls(cfg, group_size, [x[0] for x in a], [x[1] for x in a], [x[0] for x in b], [x[1] for x in b])

    def requantize(self, cfg: Config, w13, w2) -> None:
        """The same from weights that have changed, in the memory that is there (graphs hold its addresses)."""
        _layer_of(cfg, self)
        _require_weights(cfg, "W4Weights.requantize", w13, w2)
        for ws, packed, gate_up in ((w13, self.w13, True), (w2, self.w2, False)):
            for w, out in zip(ws, packed):
                mohge_pack_w4(*quantize_w4(w, self.group_size), self.group_size, gate_up, out)


def w4_scratch(cfg: Config, T: int, device="cuda") -> torch.Tensor:
    n = lib().mohge_w4_scratch_bytes(C.byref(cfg.c()), T)
    if n <= 0 and T > 0:
        raise MohgeError("mohge_w4_scratch_bytes: %s" % lib().mohge_last_error().decode())
    return torch.empty(max(16, n), dtype=torch.uint8, device=device)


def mohge_expert_fwd_w4(cfg, T, x, expert_idx, gate_w, weights: W4Weights, scratch, y, ws, y_add=None):
    _check(lib().mohge_expert_fwd_w4(C.byref(_layer_of(cfg, weights)), T, weights.group_size, _ptr(x), _ptr(expert_idx), _ptr(gate_w),
                                     weights.p13, weights.p2, _ptr(y_add), _ptr(scratch), _ptr(y), _ptr(ws), _stream()),
           "mohge_expert_fwd_w4")


def mohge_quantize_mx8(w, q, scale_tiled):
    """w [batch, rows, K] BF16 or FP32 -> operand layout."""
    batch, rows, K = w.shape
    code = _dtype_code(w, "mohge_quantize_mx8: w")
    _require_bytes("mohge_quantize_mx8: q", q, batch * rows * mohge_mx8_pitch(K))
    _require_bytes("mohge_quantize_mx8: scale_tiled", scale_tiled, mohge_mx8_tiled_bytes(batch, rows, K))
    _check(lib().mohge_quantize_mx8(batch, rows, K, code, _ptr(w), _ptr(q), _ptr(scale_tiled), _stream()), "mohge_quantize_mx8")


def quantize_mx8(w):
    """(elements, tiled scales) of the mx8 operand form of w [batch, rows, K]."""
    batch, rows, K = w.shape
    q = torch.empty(batch, rows, mohge_mx8_pitch(K), dtype=torch.uint8, device=w.device)
    s = torch.empty(mohge_mx8_tiled_bytes(batch, rows, K), dtype=torch.uint8, device=w.device)
    mohge_quantize_mx8(w, q, s)
    return q, s


def mohge_permute_mx8(cfg, T, x8, x8_scale, tok_of_prow, xp8, xp8_scale):
    _check(lib().mohge_permute_mx8(C.byref(cfg.c()), T, _ptr(x8), _ptr(x8_scale), _ptr(tok_of_prow), _ptr(xp8), _ptr(xp8_scale), _stream()), "mohge_permute_mx8")


def mohge_expert_fwd_mx8(cfg, T, xp8, xp8_scale, counts, aligned_offsets, weights: "Mx8Weights", h8, h8_scale, y_perm, ws):
    w = weights
    _check(lib().mohge_expert_fwd_mx8(C.byref(_layer_of(cfg, w)), T, _ptr(xp8), _ptr(xp8_scale), _ptr(counts), _ptr(aligned_offsets),
                                      w.p13, w.p13_scale, w.p2, w.p2_scale, _ptr(h8), _ptr(h8_scale), _ptr(y_perm),
                                      _ptr(ws), _stream()), "mohge_expert_fwd_mx8")


def mx8_rows(codes, scale):
    """E4M3 codes [T, K] and scale bytes [T, ceil(K / 32)] in the rows layout (padded with zeros)."""
    T, K = codes.shape
    q = torch.zeros(T, mohge_mx8_pitch(K), dtype=torch.uint8, device=codes.device)
    s = torch.zeros(T, mx8_scale_pitch(K), dtype=torch.uint8, device=codes.device)
    q[:, :K], s[:, :scale.shape[1]] = codes.view(torch.uint8), scale
    return q, s


def mx8_tile_scales(scale):
    """Scale bytes [batch, rows, ceil(K / 32)] in the tiled layout of the operands."""
    B, R, n = scale.shape
    if scale.element_size() == 1:
        scale = scale.view(torch.uint8)         # torch.float8_e8m0fnu among them: its bytes, not its values
    _require(not scale.is_floating_point(), "mx8_tile_scales: scales are bytes, not %s", scale.dtype)
    rb, kb = (R + 127) // 128, (n + 3) // 4
    full = torch.zeros(B, rb * 128, kb * 4, dtype=torch.uint8, device=scale.device)
    full[:, :R, :n] = scale
    return full.view(B, rb, 4, 32, kb, 4).permute(0, 1, 4, 3, 2, 5).contiguous().view(-1)


class Mx8Weights:
    """The experts' weights as mx8 operands, made once: per group g, codes w13[g] [N, 2 W_g, d] and w2[g]
    [N, d, W_g] (E4M3) with one scale byte per 32 columns [.., ceil(K / 32)]."""

    def __init__(self, cfg: Config, w13, w13_scale, w2, w2_scale):
        N, blocks = cfg.experts_per_group, lambda k: -(-k // 32)
        _require_weights(cfg, "Mx8Weights: codes", w13, w2, dtype=1)
        _require_weights(cfg, "Mx8Weights: scales", w13_scale, w2_scale, blocks, blocks)

        def elements(q):
            q = q.view(torch.uint8)
            K, pitch = q.shape[2], mohge_mx8_pitch(q.shape[2])
            if pitch == K:
                return q.contiguous()
            out = torch.zeros(q.shape[0], q.shape[1], pitch, dtype=torch.uint8, device=q.device)
            out[:, :, :K] = q
            return out

        self.layer = cfg.c().layer
        self._set([elements(q) for q in w13],
                  [mx8_tile_scales(s.reshape(2 * N, s.shape[1] // 2, s.shape[2])) for s in w13_scale],
                  [elements(q) for q in w2], [mx8_tile_scales(s) for s in w2_scale])

    def _set(self, w13, w13_scale, w2, w2_scale):
        self.w13, self.w13_scale, self.w2, self.w2_scale = w13, w13_scale, w2, w2_scale
        self._arrays = [_ptr_array(x) for x in (w13, w13_scale, w2, w2_scale)]
        self.p13, self.p13_scale, self.p2, self.p2_scale = [C.cast(a, _P) for a in self._arrays]

    @classmethod
    def quantize(cls, cfg: Config, w13, w2):
        """From the layer's own weights w13[g] [N, 2 W_g, d] and w2[g] [N, d, W_g]."""
        _require_weights(cfg, "Mx8Weights.quantize", w13, w2)
        N, d = cfg.experts_per_group, cfg.d_model
        a = [quantize_mx8(w.reshape(2 * N, w.shape[1] // 2, d)) for w in w13]
        b = [quantize_mx8(w) for w in w2]
        self = cls.__new__(cls)
        self.layer = cfg.c().layer
        self._set([x[0] for x in a], [x[1] for x in a], [x[0] for x in b], [x[1] for x in b])
        return self

    def requantize(self, cfg: Config, w13, w2) -> None:
        """The same from weights that have changed, in the memory that is there (graphs hold its addresses)."""
        _layer_of(cfg, self)
        _require_weights(cfg, "Mx8Weights.requantize", w13, w2)
        for w, q, s in zip(w13, self.w13, self.w13_scale):
            mohge_quantize_mx8(w.reshape(-1, w.shape[1] // 2, w.shape[2]), q, s)
        for w, q, s in zip(w2, self.w2, self.w2_scale):
            mohge_quantize_mx8(w, q, s)


class Mx8Buffers:
    """Device allocations for the 8-bit experts of one batch of T tokens."""

    def __init__(self, cfg: Config, T: int, device="cuda"):
        self.T = T
        rows, Tn, Ne, Ke, d, Wmax = max(128, mohge_perm_rows(cfg, T)), max(1, T), cfg.n_experts, cfg.k_experts, cfg.d_model, max(cfg.group_width)
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=device)  # noqa: E731
        u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device=device)  # noqa: E731
        self.ws = u8(mohge_workspace_bytes(cfg, T))
        self.counts, self.offsets, self.aligned = i32(Ne), i32(Ne + 4), i32(Ne + 4)
        self.row_of, self.prow_of, self.src_of = i32(Tn, Ke), i32(Tn, Ke), i32(Tn * Ke)
        self.tok_of_prow = i32(rows + 128)
        self.xp8, self.xp8_scale = u8(rows, mohge_mx8_pitch(d)), u8(mohge_mx8_tiled_bytes(1, rows, d))
        self.h8, self.h8_scale = u8(rows, mohge_mx8_pitch(Wmax)), u8(mohge_mx8_tiled_bytes(1, rows, Wmax))
        self.y_perm = torch.empty(rows, d, dtype=torch.bfloat16, device=device)
        self.y = torch.empty(Tn, d, dtype=torch.bfloat16, device=device)
        mohge_workspace_init(cfg, T, self.ws)


def _batch(cfg: Config, b, T: Optional[int]) -> int:
    """Tokens of a call on the buffers b: all that they were made for, or the first T of them."""
    if T is None or T == b.T:
        return b.T
    _require(0 <= T <= b.T, "%s tokens on buffers made for %d", T, b.T)
    _require_bytes("the workspace", b.ws, mohge_workspace_bytes(cfg, T))     # (not always less for fewer tokens)
    return T


def layer_forward_mx8(cfg: Config, b: Mx8Buffers, x8, x8_scale, expert_idx, gate_w, weights: Mx8Weights, y_add=None,
                      T: Optional[int] = None, y=None):
    """dispatch_indices -> permute_mx8 -> expert_fwd_mx8 -> combine on routed tokens; returns y, which is b.y (the
    next call's too) where none is given.  T: fewer tokens than the buffers were made for."""
    T = _batch(cfg, b, T)
    if y is None:
        y = b.y if T == b.T else b.y[:T]
    if T == 0:
        return y[:0]
    mohge_dispatch_indices(cfg, T, expert_idx, b.counts, b.offsets, b.aligned, b.row_of, b.prow_of, b.src_of,
                           b.tok_of_prow, b.ws)
    mohge_permute_mx8(cfg, T, x8, x8_scale, b.tok_of_prow, b.xp8, b.xp8_scale)
    mohge_expert_fwd_mx8(cfg, T, b.xp8, b.xp8_scale, b.counts, b.aligned, weights, b.h8, b.h8_scale, b.y_perm, b.ws)
    mohge_combine(cfg, T, b.y_perm, b.prow_of, gate_w, y, y_add=y_add)
    return y


class LayerBuffers:
    """Device allocations for one layer step (torch is used for memory only)."""

    def __init__(self, cfg: Config, T: int, device="cuda", shared_width: int = 0):
        self.cfg, self.T, self.shared_width = cfg, T, shared_width
        dt, dev = cfg.torch_dtype, device
        Ne, NL, Ke, Kg, d = cfg.n_experts, cfg.n_logits, cfg.k_experts, cfg.k_groups, cfg.d_model
        Wmax = max(cfg.group_width)
        rows = max(1, mohge_perm_rows(cfg, T))
        self.rows = rows
        Tn = max(1, T)
        e = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device=dev)
        i32, f32 = torch.int32, torch.float32
        self.ws = torch.empty(mohge_workspace_bytes(cfg, T), dtype=torch.uint8, device=dev)
        self.logits = e(Tn, NL, dtype=f32)
        self.group_idx, self.expert_idx = e(Tn, Kg, dtype=i32), e(Tn, Ke, dtype=i32)
        self.gate_w, self.gs, self.esp = e(Tn, Ke, dtype=f32), e(Tn, cfg.n_groups, dtype=f32), e(Tn, Ne, dtype=f32)
        self.group_count, self.group_psum = e(cfg.n_groups, dtype=i32), e(cfg.n_groups, dtype=f32)
        self.cnt_routed, self.cnt_lit, self.expert_psum = e(Ne, dtype=i32), e(Ne, dtype=i32), e(Ne, dtype=f32)
        self.loss = e(4, dtype=f32)
        self.counts, self.offsets, self.aligned = e(Ne, dtype=i32), e(Ne + 4, dtype=i32), e(Ne + 4, dtype=i32)
        self.row_of, self.prow_of, self.src_of = e(Tn, Ke, dtype=i32), e(Tn, Ke, dtype=i32), e(Tn * Ke, dtype=i32)
        self.x_perm, self.y_perm = e(rows, d), e(rows, d)
        self.tok_of_prow = e(rows + 128, dtype=i32)        # row map of the gathering entry points
        self.au, self.h = e(rows, 2 * Wmax), e(rows, Wmax)
        self.y = e(Tn, d)
        # backward
        self.dy_perm, self.dx_perm, self.dau = e(rows, d), e(rows, d), e(rows, 2 * Wmax)
        self.dgate, self.dlogits = e(Tn, Ke, dtype=f32), e(Tn, NL, dtype=f32)
        self.dx = e(Tn, d)
        self.dw_router = e(NL, d, dtype=f32)
        self.dw13 = [e(cfg.experts_per_group, 2 * w, d, dtype=f32) for w in cfg.group_width]
        self.dw2 = [e(cfg.experts_per_group, d, w, dtype=f32) for w in cfg.group_width]
        if shared_width:
            Ws = shared_width
            self.au_sh, self.h_sh, self.y_sh = e(Tn, 2 * Ws), e(Tn, Ws), e(Tn, d)
            self.dau_sh, self.dx_sh = e(Tn, 2 * Ws), e(Tn, d)
            self.dw13_sh, self.dw2_sh = e(2 * Ws, d, dtype=f32), e(d, Ws, dtype=f32)
        mohge_workspace_init(cfg, T, self.ws)


def layer_forward(cfg: Config, b: LayerBuffers, x, w_router, w13, w2, logit_bias=None,
                  logits_in=None, aux=True, shared=None, gather=False, T: Optional[int] = None):
    """route -> aux_stats -> dispatch -> expert_fwd (-> shared_fwd) -> combine; results stay in
    `b`.  shared = (w13_shared, w2_shared) adds the shared experts (b.shared_width wide).
    gather: no x_perm is written; the GEMMs gather the rows of x (mohge_dispatch_indices,
    mohge_expert_fwd_gather).
    T: fewer tokens than the buffers were made for (the first T rows of them are used)."""
    T = _batch(cfg, b, T)
    mohge_route(cfg, T, x, w_router, logit_bias, logits_in, b.logits, b.group_idx, b.expert_idx,
                b.gate_w, b.gs, b.esp, b.ws)
    if aux:
        mohge_aux_stats(cfg, T, b.gs, b.esp, b.group_idx, b.expert_idx, b.group_count, b.group_psum,
                        b.cnt_routed, b.cnt_lit, b.expert_psum, b.loss, b.ws)
    if gather:
        mohge_dispatch_indices(cfg, T, b.expert_idx, b.counts, b.offsets, b.aligned, b.row_of, b.prow_of,
                               b.src_of, b.tok_of_prow, b.ws)
        mohge_expert_fwd_gather(cfg, T, x, b.tok_of_prow, b.counts, b.aligned, w13, w2, b.au, b.h,
                                b.y_perm, b.ws)
    else:
        mohge_dispatch(cfg, T, x, b.expert_idx, b.counts, b.offsets, b.aligned, b.row_of, b.prow_of,
                       b.src_of, b.x_perm, b.ws)
        mohge_expert_fwd(cfg, T, b.x_perm, b.counts, b.aligned, w13, w2, b.au, b.h, b.y_perm, b.ws)
    if shared is not None:
        mohge_shared_fwd(cfg, T, b.shared_width, x, shared[0], shared[1], b.au_sh, b.h_sh, b.y_sh, b.ws)
    mohge_combine(cfg, T, b.y_perm, b.prow_of, b.gate_w, b.y,
                  y_add=b.y_sh if shared is not None else None)
    return b.y


def layer_backward(cfg: Config, b: LayerBuffers, x, w_router, w13, w2, dy, aux=True, accumulate=False,
                   shared=None, fused_dgate=True, gather=False, dy_fused=False, T: Optional[int] = None):
    """combine_bwd -> expert_bwd (-> shared_bwd) -> dispatch_bwd -> route_bwd; results stay in `b`.
    fused_dgate: the gate gradient comes out of the experts' backward (mohge_expert_bwd_dgate) and
    combine_bwd does not read y_perm; otherwise combine_bwd computes it from y_perm.
    dy_fused: no combine_bwd and no dy_perm at all (mohge_expert_bwd_dy gathers the rows of dy).
    T: as layer_forward was given it."""
    T = _batch(cfg, b, T)
    assert not (gather and dy_fused), "the backward without dy_perm reads x_perm: not with gather=True"
    if dy_fused:    # after a forward through x_perm
        if getattr(b, "hs", None) is None:
            b.hs = torch.empty_like(b.h)
            b.row_gate = torch.empty(b.h.shape[0], dtype=torch.float32, device=b.h.device)
        mohge_row_tokens(cfg, T, b.counts, b.offsets, b.aligned, b.src_of, b.tok_of_prow)
        mohge_expert_bwd_dy(cfg, T, dy, b.tok_of_prow, b.x_perm, b.au, b.h, b.counts, b.aligned, w13, w2,
                            b.dau, b.dx_perm, b.dw13, b.dw2, accumulate, b.y_perm, b.prow_of, b.gate_w,
                            b.dgate, b.hs, b.row_gate, b.ws)
    elif gather:    # after a forward with gather=True: x_perm was never written
        mohge_combine_bwd(cfg, T, dy, None, b.prow_of, b.gate_w, b.counts, b.aligned, b.dy_perm, None)
        mohge_expert_bwd_gather(cfg, T, b.dy_perm, x, b.tok_of_prow, b.au, b.h, b.counts, b.aligned, w13,
                                w2, b.dau, b.dx_perm, b.dw13, b.dw2, accumulate, dy, b.y_perm, b.prow_of,
                                b.gate_w, b.dgate, b.ws)
    elif fused_dgate:
        mohge_combine_bwd(cfg, T, dy, None, b.prow_of, b.gate_w, b.counts, b.aligned, b.dy_perm, None)
        mohge_expert_bwd_dgate(cfg, T, b.dy_perm, b.x_perm, b.au, b.h, b.counts, b.aligned, w13, w2,
                               b.dau, b.dx_perm, b.dw13, b.dw2, accumulate, dy, b.y_perm, b.prow_of,
                               b.gate_w, b.dgate, b.ws)
    else:
        mohge_combine_bwd(cfg, T, dy, b.y_perm, b.prow_of, b.gate_w, b.counts, b.aligned, b.dy_perm,
                          b.dgate)
        mohge_expert_bwd(cfg, T, b.dy_perm, b.x_perm, b.au, b.h, b.counts, b.aligned, w13, w2, b.dau,
                         b.dx_perm, b.dw13, b.dw2, accumulate, b.ws)
    if shared is not None:
        mohge_shared_bwd(cfg, T, b.shared_width, dy, x, b.au_sh, b.h_sh, shared[0], shared[1],
                         b.dau_sh, b.dx_sh, b.dw13_sh, b.dw2_sh, accumulate, b.ws)
    mohge_dispatch_bwd(cfg, T, b.dx_perm, b.prow_of, b.dx,
                       dx_add=b.dx_sh if shared is not None else None)
    cnt_e = b.cnt_lit if cfg.fe_mode == 0 else b.cnt_routed
    mohge_route_bwd(cfg, T, x, w_router, b.dgate, b.gs, b.esp, b.group_idx, b.expert_idx,
                    b.group_count if aux else None, cnt_e if aux else None, b.dlogits, b.dx,
                    b.dw_router, b.ws)
    return b.dx

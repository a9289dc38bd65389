"""Binding of libmaskkv.so: argument marshalling only.

Every function mirrors the C entry point of the same name in ``include/maskkv.h`` and takes
torch device tensors; torch is used for device memory and streams, nothing is computed here.
The arguments are unpacked by a small CPython extension (``csrc/python.cpp``), which is what a
call costs besides its kernel launches.  If the shared library or the extension has not been
built the import of this module fails loudly: there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes as ct
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# MASKKV_LIB_PATH selects another build of the same library (e.g. an instrumented one)
LIB_PATH = os.environ.get("MASKKV_LIB_PATH", os.path.join(_HERE, "libmaskkv.so"))

MASKKV_F32, MASKKV_BF16 = 0, 1
POOL_MEAN, POOL_MAX = 0, 1
MAX_BATCH = 64

SYMBOLS = [
    "maskkv_version", "maskkv_strerror", "maskkv_last_error",
    "maskkv_score_workspace_bytes", "maskkv_score", "maskkv_score_given_lse", "maskkv_score_static",
    "maskkv_select_workspace_bytes", "maskkv_select",
    "maskkv_compact",
    "maskkv_attend_workspace_bytes", "maskkv_attend", "maskkv_attend_full",
    "maskkv_compact_mx", "maskkv_expand_mx", "maskkv_attend_mx_workspace_bytes", "maskkv_attend_mx",
    "maskkv_accumulate", "maskkv_accumulate_mx", "maskkv_evict", "maskkv_evict_mx",
    "maskkv_head_budgets",
    "maskkv_layer_importance_workspace_bytes", "maskkv_layer_importance", "maskkv_layer_budgets",
    "maskkv_value_shift",
]


class MaskKVError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str):
        super().__init__(f"{what} failed: status {status} ({detail})")
        self.status = status


class _CTensor(ct.Structure):
    _fields_ = [("ptr", ct.c_void_p), ("stride_b", ct.c_int64), ("stride_h", ct.c_int64),
                ("stride_t", ct.c_int64), ("seq_start", ct.POINTER(ct.c_int32))]


class _CDesc(ct.Structure):
    _fields_ = [("B", ct.c_int32), ("H", ct.c_int32), ("d", ct.c_int32), ("dtype", ct.c_int32),
                ("n_resp", ct.c_int32), ("n_query", ct.c_int32), ("P_max", ct.c_int32), ("q_per_kv", ct.c_int32),
                ("prompt_len", ct.POINTER(ct.c_int32))]


def _load() -> ct.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2510_09309_amd.build); "
            "this package has no fallback path")
    lib = ct.CDLL(LIB_PATH)
    lib.maskkv_strerror.restype = ct.c_char_p
    lib.maskkv_last_error.restype = ct.c_char_p
    for name in SYMBOLS:
        getattr(lib, name)  # raises AttributeError if a declared entry point is not exported
    return lib


_lib = _load()


def _load_marshal():
    try:
        from . import _marshal
    except ImportError as e:
        raise ImportError(f"the argument marshalling extension of this package is missing or does not load ({e}): build "
                          "it first (python -m paper_2510_09309_amd.build)") from e
    _marshal.bind({name: ct.cast(getattr(_lib, name), ct.c_void_p).value for name in SYMBOLS})
    return _marshal


_native = _load_marshal()


@dataclass
class Desc:
    """Python mirror of maskkv_desc."""
    B: int
    H: int
    d: int
    dtype: int
    n_resp: int
    P_max: int
    n_query: Optional[int] = None
    prompt_len: Optional[Sequence[int]] = None
    q_per_kv: int = 0   # query heads per key/value head (0 or 1: multi-head attention); H counts KV heads

    def c(self) -> _CDesc:
        nq = self.n_resp if self.n_query is None else self.n_query
        c = _CDesc(self.B, self.H, self.d, self.dtype, self.n_resp, nq, self.P_max, int(self.q_per_kv), None)
        if self.prompt_len is not None:
            arr = (ct.c_int32 * len(self.prompt_len))(*[int(x) for x in self.prompt_len])
            c._keep = arr
            c.prompt_len = ct.cast(arr, ct.POINTER(ct.c_int32))
        return c


@dataclass
class MxCache:
    """Python mirror of maskkv_mx_cache: uint8 device tensors, codes [capacity, d/2] and scales [capacity, d/32]."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: Optional[torch.Tensor] = None    # (maskkv_accumulate_mx reads the keys only)
    v_scales: Optional[torch.Tensor] = None

    @classmethod
    def empty(cls, capacity: int, d: int, device="cuda") -> "MxCache":
        """Uninitialised room for `capacity` rows of head_dim d."""
        room = lambda width: torch.empty((capacity, width), dtype=torch.uint8, device=device)
        return cls(room(d // 2), room(d // 32), room(d // 2), room(d // 32))


def tensor_view(t: torch.Tensor, seq_start: Optional[Sequence[int]] = None) -> _CTensor:
    """Describe a [B, H, T, d] device tensor (any strides with a contiguous last axis)."""
    assert t.is_cuda and t.dim() == 4 and t.stride(3) == 1, "need a [B,H,T,d] device tensor with contiguous d"
    v = _CTensor(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), None)
    if seq_start is not None:
        arr = (ct.c_int32 * len(seq_start))(*[int(x) for x in seq_start])
        v._keep = arr
        v.seq_start = ct.cast(arr, ct.POINTER(ct.c_int32))
    v._tensor = t
    return v


def _as_view(t) -> _CTensor:
    return t if isinstance(t, _CTensor) else tensor_view(t)


def _stream(stream) -> ct.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ct.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(status: int, what: str) -> None:
    if status != 0:
        detail = _lib.maskkv_last_error().decode() or _lib.maskkv_strerror(status).decode()
        raise MaskKVError(status, what, detail)


def _ptr(t: Optional[torch.Tensor]) -> ct.c_void_p:
    return ct.c_void_p(0 if t is None else t.data_ptr())


def _ws(t: Optional[torch.Tensor]):
    return _ptr(t), ct.c_size_t(0 if t is None else t.numel() * t.element_size())


def maskkv_version() -> int:
    return int(_lib.maskkv_version())


def _size(n: int, what: str) -> int:
    if n < 0:
        _check(-n, what)
    return n


def maskkv_score_workspace_bytes(desc: Desc) -> int:
    return _size(_native.score_ws(desc), "maskkv_score_workspace_bytes")


def maskkv_select_workspace_bytes(desc: Desc) -> int:
    return _size(_native.select_ws(desc), "maskkv_select_workspace_bytes")


def maskkv_attend_workspace_bytes(desc: Desc, full: bool) -> int:
    return _size(_native.attend_ws(desc, full), "maskkv_attend_workspace_bytes")


def maskkv_score(desc: Desc, Q_mask, K_full, scale: float, scores: torch.Tensor, score_stride: int,
                 prompt_mass: Optional[torch.Tensor], workspace: Optional[torch.Tensor], stream=None) -> None:
    status = _native.score(desc, Q_mask, K_full, scale, scores, score_stride, prompt_mass, workspace, stream)
    if status:
        _check(status, "maskkv_score")


def maskkv_score_given_lse(desc: Desc, Q_mask, K_full, scale: float, row_lse: torch.Tensor, scores: torch.Tensor,
                           score_stride: int, prompt_mass: Optional[torch.Tensor], workspace: Optional[torch.Tensor],
                           stream=None) -> None:
    """maskkv_score from the rows' natural-log softmax normalisers (as maskkv_attend_full returns them)."""
    status = _native.score_given_lse(desc, Q_mask, K_full, scale, row_lse, scores, score_stride, prompt_mass, workspace,
                                     stream)
    if status:
        _check(status, "maskkv_score_given_lse")


def maskkv_score_static(desc: Desc, Q_mask, K_full, scale: float, scores: torch.Tensor, score_stride: int,
                        prompt_mass: Optional[torch.Tensor], stream=None) -> None:
    """maskkv_score with the library's own static scratch array instead of a caller workspace."""
    status = _native.score_static(desc, Q_mask, K_full, scale, scores, score_stride, prompt_mass, stream)
    if status:
        _check(status, "maskkv_score_static")


def maskkv_select(desc: Desc, scores: torch.Tensor, score_stride: int, pool_window: int, pool_mode: int,
                  budgets: torch.Tensor, idx: torch.Tensor, cu_budget: torch.Tensor, capacity: int,
                  workspace: Optional[torch.Tensor], stream=None, budgets_host: Optional[Sequence[int]] = None) -> None:
    status = _native.select(desc, scores, score_stride, pool_window, pool_mode, budgets, budgets_host, idx, cu_budget,
                            capacity, workspace, stream)
    if status:
        _check(status, "maskkv_select")


def maskkv_compact(desc: Desc, K, V, idx: torch.Tensor, cu_budget: torch.Tensor, capacity: int,
                   Kc: torch.Tensor, Vc: torch.Tensor, stream=None) -> None:
    status = _native.compact(desc, K, V, idx, cu_budget, capacity, Kc, Vc, stream)
    if status:
        _check(status, "maskkv_compact")


def maskkv_attend(desc: Desc, Q_resp, Kc: torch.Tensor, Vc: torch.Tensor, cu_budget: torch.Tensor, capacity: int,
                  K_resp, V_resp, scale: float, O, lse: Optional[torch.Tensor],
                  workspace: Optional[torch.Tensor], stream=None) -> None:
    status = _native.attend(desc, Q_resp, Kc, Vc, cu_budget, capacity, K_resp, V_resp, scale, O, lse, workspace, stream)
    if status:
        _check(status, "maskkv_attend")


def maskkv_attend_full(desc: Desc, Q_resp, K_full, V_full, scale: float, O, lse: Optional[torch.Tensor],
                       workspace: Optional[torch.Tensor], stream=None) -> None:
    status = _native.attend_full(desc, Q_resp, K_full, V_full, scale, O, lse, workspace, stream)
    if status:
        _check(status, "maskkv_attend_full")


def maskkv_compact_mx(desc: Desc, K, V, idx: torch.Tensor, cu_budget: torch.Tensor, capacity: int, cache: MxCache,
                      stream=None) -> None:
    """maskkv_compact into a cache in 4 bits."""
    status = _native.compact_mx(desc, K, V, idx, cu_budget, capacity, cache, stream)
    if status:
        _check(status, "maskkv_compact_mx")


def maskkv_expand_mx(desc: Desc, cache: MxCache, cu_budget: torch.Tensor, capacity: int, Kc: torch.Tensor, Vc: torch.Tensor,
                     stream=None) -> None:
    """The values that a cache in 4 bits stands for, as packed rows in the description's dtype."""
    status = _native.expand_mx(desc, cache, cu_budget, capacity, Kc, Vc, stream)
    if status:
        _check(status, "maskkv_expand_mx")


def maskkv_attend_mx_workspace_bytes(desc: Desc, capacity: int) -> int:
    return _size(_native.attend_mx_ws(desc, capacity), "maskkv_attend_mx_workspace_bytes")


def maskkv_attend_mx(desc: Desc, Q_resp, cache: MxCache, cu_budget: torch.Tensor, capacity: int, K_resp, V_resp, scale: float,
                     O, lse: Optional[torch.Tensor], workspace: Optional[torch.Tensor], stream=None) -> None:
    """maskkv_attend over a cache in 4 bits."""
    status = _native.attend_mx(desc, Q_resp, cache, cu_budget, capacity, K_resp, V_resp, scale, O, lse, workspace, stream)
    if status:
        _check(status, "maskkv_attend_mx")


def maskkv_accumulate(desc: Desc, Q_resp, Kc: torch.Tensor, cu_budget: torch.Tensor, capacity: int, scale: float,
                      row_lse: torch.Tensor, decay: float, weights_in: Optional[torch.Tensor], weights_out: torch.Tensor,
                      stream=None) -> None:
    """decay * weights_in + the attention that each cached row gets; weights_in may be weights_out, or None with decay 0."""
    status = _native.accumulate(desc, Q_resp, Kc, cu_budget, capacity, scale, row_lse, decay, weights_in, weights_out, stream)
    if status:
        _check(status, "maskkv_accumulate")


def maskkv_accumulate_mx(desc: Desc, Q_resp, cache: MxCache, cu_budget: torch.Tensor, capacity: int, scale: float,
                         row_lse: torch.Tensor, decay: float, weights_in: Optional[torch.Tensor], weights_out: torch.Tensor,
                         stream=None) -> None:
    """maskkv_accumulate over the keys of a cache in 4 bits."""
    status = _native.accumulate_mx(desc, Q_resp, cache, cu_budget, capacity, scale, row_lse, decay, weights_in, weights_out, stream)
    if status:
        _check(status, "maskkv_accumulate_mx")


def maskkv_evict(desc: Desc, weights: torch.Tensor, cu_budget: torch.Tensor, capacity: int, budgets: torch.Tensor,
                 Kc: torch.Tensor, Vc: torch.Tensor, idx: Optional[torch.Tensor], Kc_out: torch.Tensor, Vc_out: torch.Tensor,
                 idx_out: Optional[torch.Tensor], rows: torch.Tensor, weights_out: Optional[torch.Tensor],
                 cu_out: torch.Tensor, capacity_out: int, stream=None) -> None:
    """The rows of largest weight of every head, into a smaller cache; idx and idx_out (prompt positions) go together or are None."""
    status = _native.evict(desc, weights, cu_budget, capacity, budgets, Kc, Vc, idx, Kc_out, Vc_out, idx_out, rows, weights_out,
                           cu_out, capacity_out, stream)
    if status:
        _check(status, "maskkv_evict")


def maskkv_evict_mx(desc: Desc, weights: torch.Tensor, cu_budget: torch.Tensor, capacity: int, budgets: torch.Tensor,
                    cache: MxCache, idx: Optional[torch.Tensor], cache_out: MxCache, idx_out: Optional[torch.Tensor],
                    rows: torch.Tensor, weights_out: Optional[torch.Tensor], cu_out: torch.Tensor, capacity_out: int,
                    stream=None) -> None:
    """maskkv_evict of a cache in 4 bits."""
    status = _native.evict_mx(desc, weights, cu_budget, capacity, budgets, cache, idx, cache_out, idx_out, rows, weights_out,
                              cu_out, capacity_out, stream)
    if status:
        _check(status, "maskkv_evict_mx")


def maskkv_head_budgets(desc: Desc, prompt_mass: torch.Tensor, k_l: int, alpha: float, budgets: torch.Tensor,
                        stream=None) -> None:
    status = _native.head_budgets(desc, prompt_mass, k_l, alpha, budgets, stream)
    if status:
        _check(status, "maskkv_head_budgets")


def maskkv_layer_importance_workspace_bytes() -> int:
    n = ct.c_size_t(0)
    _check(_lib.maskkv_layer_importance_workspace_bytes(ct.byref(n)), "maskkv_layer_importance_workspace_bytes")
    return int(n.value)


def maskkv_layer_importance(h_in: torch.Tensor, h_out: torch.Tensor, importance: torch.Tensor,
                            workspace: Optional[torch.Tensor], stream=None) -> None:
    """h_in, h_out: [n_tokens, hidden] device tensors of the same dtype and row stride; importance: float32 [1]."""
    status = _native.layer_importance(h_in, h_out, importance, workspace, stream)
    if status:
        _check(status, "maskkv_layer_importance")


def maskkv_layer_budgets(importance: Sequence[float], k_p: int, beta: float,
                         boundary: Optional[Sequence[int]] = None) -> list:
    """Host arithmetic: per-layer budgets k_l from the layer importances."""
    n = len(importance)
    imp = (ct.c_float * n)(*[float(x) for x in importance])
    out = (ct.c_int64 * n)()
    if boundary is None:
        bptr, nb = None, 0
    else:
        barr = (ct.c_int32 * len(boundary))(*[int(x) for x in boundary])
        bptr, nb = barr, len(boundary)
    _check(_lib.maskkv_layer_budgets(imp, ct.c_int32(n), ct.c_int64(int(k_p)), ct.c_float(beta), bptr, ct.c_int32(nb),
                                     out), "maskkv_layer_budgets")
    return [int(x) for x in out]


def maskkv_value_shift(V_now: torch.Tensor, V_prev: torch.Tensor, delta: float, cos: torch.Tensor,
                       refresh: torch.Tensor, count: torch.Tensor, stream=None) -> None:
    """V_now, V_prev: [n_tokens, width] device tensors; cos: float32 [n]; refresh: int32 [n]; count: int32 [1]."""
    status = _native.value_shift(V_now, V_prev, delta, cos, refresh, count, stream)
    if status:
        _check(status, "maskkv_value_shift")


def raw_library() -> ct.CDLL:
    """The loaded CDLL (for tests that exercise error paths with hand-built arguments)."""
    return _lib

"""Python binding of librelation.so (ctypes). Argument marshalling only: every
step of the operator runs in the library's HIP kernels; torch provides device
memory and the current stream.

Functions carry the C-ABI names (relation_fwd, relation_bwd,
relation_bwd_noalloc, relation_fwd_materialized, relation_bwd_materialized,
relation_exchange_allocation, relation_layer_fwd, relation_layer_bwd,
relation_decode, relation_decode_states, relation_decode_merge, ...). ``relation`` is the differentiable wrapper
(torch.autograd.Function) over relation_fwd / relation_bwd.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librelation.so")

REL_OK, REL_ERR_INVALID_ARG, REL_ERR_UNSUPPORTED, REL_ERR_WORKSPACE, REL_ERR_HIP = 0, -1, -2, -3, -4
REL_F32, REL_BF16 = 0, 1
TAU_S = 2.0


class RelProblem(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int64), ("H", ctypes.c_int64), ("T", ctypes.c_int64), ("D", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("tau_s", ctypes.c_float), ("scale", ctypes.c_float),
        ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
    ]


class RelLayerOpts(ctypes.Structure):
    _fields_ = [("rope_base", ctypes.c_double), ("givens", ctypes.c_int32), ("transport", ctypes.c_int32)]


class RelPages(ctypes.Structure):
    _fields_ = [("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int64), ("H", ctypes.c_int64),
                ("D", ctypes.c_int64), ("dtype", ctypes.c_int32), ("stride_page", ctypes.c_int64),
                ("stride_head", ctypes.c_int64), ("stride_token", ctypes.c_int64)]


class RelPageMap(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("table_width", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("max_tokens", ctypes.c_int64), ("num_free", ctypes.c_int64)]


class RelAppend(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("Hq", ctypes.c_int64), ("D", ctypes.c_int64), ("q_token", ctypes.c_int64),
                ("q_head", ctypes.c_int64), ("kv_token", ctypes.c_int64), ("kv_head", ctypes.c_int64),
                ("rope_base", ctypes.c_double), ("givens", ctypes.c_int32)]


class RelPagedQuery(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("Hq", ctypes.c_int64), ("table_width", ctypes.c_int64),
                ("max_length", ctypes.c_int64), ("tau_s", ctypes.c_float), ("scale", ctypes.c_float)]


class RelSample(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("V", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("stride_logits", ctypes.c_int64), ("stride_noise", ctypes.c_int64)]


REL_GIVENS = {None: 0, "A": 1, "B": 2}
REL_TRANSPORT = {"full": 0, "exchange": 1}
ROPE_BASE = 1.0e4

_P = ctypes.c_void_p
_PP = ctypes.POINTER(RelProblem)
_PO = ctypes.POINTER(RelLayerOpts)
_SIGS = {
    "relation_fwd": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "relation_exchange_allocation": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P]),
    "relation_bwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(RelProblem)]),
    "relation_bwd": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                    _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_bwd_deterministic": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                                  _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_bwd_noalloc_max_scratch_bytes": (ctypes.c_size_t, []),
    "relation_bwd_noalloc": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                            _P, _P, _P, _P]),
    "relation_fwd_materialized_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(RelProblem)]),
    "relation_fwd_materialized": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P,
                                                 _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_bwd_materialized_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(RelProblem)]),
    "relation_bwd_materialized": (ctypes.c_int, [ctypes.POINTER(RelProblem), _P, _P, _P, _P, _P, _P, _P, _P,
                                                 _P, _P, ctypes.c_size_t, _P]),
    "relation_layer_saved_bytes": (ctypes.c_size_t, [_PP, _PO]),
    "relation_layer_fwd_workspace_bytes": (ctypes.c_size_t, [_PP, _PO]),
    "relation_layer_fwd": (ctypes.c_int, [_PP, _PO, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P,
                                          ctypes.c_size_t, _P]),
    "relation_layer_bwd_workspace_bytes": (ctypes.c_size_t, [_PP, _PO]),
    "relation_layer_bwd": (ctypes.c_int, [_PP, _PO, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t,
                                          _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_decode_workspace_bytes": (ctypes.c_size_t, [_PP]),
    "relation_decode": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_decode_states": (ctypes.c_int, [_PP, _P, _P, _P, _P, ctypes.c_int32, ctypes.c_int32,
                                              ctypes.c_int32, _P, _P]),
    "relation_decode_merge": (ctypes.c_int, [_PP, ctypes.c_int32, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "relation_linear_fwd_workspace_bytes": (ctypes.c_size_t, [_PP]),
    "relation_linear_fwd": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_linear_bwd_workspace_bytes": (ctypes.c_size_t, [_PP]),
    "relation_linear_bwd": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_linear_gated_fwd_workspace_bytes": (ctypes.c_size_t, [_PP, ctypes.c_int32]),
    "relation_linear_gated_fwd": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, ctypes.c_int32, ctypes.c_float, _P,
                                                 _P, _P, ctypes.c_size_t, _P]),
    "relation_linear_gated_bwd_workspace_bytes": (ctypes.c_size_t, [_PP, ctypes.c_int32]),
    "relation_linear_gated_bwd": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, ctypes.c_int32, ctypes.c_float, _P,
                                                 _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "relation_page_map": (ctypes.c_int, [ctypes.POINTER(RelPageMap)] + [_P] * 10),
    "relation_paged_append": (ctypes.c_int, [ctypes.POINTER(RelPages), ctypes.POINTER(RelAppend)] + [_P] * 10),
    "relation_paged_decode_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(RelPages),
                                                                ctypes.POINTER(RelPagedQuery)]),
    "relation_paged_decode": (ctypes.c_int, [ctypes.POINTER(RelPages), ctypes.POINTER(RelPagedQuery)] + [_P] * 9 +
                              [ctypes.c_size_t, _P]),
    "relation_sample_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(RelSample)]),
    "relation_sample": (ctypes.c_int, [ctypes.POINTER(RelSample)] + [_P] * 9 + [ctypes.c_size_t, _P]),
    "relation_profile_arm": (ctypes.c_int, [ctypes.c_char_p, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]),
    "relation_profile_disarm": (ctypes.c_int, []),
    "relation_mfma_peak_flops": (ctypes.c_int64, [ctypes.c_int, ctypes.c_int]),
    "relation_mfma_peak_probe": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, _P, _P, _P]),
    "relation_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "relation_last_error": (ctypes.c_char_p, []),
    "relation_abi_version": (ctypes.c_int, []),
}

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load librelation.so once. Raises if it has not been built: there is no
    fallback implementation."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"librelation.so not found at {path}; build it with "
                           "`python -m paper_2608_20172_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int, what: str) -> None:
    if status != REL_OK:
        lib = load_library()
        msg = lib.relation_status_string(status).decode()
        detail = lib.relation_last_error().decode()
        raise RuntimeError(f"{what} failed: {msg} ({status}): {detail}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return REL_BF16
    if dt == torch.float32:
        return REL_F32
    raise TypeError(f"unsupported dtype {dt}; use torch.bfloat16 or torch.float32")


def make_problem(q: torch.Tensor, tau_s: float = TAU_S, scale: Optional[float] = None) -> RelProblem:
    if q.dim() != 4:
        raise ValueError("tensors must be [B, H, T, D]")
    B, H, T, D = q.shape
    sb, sh, st, sd = q.stride()
    if sd != 1:
        raise ValueError("the last dimension must be contiguous")
    return RelProblem(B, H, T, D, _dtype_code(q.dtype), 1, float(tau_s),
                      0.0 if scale is None else float(scale), sb, sh, st)


def _same_layout(ref: torch.Tensor, *ts: torch.Tensor) -> list:
    out = []
    shape, strides, dtype, device = ref.shape, ref.stride(), ref.dtype, ref.device
    for t in ts:
        if t.shape != shape or t.dtype != dtype or t.device != device:
            raise ValueError("q, k, v (and o, dout) must share shape, dtype and device")
        if t.stride() != strides:
            t = torch.empty_strided(shape, strides, dtype=dtype, device=device).copy_(t)
        out.append(t)
    return out


def _dense(t: torch.Tensor, device, dtype) -> torch.Tensor:
    """``t`` on ``device`` in ``dtype``, contiguous: itself where it is (0.4 us,
    the three calls 1.6)."""
    if t.dtype == dtype and t.device == device and t.is_contiguous():
        return t
    return t.detach().to(device=device, dtype=dtype).contiguous()


def _lam_tensor(lam, device) -> torch.Tensor:
    if isinstance(lam, torch.Tensor):
        if lam.numel() != 1:
            raise ValueError("lambda must be a single scalar")
        return _dense(lam, device, torch.float32)
    return torch.tensor([float(lam)], dtype=torch.float32, device=device)


def _stream() -> int:
    # the current stream's handle without a Stream object: 0.4 against 2.8 us, and
    # 16 us on autograd's thread, whose caches the caller's thread has just emptied
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _layout_like(q: torch.Tensor) -> torch.Tensor:
    # A dense [B, H, T, D] tensor keeps q's stride order; q's own strides are
    # reused so that every tensor shares (stride_b, stride_h, stride_t).
    return torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)


def relation_fwd(q, k, v, lam, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                 want_row_stat: bool = True, want_masses: bool = False, want_lse: bool = False):
    """Fused forward. Returns dict(o, row_stat, self_mass, exch_mass, exch_lse);
    outputs that were not requested are None."""
    lib = load_library()
    k, v = _same_layout(q, k, v)
    p = make_problem(q, tau_s, scale)
    B, H, T, D = q.shape
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    o = _layout_like(q)
    rows = lambda: torch.empty((B, H, T), dtype=torch.float32, device=dev)
    row_stat = rows() if want_row_stat else None
    self_mass = rows() if want_masses else None
    exch_mass = rows() if want_masses else None
    exch_lse = rows() if want_lse else None
    st = lib.relation_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lam_t), _ptr(o),
                          _ptr(row_stat), _ptr(self_mass), _ptr(exch_mass), _ptr(exch_lse), _stream())
    _check(st, "relation_fwd")
    return {"o": o, "row_stat": row_stat, "self_mass": self_mass, "exch_mass": exch_mass,
            "exch_lse": exch_lse}


def relation_exchange_allocation(q, k, exch_lse, *, tau_s: float = TAU_S, scale: Optional[float] = None):
    """pi_ij = exp(E_ij - L^E_i) for j < i (dense [B, H, T, T] fp32)."""
    lib = load_library()
    (k,) = _same_layout(q, k)
    p = make_problem(q, tau_s, scale)
    B, H, T, D = q.shape
    pi = torch.empty((B, H, T, T), dtype=torch.float32, device=q.device)
    lse = exch_lse.contiguous().to(torch.float32)
    st = lib.relation_exchange_allocation(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(lse), _ptr(pi), _stream())
    _check(st, "relation_exchange_allocation")
    return pi


def relation_bwd_workspace_bytes(q, *, tau_s: float = TAU_S, scale: Optional[float] = None) -> int:
    lib = load_library()
    p = make_problem(q, tau_s, scale)
    return int(lib.relation_bwd_workspace_bytes(ctypes.byref(p)))


def relation_bwd(q, k, v, o, dout, lam, row_stat, *, tau_s: float = TAU_S,
                 scale: Optional[float] = None, want_dself: bool = False, workspace=None,
                 deterministic: bool = False):
    """Fused backward. Returns dict(dq, dk, dv, dlambda (1-element fp32 tensor), dself).
    deterministic=True calls relation_bwd_deterministic (bitwise repeatable dq)."""
    lib = load_library()
    k, v, o, dout = _same_layout(q, k, v, o, dout)
    p = make_problem(q, tau_s, scale)
    B, H, T, D = q.shape
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    dq, dk, dv = _layout_like(q), _layout_like(q), _layout_like(q)
    dlam = torch.empty((1,), dtype=torch.float32, device=dev)
    dself = torch.empty((B, H, T), dtype=torch.float32, device=dev) if want_dself else None
    nbytes = int(lib.relation_bwd_workspace_bytes(ctypes.byref(p)))
    if workspace is None or workspace.numel() * workspace.element_size() < nbytes:
        workspace = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    rs = row_stat.contiguous()
    fn = lib.relation_bwd_deterministic if deterministic else lib.relation_bwd
    st = fn(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lam_t),
            _ptr(rs), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlam), _ptr(dself),
            _ptr(workspace), workspace.numel() * workspace.element_size(), _stream())
    _check(st, "relation_bwd_deterministic" if deterministic else "relation_bwd")
    return {"dq": dq, "dk": dk, "dv": dv, "dlambda": dlam, "dself": dself}


def relation_bwd_noalloc(q, k, v, o, dout, lam, row_stat, *, tau_s: float = TAU_S,
                         scale: Optional[float] = None, want_dself: bool = False, out=None):
    """relation_bwd through the entry point that allocates nothing on the device
    (its scratch is the library's own per-device array). ``out`` may hold
    preallocated dq, dk, dv, dlambda (and dself) tensors. Returns the same dict."""
    lib = load_library()
    k, v, o, dout = _same_layout(q, k, v, o, dout)
    p = make_problem(q, tau_s, scale)
    B, H, T, D = q.shape
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    if out is None:
        out = {"dq": _layout_like(q), "dk": _layout_like(q), "dv": _layout_like(q),
               "dlambda": torch.empty((1,), dtype=torch.float32, device=dev),
               "dself": torch.empty((B, H, T), dtype=torch.float32, device=dev) if want_dself else None}
    rs = row_stat.contiguous()
    st = lib.relation_bwd_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lam_t),
                                  _ptr(rs), _ptr(out["dq"]), _ptr(out["dk"]), _ptr(out["dv"]), _ptr(out["dlambda"]),
                                  _ptr(out.get("dself")), _stream())
    _check(st, "relation_bwd_noalloc")
    return out


def relation_fwd_materialized_workspace_bytes(q, *, tau_s: float = TAU_S,
                                              scale: Optional[float] = None) -> int:
    lib = load_library()
    p = make_problem(q, tau_s, scale)
    return int(lib.relation_fwd_materialized_workspace_bytes(ctypes.byref(p)))


def relation_fwd_materialized(q, k, v, lam, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                              want_R: bool = False, want_F: bool = False, want_pi: bool = False,
                              want_masses: bool = False, workspace=None):
    """Materialised baseline. Returns dict(o, R, F, pi, self_mass, exch_mass)."""
    lib = load_library()
    k, v = _same_layout(q, k, v)
    p = make_problem(q, tau_s, scale)
    B, H, T, D = q.shape
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    o = _layout_like(q)
    mat = lambda: torch.empty((B, H, T, T), dtype=torch.float32, device=dev)
    rows = lambda: torch.empty((B, H, T), dtype=torch.float32, device=dev)
    R = mat() if want_R else None
    F = mat() if want_F else None
    pi = mat() if want_pi else None
    sm = rows() if want_masses else None
    em = rows() if want_masses else None
    nbytes = int(lib.relation_fwd_materialized_workspace_bytes(ctypes.byref(p)))
    if workspace is None or workspace.numel() * workspace.element_size() < nbytes:
        workspace = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    st = lib.relation_fwd_materialized(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lam_t), _ptr(o),
                                       _ptr(R), _ptr(F), _ptr(pi), _ptr(sm), _ptr(em), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream())
    _check(st, "relation_fwd_materialized")
    return {"o": o, "R": R, "F": F, "pi": pi, "self_mass": sm, "exch_mass": em}


def relation_bwd_materialized_workspace_bytes(q, *, tau_s: float = TAU_S,
                                              scale: Optional[float] = None) -> int:
    lib = load_library()
    p = make_problem(q, tau_s, scale)
    return int(lib.relation_bwd_materialized_workspace_bytes(ctypes.byref(p)))


def relation_bwd_materialized(q, k, v, dout, lam, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                              workspace=None):
    """Materialised backward baseline (every T x T tensor in HBM). Returns
    dict(dq, dk, dv, dlambda (1-element fp32 tensor))."""
    lib = load_library()
    k, v, dout = _same_layout(q, k, v, dout)
    p = make_problem(q, tau_s, scale)
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    dq, dk, dv = _layout_like(q), _layout_like(q), _layout_like(q)
    dlam = torch.empty((1,), dtype=torch.float32, device=dev)
    nbytes = int(lib.relation_bwd_materialized_workspace_bytes(ctypes.byref(p)))
    if workspace is None or workspace.numel() * workspace.element_size() < nbytes:
        workspace = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    st = lib.relation_bwd_materialized(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(lam_t),
                                       _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlam), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream())
    _check(st, "relation_bwd_materialized")
    return {"dq": dq, "dk": dk, "dv": dv, "dlambda": dlam}


def make_layer_opts(pairing: Optional[str] = None, rope_base: float = ROPE_BASE,
                    transport: str = "full") -> RelLayerOpts:
    if pairing not in REL_GIVENS:
        raise ValueError("pairing must be None, 'A' or 'B'")
    if transport not in REL_TRANSPORT:
        raise ValueError("transport must be 'full' or 'exchange'")
    return RelLayerOpts(float(rope_base or 0.0), REL_GIVENS[pairing], REL_TRANSPORT[transport])


def _theta_tensor(theta, H: int, device):
    if theta is None:
        return None
    if isinstance(theta, torch.Tensor):
        t = _dense(theta, device, torch.float32)
    else:
        t = torch.as_tensor(theta, dtype=torch.float32, device=device).reshape(-1).contiguous()
    if t.numel() != H // 2:
        raise ValueError("theta must hold H/2 angles")
    return t


def _workspace(nbytes: int, ws, device):
    if nbytes == 0:
        return None
    if ws is None or ws.numel() * ws.element_size() < nbytes:
        ws = torch.empty((nbytes,), dtype=torch.uint8, device=device)
    return ws


def _layer_size(fn: str, q, pairing, rope_base, tau_s, scale) -> int:
    p, o = make_problem(q, tau_s, scale), make_layer_opts(pairing, rope_base)
    return int(getattr(load_library(), fn)(ctypes.byref(p), ctypes.byref(o)))


def relation_layer_saved_bytes(q, *, pairing: Optional[str] = None, rope_base: float = ROPE_BASE,
                               tau_s: float = TAU_S, scale: Optional[float] = None) -> int:
    return _layer_size("relation_layer_saved_bytes", q, pairing, rope_base, tau_s, scale)


def relation_layer_fwd_workspace_bytes(q, *, pairing: Optional[str] = None, rope_base: float = ROPE_BASE,
                                       tau_s: float = TAU_S, scale: Optional[float] = None) -> int:
    return _layer_size("relation_layer_fwd_workspace_bytes", q, pairing, rope_base, tau_s, scale)


def relation_layer_bwd_workspace_bytes(q, *, pairing: Optional[str] = None, rope_base: float = ROPE_BASE,
                                       tau_s: float = TAU_S, scale: Optional[float] = None) -> int:
    return _layer_size("relation_layer_bwd_workspace_bytes", q, pairing, rope_base, tau_s, scale)


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def relation_layer_fwd(q, k, v, lam, theta=None, *, pairing: Optional[str] = None,
                       rope_base: float = ROPE_BASE, transport: str = "full", tau_s: float = TAU_S,
                       scale: Optional[float] = None, keep_saved: bool = True, workspace=None):
    """Layer forward: RoPE on q, k (rope_base 0: off), Givens mixing of v over
    head pairs ("A", "B" or None) with angles ``theta`` [H/2], then the fused
    operator. Any head width up to 128. Returns dict(o, row_stat, saved):
    ``saved`` (a uint8 device tensor, or None) holds the prepared operands for
    relation_layer_bwd; with keep_saved=False it is None and the backward pass
    prepares them again."""
    lib = load_library()
    k, v = _same_layout(q, k, v)
    p = make_problem(q, tau_s, scale)
    opts = make_layer_opts(pairing, rope_base, transport)
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    th = _theta_tensor(theta, q.shape[1], dev) if pairing else None
    o = _layout_like(q)
    rs = torch.empty(q.shape[:3], dtype=torch.float32, device=dev)
    nsaved = int(lib.relation_layer_saved_bytes(ctypes.byref(p), ctypes.byref(opts)))
    saved = torch.empty((nsaved,), dtype=torch.uint8, device=dev) if keep_saved and nsaved else None
    ws = None if saved is not None else _workspace(
        int(lib.relation_layer_fwd_workspace_bytes(ctypes.byref(p), ctypes.byref(opts))), workspace, dev)
    st = lib.relation_layer_fwd(ctypes.byref(p), ctypes.byref(opts), _ptr(q), _ptr(k), _ptr(v), _ptr(lam_t),
                                _ptr(th), _ptr(o), _ptr(rs), _ptr(saved), _nbytes(saved), _ptr(ws), _nbytes(ws),
                                _stream())
    _check(st, "relation_layer_fwd")
    return {"o": o, "row_stat": rs, "saved": saved}


def relation_layer_bwd(q, k, v, o, dout, lam, row_stat, theta=None, *, saved=None, pairing: Optional[str] = None,
                       rope_base: float = ROPE_BASE, transport: str = "full", tau_s: float = TAU_S,
                       scale: Optional[float] = None, workspace=None):
    """Layer backward; ``saved`` is the forward call's (None: recompute).
    Returns dict(dq, dk, dv, dlambda [1], dtheta [H/2] or None)."""
    lib = load_library()
    k, v, o, dout = _same_layout(q, k, v, o, dout)
    p = make_problem(q, tau_s, scale)
    opts = make_layer_opts(pairing, rope_base, transport)
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    H = q.shape[1]
    th = _theta_tensor(theta, H, dev) if pairing else None
    rs = row_stat.contiguous()
    dq, dk, dv = _layout_like(q), _layout_like(q), _layout_like(q)
    dlam = torch.empty((1,), dtype=torch.float32, device=dev)
    dth = torch.empty((H // 2,), dtype=torch.float32, device=dev) if pairing else None
    nbytes = int(lib.relation_layer_bwd_workspace_bytes(ctypes.byref(p), ctypes.byref(opts)))
    ws = _workspace(max(nbytes, 1), workspace, dev)
    st = lib.relation_layer_bwd(ctypes.byref(p), ctypes.byref(opts), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                _ptr(dout), _ptr(lam_t), _ptr(th), _ptr(rs), _ptr(saved), _nbytes(saved),
                                _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlam), _ptr(dth), _ptr(ws), _nbytes(ws),
                                _stream())
    _check(st, "relation_layer_bwd")
    return {"dq": dq, "dk": dk, "dv": dv, "dlambda": dlam, "dtheta": dth}


def _decode_io(q, k_cache, v_cache, lengths, tau_s, scale):
    v_cache = _same_layout(k_cache, v_cache)[0]
    B, H, T, D = k_cache.shape
    if q.shape != (B, H, D) or q.dtype != k_cache.dtype:
        raise ValueError("q must be [B, H, D] with the caches' dtype")
    q = q.contiguous()
    if not isinstance(lengths, torch.Tensor) or lengths.shape != (B,):
        lengths = torch.as_tensor(lengths, dtype=torch.int32, device=q.device).reshape(B)
    lengths = _dense(lengths, q.device, torch.int32)
    return q, k_cache, v_cache, lengths, make_problem(k_cache, tau_s, scale)


def relation_decode(q, k_cache, v_cache, lengths, lam, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                    workspace=None):
    """One decode step: q [B, H, D] of the new tokens, caches [B, H, Tmax, D]
    holding lengths[b] entries each (the new token's own entry last).
    Returns dict(o [B, H, D], row_stat [B, H])."""
    lib = load_library()
    q, k_cache, v_cache, lengths, p = _decode_io(q, k_cache, v_cache, lengths, tau_s, scale)
    dev = q.device
    lam_t = _lam_tensor(lam, dev)
    o = torch.empty_like(q)
    rs = torch.empty(q.shape[:2], dtype=torch.float32, device=dev)
    ws = _workspace(max(1, int(lib.relation_decode_workspace_bytes(ctypes.byref(p)))), workspace, dev)
    st = lib.relation_decode(ctypes.byref(p), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lengths), _ptr(lam_t),
                             _ptr(o), _ptr(rs), _ptr(ws), _nbytes(ws), _stream())
    _check(st, "relation_decode")
    return {"o": o, "row_stat": rs}


def relation_decode_states(q, k_cache, v_cache, lengths, key_begin: int, key_end: int, nstates: int = 1, *,
                           tau_s: float = TAU_S, scale: Optional[float] = None):
    """Exchange scan states [nstates, B*H, D + 2] (m, l, z) of cache keys
    [key_begin, key_end) for the new tokens' rows."""
    lib = load_library()
    q, k_cache, v_cache, lengths, p = _decode_io(q, k_cache, v_cache, lengths, tau_s, scale)
    B, H, _, D = k_cache.shape
    states = torch.empty((nstates, B * H, D + 2), dtype=torch.float32, device=q.device)
    st = lib.relation_decode_states(ctypes.byref(p), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lengths),
                                    int(key_begin), int(key_end), int(nstates), _ptr(states), _stream())
    _check(st, "relation_decode_states")
    return states


def relation_decode_merge(states, q, k_cache, v_cache, lengths, lam, *, tau_s: float = TAU_S,
                          scale: Optional[float] = None):
    """Merge states [n, B*H, D + 2] with the Self entry; dict(o, row_stat)."""
    lib = load_library()
    q, k_cache, v_cache, lengths, p = _decode_io(q, k_cache, v_cache, lengths, tau_s, scale)
    dev = q.device
    states = states.to(dtype=torch.float32).contiguous()
    lam_t = _lam_tensor(lam, dev)
    o = torch.empty_like(q)
    rs = torch.empty(q.shape[:2], dtype=torch.float32, device=dev)
    st = lib.relation_decode_merge(ctypes.byref(p), int(states.shape[0]), _ptr(states), _ptr(q), _ptr(k_cache),
                                   _ptr(v_cache), _ptr(lengths), _ptr(lam_t), _ptr(o), _ptr(rs), _stream())
    _check(st, "relation_decode_merge")
    return {"o": o, "row_stat": rs}


def relation_linear_fwd(p1, p2, v, g, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                        want_state: bool = False, workspace=None):
    """Linear Relation forward over [B, H, T, D] tensors; g is the fp32
    log-retention. Returns dict(o, state (the [B, H, D, D] state after the last
    token, or None))."""
    lib = load_library()
    p2, v = _same_layout(p1, p2, v)
    p = make_problem(p1, tau_s, scale)
    dev = p1.device
    g = _dense(g, dev, torch.float32)
    if g.shape != p1.shape:
        raise ValueError("g must have the shape of p1")
    o = _layout_like(p1)
    B, H, T, D = p1.shape
    state = torch.empty((B, H, D, D), dtype=torch.float32, device=dev) if want_state else None
    ws = _workspace(max(1, int(lib.relation_linear_fwd_workspace_bytes(ctypes.byref(p)))), workspace, dev)
    st = lib.relation_linear_fwd(ctypes.byref(p), _ptr(p1), _ptr(p2), _ptr(v), _ptr(g), _ptr(o), _ptr(state),
                                 _ptr(ws), _nbytes(ws), _stream())
    _check(st, "relation_linear_fwd")
    return {"o": o, "state": state}


def relation_linear_bwd(p1, p2, v, g, dout, *, tau_s: float = TAU_S, scale: Optional[float] = None,
                        workspace=None):
    """Linear Relation backward. Returns dict(dp1, dp2, dv, dg (fp32))."""
    lib = load_library()
    p2, v, dout = _same_layout(p1, p2, v, dout)
    p = make_problem(p1, tau_s, scale)
    dev = p1.device
    g = _dense(g, dev, torch.float32)
    dp1, dp2, dv = _layout_like(p1), _layout_like(p1), _layout_like(p1)
    dg = torch.empty(p1.shape, dtype=torch.float32, device=dev)
    ws = _workspace(max(1, int(lib.relation_linear_bwd_workspace_bytes(ctypes.byref(p)))), workspace, dev)
    st = lib.relation_linear_bwd(ctypes.byref(p), _ptr(p1), _ptr(p2), _ptr(v), _ptr(g), _ptr(dout), _ptr(dp1),
                                 _ptr(dp2), _ptr(dv), _ptr(dg), _ptr(ws), _nbytes(ws), _stream())
    _check(st, "relation_linear_bwd")
    return {"dp1": dp1, "dp2": dp2, "dv": dv, "dg": dg}


def _gate_params(a_log, dt_bias, p1):
    H, D = p1.shape[1], p1.shape[3]
    out = []
    for name, x in (("a_log", a_log), ("dt_bias", dt_bias)):
        x = _dense(x, p1.device, torch.float32)
        if tuple(x.shape) != (H, D):
            raise ValueError(f"{name} must have shape [H, D] = [{H}, {D}]")
        out.append(x)
    return out


def relation_linear_gated_fwd(p1, p2, v, r, a_log, dt_bias, *, rope_dim: int = 0, rope_base: float = 1.0e4,
                              tau_s: float = TAU_S, scale: Optional[float] = None, want_state: bool = False,
                              workspace=None):
    """Linear Relation forward with the retention gate of eq. 15 formed in the
    kernels from r ([B, H, T, D] fp32) and a_log, dt_bias ([H, D] fp32), and
    RoPE over the first rope_dim channels of p1, p2 (0: none).
    Returns dict(o, state)."""
    lib = load_library()
    p2, v = _same_layout(p1, p2, v)
    p = make_problem(p1, tau_s, scale)
    dev = p1.device
    r = _dense(r, dev, torch.float32)
    if r.shape != p1.shape:
        raise ValueError("r must have the shape of p1")
    a_log, dt_bias = _gate_params(a_log, dt_bias, p1)
    o = _layout_like(p1)
    B, H, T, D = p1.shape
    state = torch.empty((B, H, D, D), dtype=torch.float32, device=dev) if want_state else None
    ws = _workspace(max(1, int(lib.relation_linear_gated_fwd_workspace_bytes(ctypes.byref(p), rope_dim))),
                    workspace, dev)
    st = lib.relation_linear_gated_fwd(ctypes.byref(p), _ptr(p1), _ptr(p2), _ptr(v), _ptr(r), _ptr(a_log),
                                       _ptr(dt_bias), rope_dim, rope_base, _ptr(o), _ptr(state), _ptr(ws),
                                       _nbytes(ws), _stream())
    _check(st, "relation_linear_gated_fwd")
    return {"o": o, "state": state}


def relation_linear_gated_bwd(p1, p2, v, r, a_log, dt_bias, dout, *, rope_dim: int = 0, rope_base: float = 1.0e4,
                              tau_s: float = TAU_S, scale: Optional[float] = None, workspace=None):
    """Backward of relation_linear_gated_fwd. Returns dict(dp1, dp2, dv, dr
    (fp32), da_log, ddt_bias ([H, D] fp32))."""
    lib = load_library()
    p2, v, dout = _same_layout(p1, p2, v, dout)
    p = make_problem(p1, tau_s, scale)
    dev = p1.device
    r = _dense(r, dev, torch.float32)
    a_log, dt_bias = _gate_params(a_log, dt_bias, p1)
    dp1, dp2, dv = _layout_like(p1), _layout_like(p1), _layout_like(p1)
    dr = torch.empty(p1.shape, dtype=torch.float32, device=dev)
    da_log, ddt_bias = torch.empty_like(a_log), torch.empty_like(dt_bias)
    ws = _workspace(max(1, int(lib.relation_linear_gated_bwd_workspace_bytes(ctypes.byref(p), rope_dim))),
                    workspace, dev)
    st = lib.relation_linear_gated_bwd(ctypes.byref(p), _ptr(p1), _ptr(p2), _ptr(v), _ptr(r), _ptr(a_log),
                                       _ptr(dt_bias), rope_dim, rope_base, _ptr(dout), _ptr(dp1), _ptr(dp2),
                                       _ptr(dv), _ptr(dr), _ptr(da_log), _ptr(ddt_bias), _ptr(ws), _nbytes(ws),
                                       _stream())
    _check(st, "relation_linear_gated_bwd")
    return {"dp1": dp1, "dp2": dp2, "dv": dv, "dr": dr, "da_log": da_log, "ddt_bias": ddt_bias}


# ---------------------------------------------------------------------------
# Serving from a paged cache
# ---------------------------------------------------------------------------
def _on_gpu(first, *rest) -> int:
    """The index of the GPU that all the given tensors (None apart) are on. A step of a serving loop is a few calls
    of microseconds: the checks of these functions are kept to one look at each tensor."""
    dev = first.get_device() if isinstance(first, torch.Tensor) else -1
    if dev < 0:
        raise ValueError("the tensors must be on the GPU")
    for t in rest:
        if t is not None and (not isinstance(t, torch.Tensor) or t.get_device() != dev):
            raise ValueError("all tensors must be on the GPU of the first")
    return dev


def _stream_on(dev: int) -> int:
    """The current stream, on the GPU that the tensors are on."""
    if torch.cuda.current_device() != dev:
        raise ValueError(f"the tensors are on GPU {dev}, the current one is {torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _given(out, name, shape, dtype, dev):
    """out[name] where the caller gives it (checked), or None."""
    t = None if out is None else out.get(name)
    if t is not None and (t.shape != torch.Size(shape) or t.dtype != dtype or t.get_device() != dev or
                          not t.is_contiguous()):
        raise ValueError(f"out[{name!r}] must be a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {dev}")
    return t


def _ready(t: torch.Tensor, dtype) -> torch.Tensor:
    """``t`` in ``dtype``, contiguous: itself where it is."""
    return t if t.dtype == dtype and t.is_contiguous() else t.detach().to(dtype).contiguous()


INT32_MAX = 2 ** 31 - 1


def _int32(t: torch.Tensor) -> torch.Tensor:
    """``t`` in int32, contiguous: itself where it is. A number past 32 bits becomes the nearest that fits, which is out
    of range for lengths, counts and page ids as the number itself is, and no bound for top_k; NaN becomes -1."""
    if t.dtype == torch.int32:
        return t if t.is_contiguous() else t.contiguous()
    t = t.detach()
    t = t.double().nan_to_num(nan=-1.0) if t.is_floating_point() else t.to(torch.int64)
    return t.clamp(-INT32_MAX - 1, INT32_MAX).to(torch.int32).contiguous()


def _positions(t: torch.Tensor) -> torch.Tensor:
    """Positions in int32; one past 32 bits becomes -1, a token that is not written."""
    p = _int32(t)
    return p if t.dtype == torch.int32 else torch.where(t.detach() > INT32_MAX, -1, p)


def make_pages(k_cache: torch.Tensor, v_cache: torch.Tensor) -> RelPages:
    """The pools [num_pages, H, page_size, D], with any strides that the library takes."""
    shape, strides, dt = k_cache.shape, k_cache.stride(), k_cache.dtype
    if len(shape) != 4:
        raise ValueError("caches must be [num_pages, H, page_size, D]")
    if v_cache.shape != shape or v_cache.stride() != strides or v_cache.dtype != dt:
        raise ValueError("k_cache and v_cache must share shape, strides and dtype")
    P, H, page, D = shape
    sp, sh, st, sd = strides
    if sd != 1 and D != 1:
        raise ValueError("the last dimension must be contiguous")
    # a stride over one entry says nothing
    return RelPages(P, page, H, D, _dtype_code(dt), sp if P > 1 else 0, sh if H > 1 else 0, st if page > 1 else 0)


def relation_page_map(cached, added, table, free_pages, page_size: int, max_tokens: int, *, out=None):
    """Block tables, slots and positions of a step. cached, added: int32 [B]; table: int32 [B, W], updated in
    place; free_pages: int32 [F]; max_tokens: the step's token buffers. Returns dict(table, lengths [B],
    row_start [B + 1], slots int64 [max_tokens], positions [max_tokens], counts [3]: pages taken, tokens mapped,
    requests not served), in the tensors of ``out`` where given. A request that is not served has length 0 there and
    keeps its place: where requests may wait for pages, the next step's cached is
    torch.where(m["lengths"] > 0, m["lengths"], cached)."""
    lib = load_library()
    i32 = torch.int32
    dev = _on_gpu(table, cached, added, free_pages)
    if table.dim() != 2 or table.dtype != i32 or not table.is_contiguous():
        raise ValueError("table must be a contiguous int32 [B, W] tensor")
    B, W = table.shape
    if cached.shape != (B,) or added.shape != (B,) or free_pages.dim() != 1:
        raise ValueError("cached and added must be [B], free_pages [F]")
    cached, added, free_pages = _int32(cached), _int32(added), _int32(free_pages)
    N = int(max_tokens)
    if N < 0:
        raise ValueError("max_tokens must not be negative")
    if out is None:  # one allocation for the int32 outputs
        lengths, row_start, positions, counts = table.new_empty(2 * B + N + 4).split_with_sizes((B, B + 1, N, 3))
        slots = table.new_empty(N, dtype=torch.int64)
    else:
        new = lambda name, n, dt: _given(out, name, (n,), dt, dev) if out.get(name) is not None else \
            table.new_empty(n, dtype=dt)
        lengths, row_start, positions = new("lengths", B, i32), new("row_start", B + 1, i32), new("positions", N, i32)
        counts, slots = new("counts", 3, i32), new("slots", N, torch.int64)
    m = RelPageMap(B, W, int(page_size), N, free_pages.shape[0])
    st = lib.relation_page_map(ctypes.byref(m), cached.data_ptr(), added.data_ptr(), free_pages.data_ptr(),
                               table.data_ptr(), lengths.data_ptr(), row_start.data_ptr(), slots.data_ptr(),
                               positions.data_ptr(), counts.data_ptr(), _stream_on(dev))
    if st:
        _check(st, "relation_page_map")
    return {"table": table, "lengths": lengths, "row_start": row_start, "slots": slots, "positions": positions,
            "counts": counts}


def _rows(t: torch.Tensor) -> torch.Tensor:
    return t if t.stride(2) == 1 or t.shape[2] == 1 else t.contiguous()


def relation_paged_append(k, v, k_cache, v_cache, slots, positions, *, q=None, theta=None,
                          pairing: Optional[str] = None, rope_base: float = ROPE_BASE, out=None):
    """New tokens' rows into the cache, in place: k (RoPE at the positions) and v (Givens mixing), [N, H, D], to
    slots (int64 [N], those in use all different) of the caches [num_pages, H, page_size, Dc], zero-padded to Dc (then
    relation_paged_decode needs head_dim=D). With q [N, Hq, D], returns the rotated and padded queries [N, Hq, Dc]
    (out["q"] where given), else None. rope_base 0 or None: no RoPE."""
    lib = load_library()
    dev = _on_gpu(k, v, k_cache, v_cache, slots, positions, q)
    c = make_pages(k_cache, v_cache)
    givens = REL_GIVENS.get(pairing)
    if givens is None:
        raise ValueError("pairing must be None, 'A' or 'B'")
    if k.dim() != 3 or k.shape[1] != c.H or k.dtype != k_cache.dtype:
        raise ValueError("k and v must be [N, H, D] with the caches' heads and dtype")
    N, H, D = k.shape
    k = _rows(k)
    ks = k.stride()
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("v must be as k")
    if v.stride() != ks:
        if 0 in ks:  # expanded keys: no layout that the values could be copied to
            k = k.contiguous()
            ks = k.stride()
        v = _same_layout(k, v)[0]
    if slots.shape != (N,) or positions.shape != (N,):
        raise ValueError("slots and positions must be [N]")
    slots, positions = _ready(slots, torch.int64), _positions(positions)
    th = None if theta is None else _theta_tensor(theta, H, k.device)
    if givens and th is None:
        raise ValueError("theta is required for Givens mixing")
    Hq = qt = qh = 0
    q_out = None
    if q is not None:
        if q.dim() != 3 or q.shape[0] != N or q.shape[2] != D or q.dtype != k.dtype:
            raise ValueError("q must be [N, Hq, D] with k's dtype")
        q = _rows(q)
        Hq = q.shape[1]
        qt, qh, _ = q.stride()
        q_out = _given(out, "q", (N, Hq, c.D), q.dtype, dev)
        if q_out is None:
            q_out = q.new_empty((N, Hq, c.D))
    n = RelAppend(N, Hq, D, qt, qh, ks[0], ks[1], float(rope_base or 0.0), givens)
    st = lib.relation_paged_append(ctypes.byref(c), ctypes.byref(n), _ptr(q), k.data_ptr(), v.data_ptr(),
                                   slots.data_ptr(), positions.data_ptr(), _ptr(th), _ptr(q_out), k_cache.data_ptr(),
                                   v_cache.data_ptr(), _stream_on(dev))
    if st:
        _check(st, "relation_paged_append")
    return q_out


def relation_paged_decode(q, k_cache, v_cache, table, lengths, lam, *, max_length: Optional[int] = None,
                          tau_s: float = TAU_S, scale: Optional[float] = None, head_dim: Optional[int] = None,
                          workspace=None, out=None):
    """One decode step over pages: q [B, Hq, D] of the new tokens, caches [num_pages, H, page_size, D] (Hq a
    multiple of H), table int32 [B, W], lengths int32 [B] (the new token's own entry last), max_length a bound of
    the lengths (default W * page_size). Returns dict(o [B, Hq, D], row_stat [B, Hq]).

    The default scale is 1/sqrt(head_dim), and head_dim defaults to the caches' width D. Where relation_paged_append
    padded narrower heads to D, the zeros change no product, but the scale is that of the true width: give it as
    head_dim (or give scale), or the rows differ from relation_layer_fwd's."""
    lib = load_library()
    dev = _on_gpu(q, k_cache, v_cache, table, lengths)
    c = make_pages(k_cache, v_cache)
    if q.dim() != 3 or q.shape[2] != c.D or q.dtype != k_cache.dtype:
        raise ValueError("q must be [B, Hq, D] with the caches' width and dtype")
    B, Hq, D = q.shape
    if table.dim() != 2 or table.shape[0] != B or lengths.shape != (B,):
        raise ValueError("table must be [B, W] and lengths [B]")
    if head_dim is not None:
        if scale is not None:
            raise ValueError("give scale or head_dim, not both")
        if not 1 <= head_dim <= D:
            raise ValueError(f"head_dim must be in 1 .. the caches' width {D}")
        scale = head_dim ** -0.5
    if not q.is_contiguous():
        q = q.contiguous()
    table, lengths = _int32(table), _int32(lengths)
    lam_t = _lam_tensor(lam, q.device)
    d = RelPagedQuery(B, Hq, table.shape[1], int(max_length or 0), tau_s, 0.0 if scale is None else scale)
    o, rs = _given(out, "o", (B, Hq, D), q.dtype, dev), _given(out, "row_stat", (B, Hq), torch.float32, dev)
    if o is None:
        o = torch.empty_like(q)
    if rs is None:
        rs = q.new_empty((B, Hq), dtype=torch.float32)
    need = lib.relation_paged_decode_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
    ws = _workspace(need, workspace, q.device) if need else None
    st = lib.relation_paged_decode(ctypes.byref(c), ctypes.byref(d), q.data_ptr(), k_cache.data_ptr(),
                                   v_cache.data_ptr(), table.data_ptr(), lengths.data_ptr(), lam_t.data_ptr(),
                                   o.data_ptr(), rs.data_ptr(), _ptr(ws), 0 if ws is None else _nbytes(ws), _stream_on(dev))
    if st:
        _check(st, "relation_paged_decode")
    return {"o": o, "row_stat": rs}


def _per_row(x, name, B, dtype, logits):
    """Pointer (None: off) and tensor of a sampling parameter."""
    if x is None:
        return None, None
    if not isinstance(x, torch.Tensor):
        if dtype == torch.int32:
            x = max(-1, min(x, INT32_MAX))
        x = logits.new_full((B,), x, dtype=dtype)
    elif x.shape != (B,) or x.get_device() != logits.get_device():
        raise ValueError(f"{name} must be a number, or [B] on the logits' GPU")
    else:
        x = _int32(x) if dtype == torch.int32 else _ready(x, dtype)
    return x.data_ptr(), x


def relation_sample(logits, noise, *, temperature=None, top_k=None, top_p=None, min_p=None, workspace=None, out=None):
    """One token of each row of logits [B, V], drawn by noise (fp32 [B, V], independent exponential variates).
    temperature, top_k, top_p, min_p: numbers, [B] tensors, or None (off). Returns dict(tokens int64 [B],
    logprob fp32 [B]: log softmax(logits / temperature) of the token)."""
    lib = load_library()
    dev = _on_gpu(logits, noise)
    if logits.dim() != 2 or noise.shape != logits.shape or noise.dtype != torch.float32:
        raise ValueError("logits must be [B, V] and noise fp32 [B, V]")
    B, V = logits.shape
    (sl, se), (sn, ne) = logits.stride(), noise.stride()
    if V > 1 and se != 1:
        logits, sl = logits.contiguous(), V
    if V > 1 and ne != 1:
        noise, sn = noise.contiguous(), V
    f32 = torch.float32
    pt, t1 = _per_row(temperature, "temperature", B, f32, logits)
    pk, t2 = _per_row(top_k, "top_k", B, torch.int32, logits)
    pp, t3 = _per_row(top_p, "top_p", B, f32, logits)
    pm, t4 = _per_row(min_p, "min_p", B, f32, logits)
    s = RelSample(B, V, _dtype_code(logits.dtype), sl, sn)
    tokens, logprob = _given(out, "tokens", (B,), torch.int64, dev), _given(out, "logprob", (B,), f32, dev)
    if tokens is None:
        tokens = noise.new_empty(B, dtype=torch.int64)
    if logprob is None:
        logprob = noise.new_empty(B)
    need = lib.relation_sample_workspace_bytes(ctypes.byref(s))
    ws = _workspace(need, workspace, logits.device) if need else None
    st = lib.relation_sample(ctypes.byref(s), logits.data_ptr(), noise.data_ptr(), pt, pk, pp, pm, tokens.data_ptr(),
                             logprob.data_ptr(), _ptr(ws), 0 if ws is None else _nbytes(ws), _stream_on(dev))
    if st:
        _check(st, "relation_sample")
    return {"tokens": tokens, "logprob": logprob}


def relation_profile_arm(kernel: str, events: list) -> None:
    """Record each listed torch.cuda.Event pair around successive launches of
    ``kernel`` ("fwd" or "bwd"); events = [start0, stop0, start1, stop1, ...]."""
    lib = load_library()
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _check(lib.relation_profile_arm(kernel.encode(), arr, len(events) // 2), "relation_profile_arm")
    relation_profile_arm._keep = arr


def relation_profile_disarm() -> int:
    return int(load_library().relation_profile_disarm())


class _RelationFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, lam, tau_s, scale):
        out = relation_fwd(q, k, v, lam, tau_s=tau_s, scale=scale)
        ctx.save_for_backward(q, k, v, out["o"], lam, out["row_stat"])
        ctx.tau_s, ctx.scale = tau_s, scale
        return out["o"]

    @staticmethod
    def backward(ctx, dout):
        q, k, v, o, lam, row_stat = ctx.saved_tensors
        g = relation_bwd(q, k, v, o, dout, lam, row_stat, tau_s=ctx.tau_s, scale=ctx.scale)
        dlam = g["dlambda"]
        if dlam.shape != lam.shape or dlam.dtype != lam.dtype:
            dlam = dlam.reshape(lam.shape).to(lam.dtype)
        return g["dq"], g["dk"], g["dv"], dlam, None, None


def relation(q, k, v, lam, tau_s: float = TAU_S, scale: Optional[float] = None) -> torch.Tensor:
    """Differentiable causal Full Relation over [B, H, T, D] tensors (fused
    FlashRelation kernels). ``lam`` is a scalar tensor (the layer's lambda)."""
    if not isinstance(lam, torch.Tensor):
        lam = torch.tensor(float(lam), dtype=torch.float32, device=q.device)
    return _RelationFn.apply(q, k, v, lam, tau_s, scale)


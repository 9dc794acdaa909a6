"""Thin Python binding of the LoGo C ABI (``include/logo.h``).

Argument marshalling only: every function here checks dtypes/shapes, allocates
missing outputs and workspaces through torch (device memory is torch's job),
and calls the entry point of the same name in ``_lib/liblogo.so`` on the
current CUDA stream.  All computation runs in the library's CUDA kernels;
there is no CPU path.  If the library has not been built, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import typing

import torch

from . import build as _build

_c_int = ctypes.c_int
_c_float = ctypes.c_float
_c_size = ctypes.c_size_t
_vp = ctypes.c_void_p

LOGO_OK = 0
LOGO_ERR_INVALID_ARG = -1
LOGO_ERR_UNSUPPORTED = -2
LOGO_ERR_CUDA = -3
LOGO_ERR_TIMEOUT = -4
LOGO_ERR_WORKSPACE = -5
LOGO_ERR_SCRATCH_LIMIT = -6
LOGO_SELECT_THRESHOLD = 0
LOGO_SELECT_RATIO = 1

_ERR_NAMES = {
    LOGO_ERR_INVALID_ARG: "LOGO_ERR_INVALID_ARG",
    LOGO_ERR_UNSUPPORTED: "LOGO_ERR_UNSUPPORTED",
    LOGO_ERR_CUDA: "LOGO_ERR_CUDA",
    LOGO_ERR_TIMEOUT: "LOGO_ERR_TIMEOUT",
    LOGO_ERR_WORKSPACE: "LOGO_ERR_WORKSPACE",
    LOGO_ERR_SCRATCH_LIMIT: "LOGO_ERR_SCRATCH_LIMIT",
}


class LogoError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} returned {_ERR_NAMES.get(code, code)}")
        self.code = code


class Dims(ctypes.Structure):
    _fields_ = [("B", _c_int), ("T", _c_int), ("Hq", _c_int), ("Hkv", _c_int), ("D", _c_int)]


class Cache4(typing.NamedTuple):
    """A key-value cache held in 4 bits: codes k, v [B, Hkv, L, D/2] and scales
    k_scale, v_scale [B, Hkv, L, D/16], uint8 (the format is in include/logo.h)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


class _Cache4Ptrs(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp)]


@functools.lru_cache(maxsize=256)
def _dims(*sizes):  # passed by value: one struct for all calls of these sizes
    return Dims(*sizes)


_lib = None
_fns = {}  # name -> its function in the loaded library

_SIGS = {
    "logo_get_device_status": (_c_int, [ctypes.POINTER(_c_int)]),
    "logo_num_sms": (_c_int, []),
    "logo_selftest_wait_expiry": (_c_int, [ctypes.c_uint64, _vp]),
    "logo_select_workspace_size": (_c_size, [Dims]),
    "logo_select": (_c_int, [_vp, Dims, _c_int, _c_float, _c_float, _vp, _vp, _vp, _vp, _vp, _vp, _c_size, _vp]),
    "logo_gate_select": (_c_int, [_vp, _vp, _c_int, Dims, _c_int, _c_float, _c_float, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp, _c_size, _vp]),
    "logo_gate_bwd_workspace_size": (_c_size, [Dims, _c_int]),
    "logo_branch_transform": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _vp]),
    "logo_branch_transform_bwd_workspace_size": (_c_size, [Dims]),
    "logo_branch_transform_bwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _vp, _vp, _vp, Dims, _vp,
                                           _c_size, _vp]),
    "logo_gate_bwd": (_c_int, [_vp, _vp, _vp, _vp, _c_int, Dims, _vp, _c_int, _vp, _vp, _c_size, _vp]),
    "logo_select_noalloc": (_c_int, [_vp, Dims, _c_int, _c_float, _c_float, _vp, _vp, _vp, _vp, _vp, _vp]),
    "logo_select_device_threshold": (_c_int, [_vp, Dims, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_size, _vp]),
    "logo_budget_update": (_c_int, [_vp, Dims, _c_float, _c_float, _vp, _vp, _vp]),
    "logo_pmask_initial_threshold": (_c_float, [_c_float, ctypes.c_longlong]),
    "logo_decode_workspace_size": (_c_size, [Dims]),
    "logo_decode_local_attn": (_c_int, [_vp, _vp, _vp, _vp, _vp, Dims, _c_int, _c_float, _vp, _c_size, _vp]),
    "logo_decode_global_sparse_attn": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_float, _vp, _c_size,
                                                _vp]),
    "logo_decode_prefix_workspace_size": (_c_size, [Dims, _c_int, _c_int, _c_int]),
    "logo_decode_prefix_attn": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_int,
                                         _c_int, _c_float, _vp, _c_size, _vp]),
    "logo_cache_evict_workspace_size": (_c_size, [Dims]),
    "logo_cache_evict": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_int, _c_int, _vp, _c_size,
                                  _vp]),
    "logo_verify_draft_workspace_size": (_c_size, [_c_int, _c_int, _c_int]),
    "logo_verify_draft": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _vp, _c_size,
                                   _vp]),
    "logo_cache4_append": (_c_int, [_Cache4Ptrs, _vp, _vp, _vp, _vp, Dims, _c_int, _vp]),
    "logo_cache4_read": (_c_int, [_Cache4Ptrs, _vp, _vp, _vp, _vp, Dims, _c_int, _vp]),
    "logo_decode_cache4_workspace_size": (_c_size, [Dims, _c_int]),
    "logo_decode_cache4_attn": (_c_int, [_vp, _Cache4Ptrs, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_int, _c_float, _vp,
                                         _c_size, _vp]),
    "logo_target_probs_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "logo_target_probs": (_c_int, [_vp, _c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int,
                                   _c_int, _c_int, _c_int, _vp, _c_size, _vp]),
    "logo_local_attn_fwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, Dims, _c_int, _c_float, _vp]),
    "logo_local_attn_bwd_workspace_size": (_c_size, [Dims]),
    "logo_local_attn_bwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_int, _c_float, _vp,
                                     _c_size, _vp]),
    "logo_global_attn_fwd_workspace_size": (_c_size, [Dims]),
    "logo_global_sparse_attn_fwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims, _c_float, _vp, _c_size,
                                             _vp]),
    "logo_global_attn_bwd_workspace_size": (_c_size, [Dims]),
    "logo_global_sparse_attn_bwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, Dims,
                                             _c_float, _vp, _c_size, _vp]),
    "logo_combine": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_float, _vp, _vp, _vp, Dims, _vp]),
    "logo_combine_bwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_float, _vp, _vp, _vp, Dims, _vp]),
    "logo_combine_bwd_workspace_size": (_c_size, [Dims]),
    "logo_combine_bwd_gains": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_float, _vp, _vp, _vp, _vp, _vp,
                                        Dims, _vp, _c_size, _vp]),
}


def library_path() -> str:
    return _build.LIB


def lib():
    """Load liblogo.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if not os.path.exists(path):
            raise RuntimeError(f"LoGo CUDA library not built ({path}); run python -m paper_2608_29539_gb300.build")
        L = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
            _fns[name] = fn
        _lib = L
    return _lib


def _p(t):
    return None if t is None else _vp(t.data_ptr())


def _stream():
    # the raw handle of torch.cuda.current_stream() (0.1 us; the object costs 3);
    # a call has CUDA tensors, so CUDA has been initialised
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _call(name, *args):
    fn = _fns.get(name)
    rc = fn(*args) if fn is not None else getattr(lib(), name)(*args)
    if rc != LOGO_OK:
        raise LogoError(name, rc)


def _need(t, dtype, name, shape=None):
    try:  # one pass over what has to hold; what does not is named below
        if t.dtype is dtype and t.is_cuda and t.is_contiguous() and (shape is None or t.shape == shape):
            return t
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def dims_of(q: torch.Tensor, k: torch.Tensor) -> Dims:
    B, T, Hq, D = q.shape
    return Dims(B, T, Hq, k.shape[2], D)


def _given_workspace(ws):
    if not ws.is_cuda or not ws.is_contiguous():  # the library takes an address and a size
        raise ValueError("workspace must be a contiguous CUDA tensor")
    return ws


def _workspace(nbytes: int, device, ws=None):
    if ws is not None:
        _given_workspace(ws)
        if ws.numel() * ws.element_size() < nbytes:
            raise ValueError("workspace too small")
        return ws
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def workspace_bytes(kind: str, dims: Dims) -> int:
    fn = {"select": "logo_select_workspace_size", "local_bwd": "logo_local_attn_bwd_workspace_size",
          "global_fwd": "logo_global_attn_fwd_workspace_size",
          "global_bwd": "logo_global_attn_bwd_workspace_size",
          "combine_bwd_gains": "logo_combine_bwd_workspace_size"}[kind]
    return int(getattr(lib(), fn)(dims))


# ----------------------------------------------------------------------- API
def logo_get_device_status() -> int:
    st = _c_int(0)
    _call("logo_get_device_status", ctypes.byref(st))
    return st.value


def logo_num_sms() -> int:
    return int(lib().logo_num_sms())


def logo_selftest_wait_expiry(budget_ns: int) -> None:
    """Launch one warp whose bounded mbarrier wait can never complete; after
    budget_ns it records LOGO_ERR_TIMEOUT (read it with logo_get_device_status)."""
    torch.cuda.init()  # (no tensor has done so)
    _call("logo_selftest_wait_expiry", int(budget_ns), _stream())


def logo_select(gate_p, mode: int, b_th: float = 0.5, ratio: float = 0.0, z=None, pos=None, cu_q=None,
                row_of=None, n_sel_total=None, workspace=None):
    """Eq. 7 routing and packing of I.  Returns (z, pos, cu_q, row_of, n_sel_total)."""
    _need(gate_p, torch.float32, "gate_p")
    B, T = gate_p.shape
    dev = gate_p.device
    dims = Dims(B, T, 1, 1, 64)
    z = z if z is not None else torch.empty((B, T), dtype=torch.uint8, device=dev)
    pos = pos if pos is not None else torch.empty((B * T,), dtype=torch.int32, device=dev)
    cu_q = cu_q if cu_q is not None else torch.empty((B + 1,), dtype=torch.int32, device=dev)
    row_of = row_of if row_of is not None else torch.empty((B, T), dtype=torch.int32, device=dev)
    n_sel_total = n_sel_total if n_sel_total is not None else torch.empty((1,), dtype=torch.int32, device=dev)
    nbytes = workspace_bytes("select", dims)
    ws = _workspace(nbytes, dev, workspace)
    _call("logo_select", _p(gate_p), dims, int(mode), float(b_th), float(ratio), _p(z), _p(pos), _p(cu_q),
          _p(row_of), _p(n_sel_total), _p(ws), nbytes, _stream())
    return z, pos, cu_q, row_of, n_sel_total


def logo_gate_select(x, w_g, mode: int, b_th: float = 0.5, ratio: float = 0.0, gate_p=None, z=None, pos=None,
                     cu_q=None, row_of=None, n_sel_total=None, workspace=None):
    """Eq. 7 gate p = sigmoid(x . w_g) (x [B, T, d_model] bf16, w_g [d_model]
    float32) followed by the routing of logo_select.  Returns
    (gate_p, z, pos, cu_q, row_of, n_sel_total)."""
    _need(x, torch.bfloat16, "x")
    _need(w_g, torch.float32, "w_g")
    B, T, dm = x.shape
    dev = x.device
    dims = Dims(B, T, 1, 1, 64)
    gate_p = gate_p if gate_p is not None else torch.empty((B, T), dtype=torch.float32, device=dev)
    z = z if z is not None else torch.empty((B, T), dtype=torch.uint8, device=dev)
    pos = pos if pos is not None else torch.empty((B * T,), dtype=torch.int32, device=dev)
    cu_q = cu_q if cu_q is not None else torch.empty((B + 1,), dtype=torch.int32, device=dev)
    row_of = row_of if row_of is not None else torch.empty((B, T), dtype=torch.int32, device=dev)
    n_sel_total = n_sel_total if n_sel_total is not None else torch.empty((1,), dtype=torch.int32, device=dev)
    nbytes = workspace_bytes("select", dims)
    ws = _workspace(nbytes, dev, workspace)
    _call("logo_gate_select", _p(x), _p(w_g), int(dm), dims, int(mode), float(b_th), float(ratio), _p(gate_p), _p(z),
          _p(pos), _p(cu_q), _p(row_of), _p(n_sel_total), _p(ws), nbytes, _stream())
    return gate_p, z, pos, cu_q, row_of, n_sel_total


def logo_gate_bwd(x, w_g, gate_p, dgate_p, dx=None, accumulate: bool = False, dw_g=None, want_dx: bool = True,
                  want_dw: bool = True, workspace=None):
    """Backward of the gate: dx = dlogit w_g (written, or added to dx when
    accumulate), dw_g = sum_t dlogit_t x_t with dlogit = dp p (1 - p).
    Returns (dx, dw_g) (None for a part not asked for)."""
    _need(x, torch.bfloat16, "x")
    B, T, dm = x.shape
    dev = x.device
    dims = Dims(B, T, 1, 1, 64)
    if want_dx and dx is None:
        if accumulate:
            raise ValueError("accumulate needs the dx to add to")
        dx = torch.empty_like(x)
    if not want_dx:
        dx = None
    dw_g = (dw_g if dw_g is not None else torch.empty((dm,), dtype=torch.float32, device=dev)) if want_dw else None
    nbytes = int(lib().logo_gate_bwd_workspace_size(dims, dm)) if want_dw else 0
    ws = _workspace(nbytes, dev, workspace) if want_dw else None
    _call("logo_gate_bwd", _p(x), _p(w_g), _p(gate_p), _p(dgate_p), int(dm), dims, _p(dx), int(bool(accumulate)),
          _p(dw_g), _p(ws), nbytes, _stream())
    return dx, dw_g


def _transform_rows(rows):
    if rows is None:
        return None, None, None
    pos, cu_q, n_sel_total = rows
    return pos, cu_q, n_sel_total


def logo_branch_transform(u_l, a=None, s=None, b=None, rows=None, u_g=None):
    """Eq. 5: U^G = U^L A (LP, a [H, D, D] bf16) or U^L * s + b (SO, s and b
    [H, D] float32), on every row, or on the packed selected rows when rows =
    (pos, cu_q, n_sel_total).  u_l [B, T, H, D] bf16.  Returns u_g."""
    _need(u_l, torch.bfloat16, "u_l")
    B, T, H, D = u_l.shape
    u_g = u_g if u_g is not None else torch.empty_like(u_l)
    pos, cu_q, n_sel = _transform_rows(rows)
    _call("logo_branch_transform", _p(u_l), _p(a), _p(s), _p(b), _p(pos), _p(cu_q), _p(n_sel), _p(u_g),
          Dims(B, T, H, H, D), _stream())
    return u_g


def logo_branch_transform_bwd(u_l, du_g, a=None, s=None, rows=None, du_l=None, accumulate: bool = False,
                              workspace=None):
    """Gradients of logo_branch_transform.  Returns (du_l, da) for LP and
    (du_l, ds, db) for SO."""
    _need(u_l, torch.bfloat16, "u_l")
    B, T, H, D = u_l.shape
    dev = u_l.device
    dims = Dims(B, T, H, H, D)
    if du_l is None:
        if accumulate:
            raise ValueError("accumulate needs the du_l to add to")
        du_l = torch.empty_like(u_l)
    da = torch.empty((H, D, D), dtype=torch.float32, device=dev) if a is not None else None
    ds = torch.empty((H, D), dtype=torch.float32, device=dev) if a is None else None
    db = torch.empty((H, D), dtype=torch.float32, device=dev) if a is None else None
    nbytes = int(lib().logo_branch_transform_bwd_workspace_size(dims))
    ws = _workspace(nbytes, dev, workspace)
    pos, cu_q, n_sel = _transform_rows(rows)
    _call("logo_branch_transform_bwd", _p(u_l), _p(a), _p(s), _p(pos), _p(cu_q), _p(n_sel), _p(du_g), _p(du_l),
          int(bool(accumulate)), _p(da), _p(ds), _p(db), dims, _p(ws), nbytes, _stream())
    return (du_l, da) if a is not None else (du_l, ds, db)


def logo_select_device_threshold(gate_p, b_th, z=None, pos=None, cu_q=None, row_of=None, n_sel_total=None,
                                 workspace=None):
    """Eq. 7 routing with the threshold read on the device from b_th (a
    one-element float32 CUDA tensor).  Returns (z, pos, cu_q, row_of, n_sel_total)."""
    _need(gate_p, torch.float32, "gate_p")
    _need(b_th, torch.float32, "b_th", (1,))
    B, T = gate_p.shape
    dev = gate_p.device
    dims = Dims(B, T, 1, 1, 64)
    z = z if z is not None else torch.empty((B, T), dtype=torch.uint8, device=dev)
    pos = pos if pos is not None else torch.empty((B * T,), dtype=torch.int32, device=dev)
    cu_q = cu_q if cu_q is not None else torch.empty((B + 1,), dtype=torch.int32, device=dev)
    row_of = row_of if row_of is not None else torch.empty((B, T), dtype=torch.int32, device=dev)
    n_sel_total = n_sel_total if n_sel_total is not None else torch.empty((1,), dtype=torch.int32, device=dev)
    nbytes = workspace_bytes("select", dims)
    ws = _workspace(nbytes, dev, workspace)
    _call("logo_select_device_threshold", _p(gate_p), dims, _p(b_th), _p(z), _p(pos), _p(cu_q), _p(row_of),
          _p(n_sel_total), _p(ws), nbytes, _stream())
    return z, pos, cu_q, row_of, n_sel_total


def logo_budget_update(n_sel_total, B: int, T: int, rho: float, gamma: float, b_th, f_out=None):
    """Eq. 3 + Eq. 11 on the device: b_th (one-element float32 CUDA tensor) is
    moved by gamma * sign(N / (B*T) - rho) in place; f_out (optional, same
    kind) receives F.  Returns b_th."""
    _need(n_sel_total, torch.int32, "n_sel_total", (1,))
    _need(b_th, torch.float32, "b_th", (1,))
    if f_out is not None:
        _need(f_out, torch.float32, "f_out", (1,))
    _call("logo_budget_update", _p(n_sel_total), Dims(int(B), int(T), 1, 1, 64), float(rho), float(gamma),
          _p(b_th), _p(f_out), _stream())
    return b_th


def logo_pmask_initial_threshold(gamma: float, pmask_steps: int) -> float:
    """P-mask start value 0.5 - gamma * steps (Sec. 3.2, App. C.1); host only."""
    return float(lib().logo_pmask_initial_threshold(float(gamma), int(pmask_steps)))


def _decode_dims(q, k):
    B, Hq, D = q.shape
    return Dims(B, k.shape[1], Hq, k.shape[2], D)


def logo_decode_local_attn(q, k_ring, v_ring, seq_len, window: int, scale: float = 0.0, o=None, workspace=None):
    """One decoding step of the local branch (Eq. 6) from ring caches
    [B, R, Hkv, D] (position s in slot s mod R).  q [B, Hq, D]; seq_len [B]
    int32 (cache length, the new token included).  Returns o [B, Hq, D]."""
    _need(q, torch.bfloat16, "q")
    _need(k_ring, torch.bfloat16, "k_ring")
    _need(v_ring, torch.bfloat16, "v_ring", k_ring.shape)
    _need(seq_len, torch.int32, "seq_len", (q.shape[0],))
    dims = _decode_dims(q, k_ring)
    o = o if o is not None else torch.empty_like(q)
    nbytes = int(lib().logo_decode_workspace_size(dims))
    ws = _workspace(nbytes, q.device, workspace)
    _call("logo_decode_local_attn", _p(q), _p(k_ring), _p(v_ring), _p(seq_len), _p(o), dims, int(window),
          float(scale), _p(ws), nbytes, _stream())
    return o


def logo_decode_global_sparse_attn(q, k_cache, v_cache, seq_len, cu_q, n_sel_total, scale: float = 0.0, o_c=None,
                                   workspace=None):
    """One decoding step of the global branch (Eq. 8) for the selected
    sequences only (packed rows of a (B, 1) selection), from dense caches
    [B, L, Hkv, D].  Returns o_c [B, Hq, D] (packed rows; rows >= n_sel untouched)."""
    _need(q, torch.bfloat16, "q")
    _need(k_cache, torch.bfloat16, "k_cache")
    _need(v_cache, torch.bfloat16, "v_cache", k_cache.shape)
    _need(seq_len, torch.int32, "seq_len", (q.shape[0],))
    _need(cu_q, torch.int32, "cu_q", (q.shape[0] + 1,))
    _need(n_sel_total, torch.int32, "n_sel_total", (1,))
    dims = _decode_dims(q, k_cache)
    o_c = o_c if o_c is not None else torch.empty_like(q)
    nbytes = int(lib().logo_decode_workspace_size(dims))
    ws = _workspace(nbytes, q.device, workspace)
    _call("logo_decode_global_sparse_attn", _p(q), _p(k_cache), _p(v_cache), _p(seq_len), _p(cu_q),
          _p(n_sel_total), _p(o_c), dims, float(scale), _p(ws), nbytes, _stream())
    return o_c


def logo_decode_prefix_workspace(q, k_prefix, k_cache, with_mass: bool = False):
    """A workspace for logo_decode_prefix_attn calls of these shapes (one per
    call in flight)."""
    B, n_new, Hq, D = q.shape
    dims = Dims(B, k_cache.shape[1], Hq, k_cache.shape[2], D)
    P = 0 if k_prefix is None else k_prefix.shape[0]
    return _workspace(int(lib().logo_decode_prefix_workspace_size(dims, n_new, P, int(bool(with_mass)))), q.device)


def logo_decode_prefix_attn(q, k_prefix, v_prefix, k_cache, v_cache, seq_len, pos, cu_q, n_sel_total,
                            scale: float = 0.0, mass_in=None, mass_out=None, o_c=None, lse_c=None, workspace=None):
    """One serving step of the global branch (Eq. 8) over a prefix that all
    sequences share and each sequence's own cache.

    q [B, n_new, Hq, D]; k_prefix / v_prefix [P, Hkv, D] (None: no prefix);
    k_cache / v_cache [B, L, Hkv, D]; seq_len [B] int32 (own tokens, the n_new
    new ones included and last); pos, cu_q, n_sel_total from logo_select on
    (B, n_new) gates.  With mass_in [B, Hkv, L] float32 the attention weight
    each own cache row receives is added into mass_out (None: mass_in itself).
    Returns (o_c [B*n_new, Hq, D], lse_c [Hq, B*n_new], mass_out or None);
    packed rows >= n_sel_total are untouched."""
    _need(q, torch.bfloat16, "q")
    if q.dim() != 4:
        raise ValueError("q must be [B, n_new, Hq, D]")
    B, n_new, Hq, D = q.shape
    _need(k_cache, torch.bfloat16, "k_cache")
    if k_cache.dim() != 4 or k_cache.shape[0] != B or k_cache.shape[3] != D:
        raise ValueError(f"k_cache has shape {tuple(k_cache.shape)}, expected ({B}, L, Hkv, {D})")
    _, Lc, Hkv, _ = k_cache.shape
    _need(v_cache, torch.bfloat16, "v_cache", k_cache.shape)
    if (k_prefix is None) != (v_prefix is None):
        raise ValueError("k_prefix and v_prefix come together")
    P = 0
    if k_prefix is not None:
        P = k_prefix.shape[0]
        _need(k_prefix, torch.bfloat16, "k_prefix", (P, Hkv, D))
        _need(v_prefix, torch.bfloat16, "v_prefix", (P, Hkv, D))
    cap = B * n_new
    _need(seq_len, torch.int32, "seq_len", (B,))
    _need(pos, torch.int32, "pos", (cap,))
    _need(cu_q, torch.int32, "cu_q", (B + 1,))
    _need(n_sel_total, torch.int32, "n_sel_total", (1,))
    if mass_in is None:
        if mass_out is not None:
            raise ValueError("mass_out needs mass_in")
    else:
        _need(mass_in, torch.float32, "mass_in", (B, Hkv, Lc))
        if mass_out is None:
            mass_out = mass_in
        else:
            _need(mass_out, torch.float32, "mass_out", (B, Hkv, Lc))
    if o_c is None:
        o_c = torch.empty((cap, Hq, D), dtype=torch.bfloat16, device=q.device)
    else:
        _need(o_c, torch.bfloat16, "o_c", (cap, Hq, D))
    if lse_c is None:
        lse_c = torch.empty((Hq, cap), dtype=torch.float32, device=q.device)
    else:
        _need(lse_c, torch.float32, "lse_c", (Hq, cap))
    dims = _dims(B, Lc, Hq, Hkv, D)
    if workspace is None:
        workspace = logo_decode_prefix_workspace(q, k_prefix, k_cache, mass_in is not None)
    else:
        _given_workspace(workspace)
    _call("logo_decode_prefix_attn", q.data_ptr(), k_prefix.data_ptr() if P else None,
          v_prefix.data_ptr() if P else None, k_cache.data_ptr(), v_cache.data_ptr(), seq_len.data_ptr(),
          pos.data_ptr(), cu_q.data_ptr(), n_sel_total.data_ptr(), o_c.data_ptr(), lse_c.data_ptr(),
          None if mass_in is None else mass_in.data_ptr(), None if mass_out is None else mass_out.data_ptr(), dims,
          n_new, P, float(scale), workspace.data_ptr(), workspace.nbytes, _stream())
    return o_c, lse_c, mass_out


def logo_cache_evict_workspace(k_cache):
    """A workspace for logo_cache_evict calls on caches of this shape."""
    B, Lc, Hkv, D = k_cache.shape
    return _workspace(int(lib().logo_cache_evict_workspace_size(Dims(B, Lc, Hkv, Hkv, D))), k_cache.device)


def logo_cache_evict(k_cache, v_cache, mass, slot_pos, seq_len, n_seen, budget: int, recent: int, mass_out=None,
                     slot_pos_out=None, new_len=None, workspace=None):
    """Cut every (sequence, KV head) back to `budget` cache rows: those whose
    slot_pos >= n_seen - recent, then the largest mass, ties to the lower row.

    k_cache / v_cache [B, L, Hkv, D] bf16 change in place (rows that stay move
    into the places of rows that go; the order is not kept); mass [B, Hkv, L]
    float32 and slot_pos [B, Hkv, L] int32 (token position of each row) go
    along, into mass_out / slot_pos_out (None: in place); seq_len, n_seen [B]
    int32.  Returns (mass_out, slot_pos_out, new_len [B] int32)."""
    _need(k_cache, torch.bfloat16, "k_cache")
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [B, L, Hkv, D]")
    B, Lc, Hkv, D = k_cache.shape
    _need(v_cache, torch.bfloat16, "v_cache", k_cache.shape)
    _need(mass, torch.float32, "mass", (B, Hkv, Lc))
    _need(slot_pos, torch.int32, "slot_pos", (B, Hkv, Lc))
    _need(seq_len, torch.int32, "seq_len", (B,))
    _need(n_seen, torch.int32, "n_seen", (B,))
    mass_out = mass if mass_out is None else _need(mass_out, torch.float32, "mass_out", (B, Hkv, Lc))
    slot_pos_out = (slot_pos if slot_pos_out is None
                    else _need(slot_pos_out, torch.int32, "slot_pos_out", (B, Hkv, Lc)))
    if new_len is None:
        new_len = torch.empty((B,), dtype=torch.int32, device=k_cache.device)
    else:
        _need(new_len, torch.int32, "new_len", (B,))
    if workspace is None:
        workspace = logo_cache_evict_workspace(k_cache)
    else:
        _given_workspace(workspace)
    _call("logo_cache_evict", k_cache.data_ptr(), v_cache.data_ptr(), mass.data_ptr(), slot_pos.data_ptr(),
          seq_len.data_ptr(), n_seen.data_ptr(), mass_out.data_ptr(), slot_pos_out.data_ptr(), new_len.data_ptr(),
          _dims(B, Lc, Hkv, Hkv, D), int(budget), int(recent), workspace.data_ptr(), workspace.nbytes, _stream())
    return mass_out, slot_pos_out, new_len


def logo_verify_draft_workspace(p_target):
    """A workspace for logo_verify_draft calls on probabilities of this shape."""
    B, m1, V = p_target.shape
    return _workspace(int(lib().logo_verify_draft_workspace_size(B, m1 - 1, V)), p_target.device)


def logo_verify_draft(draft, q_draft, p_target, u, noise, draft_len=None, tokens=None, n_accept=None, workspace=None):
    """Speculative sampling: accept the drafts draft [B, m] int32 (drawn from
    q_draft [B, m, V] float32) against p_target [B, m+1, V] float32 with the
    uniforms u [B, m], and draw the next token with the exponentials noise
    [B, V].  draft_len [B] int32: drafts of each sequence (None: m).  Returns
    (tokens [B, m+1] int32: accepted drafts, the drawn token, -1 ...;
    n_accept [B] int32)."""
    _need(p_target, torch.float32, "p_target")
    if p_target.dim() != 3 or p_target.shape[1] < 1:
        raise ValueError("p_target must be [B, m + 1, V]")
    B, m1, V = p_target.shape
    m = m1 - 1
    _need(draft, torch.int32, "draft", (B, m))
    _need(q_draft, torch.float32, "q_draft", (B, m, V))
    _need(u, torch.float32, "u", (B, m))
    _need(noise, torch.float32, "noise", (B, V))
    if draft_len is not None:
        _need(draft_len, torch.int32, "draft_len", (B,))
    if tokens is None:
        tokens = torch.empty((B, m1), dtype=torch.int32, device=p_target.device)
    else:
        _need(tokens, torch.int32, "tokens", (B, m1))
    if n_accept is None:
        n_accept = torch.empty((B,), dtype=torch.int32, device=p_target.device)
    else:
        _need(n_accept, torch.int32, "n_accept", (B,))
    if workspace is None:
        workspace = logo_verify_draft_workspace(p_target)
    else:
        _given_workspace(workspace)
    _call("logo_verify_draft", draft.data_ptr() if m else None, q_draft.data_ptr() if m else None,
          p_target.data_ptr(), u.data_ptr() if m else None, noise.data_ptr(),
          None if draft_len is None else draft_len.data_ptr(), tokens.data_ptr(), n_accept.data_ptr(), B, m, V,
          workspace.data_ptr(), workspace.nbytes, _stream())
    return tokens, n_accept


def logo_cache4_empty(B: int, L: int, Hkv: int, D: int, device="cuda") -> Cache4:
    """A 4-bit cache of L rows a sequence; the rows hold nothing yet."""
    e = lambda w: torch.zeros((B, Hkv, L, w), dtype=torch.uint8, device=device)  # noqa: E731
    return Cache4(e(D // 2), e(D // 2), e(D // 16), e(D // 16))


def _on(t, dev, dtype, name, shape):
    """_need, and on device number dev."""
    try:  # one pass over what has to hold; what does not is named below
        if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and t.shape == shape:
            return
    except AttributeError:
        pass
    _need(t, dtype, name, shape)
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{dev} as the others")


def _here(dev):
    """The current stream of device number dev, on which the tensors are.  The kernels run
    on the current device: tensors on another are refused."""
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on cuda:{dev}, the current device is cuda:{torch._C._cuda_getDevice()}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _cache4(cache):
    """(its addresses, B, Hkv, L, D, device number) of a Cache4."""
    k, v, ks, vs = cache
    _need(k, torch.uint8, "cache.k")
    shape = k.shape
    if len(shape) != 4:
        raise ValueError("cache.k must be [B, Hkv, L, D/2]")
    B, Hkv, L, half = shape
    dev = k.get_device()
    _on(v, dev, torch.uint8, "cache.v", shape)
    shape = (B, Hkv, L, half // 8)
    _on(ks, dev, torch.uint8, "cache.k_scale", shape)
    _on(vs, dev, torch.uint8, "cache.v_scale", shape)
    return _Cache4Ptrs(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr()), B, Hkv, L, 2 * half, dev


def logo_cache4_append(cache: Cache4, k_new, v_new, seq_len, n_valid=None):
    """Quantise new tokens' k_new, v_new [B, n_new, Hkv, D] bf16 into the 4-bit
    cache.  seq_len [B] int32 counts each sequence's tokens, the new ones included;
    of those the first n_valid [B] int32 of the n_new are new ones (None: all), and
    go to the rows that end at seq_len.  Returns the cache."""
    ptrs, B, Hkv, L, D, dev = _cache4(cache)
    shape = (B, k_new.shape[1] if k_new.dim() == 4 else 0, Hkv, D)
    _on(k_new, dev, torch.bfloat16, "k_new", shape)
    _on(v_new, dev, torch.bfloat16, "v_new", shape)
    _on(seq_len, dev, torch.int32, "seq_len", (B,))
    if n_valid is not None:
        _on(n_valid, dev, torch.int32, "n_valid", (B,))
    stream = _here(dev)
    _call("logo_cache4_append", ptrs, k_new.data_ptr(), v_new.data_ptr(), seq_len.data_ptr(),
          None if n_valid is None else n_valid.data_ptr(), _dims(B, L, Hkv, Hkv, D), shape[1], stream)
    return cache


def logo_cache4_read(cache: Cache4, seq_len, rows=None, m=None, k=None, v=None):
    """Rows of a 4-bit cache as the bf16 values that they hold: the listed rows
    [B, m] int32, or rows 0 .. m-1 (m None: as k has, or all L).  Rows outside
    [0, seq_len) read as zeros.  Returns (k, v) [B, m, Hkv, D]."""
    ptrs, B, Hkv, L, D, dev = _cache4(cache)
    _on(seq_len, dev, torch.int32, "seq_len", (B,))
    if rows is not None:
        if rows.dim() != 2 or (m is not None and m != rows.shape[1]):
            raise ValueError("rows must be [B, m]")
        m = rows.shape[1]
        _on(rows, dev, torch.int32, "rows", (B, m))
    elif m is None:
        m = L if k is None else k.shape[1]
    shape = (B, m, Hkv, D)
    stream = _here(dev)
    k = torch.empty(shape, dtype=torch.bfloat16, device=seq_len.device) if k is None else k
    v = torch.empty(shape, dtype=torch.bfloat16, device=seq_len.device) if v is None else v
    _on(k, dev, torch.bfloat16, "k", shape)
    _on(v, dev, torch.bfloat16, "v", shape)
    _call("logo_cache4_read", ptrs, seq_len.data_ptr(), None if rows is None else rows.data_ptr(), k.data_ptr(),
          v.data_ptr(), _dims(B, L, Hkv, Hkv, D), m, stream)
    return k, v


def logo_decode_cache4_workspace(q, cache: Cache4):
    """A workspace for logo_decode_cache4_attn calls of these shapes (one per call
    in flight)."""
    B, n_new, Hq, D = q.shape
    dims = Dims(B, cache.k.shape[2], Hq, cache.k.shape[1], D)
    return _workspace(int(lib().logo_decode_cache4_workspace_size(dims, n_new)), q.device)


def logo_decode_cache4_attn(q, cache: Cache4, seq_len, pos, cu_q, n_sel_total, scale: float = 0.0, o_c=None,
                            lse_c=None, workspace=None):
    """One serving step of the global branch (Eq. 8) over 4-bit caches.

    q [B, n_new, Hq, D] bf16; seq_len [B] int32 (tokens of each cache, the n_new new
    ones included and last); pos, cu_q, n_sel_total from logo_select on (B, n_new)
    gates.  Returns (o_c [B*n_new, Hq, D], lse_c [Hq, B*n_new]); packed rows >=
    n_sel_total are untouched."""
    ptrs, B, Hkv, L, D, dev = _cache4(cache)
    if not isinstance(q, torch.Tensor) or q.dim() != 4 or q.shape[0] != B or q.shape[3] != D:
        raise ValueError(f"q has to be a tensor of shape ({B}, n_new, Hq, {D})")
    shape = q.shape
    _, n_new, Hq, _ = shape
    cap = B * n_new
    _on(q, dev, torch.bfloat16, "q", shape)
    _on(seq_len, dev, torch.int32, "seq_len", (B,))
    _on(pos, dev, torch.int32, "pos", (cap,))
    _on(cu_q, dev, torch.int32, "cu_q", (B + 1,))
    _on(n_sel_total, dev, torch.int32, "n_sel_total", (1,))
    stream = _here(dev)
    if o_c is None:
        o_c = torch.empty((cap, Hq, D), dtype=torch.bfloat16, device=q.device)
    else:
        _on(o_c, dev, torch.bfloat16, "o_c", (cap, Hq, D))
    if lse_c is None:
        lse_c = torch.empty((Hq, cap), dtype=torch.float32, device=q.device)
    else:
        _on(lse_c, dev, torch.float32, "lse_c", (Hq, cap))
    if workspace is None:
        workspace = logo_decode_cache4_workspace(q, cache)
    elif _given_workspace(workspace).get_device() != dev:
        raise ValueError(f"workspace is on {workspace.device}, not on cuda:{dev} as the others")
    _call("logo_decode_cache4_attn", q.data_ptr(), ptrs, seq_len.data_ptr(), pos.data_ptr(), cu_q.data_ptr(),
          n_sel_total.data_ptr(), o_c.data_ptr(), lse_c.data_ptr(), _dims(B, L, Hq, Hkv, D), n_new, float(scale),
          workspace.data_ptr(), workspace.nbytes, stream)
    return o_c, lse_c


@functools.lru_cache(maxsize=256)
def _target_probs_bytes(*sizes):
    return int(lib().logo_target_probs_workspace_size(*sizes))


def logo_target_probs_workspace(logits, H: int = 0, K: int = 0):
    """A workspace for logo_target_probs calls on logits of this shape with histories
    [B, H] and biases [B, K] (one per call in flight)."""
    B, m1, V = logits.shape
    return _workspace(_target_probs_bytes(B, m1, V, H, K), logits.device)


def logo_target_probs(logits, temperature=None, penalty=None, history=None, hist_len=None, n_prompt=None, draft=None,
                      bias_tok=None, bias_val=None, allowed=None, p=None, workspace=None):
    """The target's probabilities [B, m1, V] float32, as logo_verify_draft takes
    them, from logits [B, m1, V] (float32 or bf16).

    penalty [B, 3] float32: repetition (over the history and the drafts before the
    row), frequency and presence (over the generated ones of these); history [B, H]
    int32 with hist_len [B] int32 tokens of which the first n_prompt [B] int32 are the
    prompt's; draft [B, m1 - 1] int32.  bias_tok [B, K] int32 with bias_val [B, K]
    float32: added to the listed tokens.  allowed [B, m1, ceil(V / 32)] int32: a bit
    per token.  temperature [B] float32, 0 for greedy.  Token numbers outside [0, V)
    count for nothing.  p may be float32 logits themselves."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be a float32 or bf16 CUDA tensor")
    _need(logits, logits.dtype, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must be [B, m1, V]")
    B, m1, V = logits.shape
    dev = logits.get_device()
    i32, f32 = torch.int32, torch.float32
    H = K = 0
    a_T = a_pen = a_hist = a_len = a_prompt = a_draft = a_tok = a_val = a_ok = None
    if temperature is not None:
        _on(temperature, dev, f32, "temperature", (B,))
        a_T = temperature.data_ptr()
    if penalty is not None:
        _on(penalty, dev, f32, "penalty", (B, 3))
        a_pen = penalty.data_ptr()
    elif history is not None or draft is not None:
        raise ValueError("history and draft need penalty")
    if history is not None:
        if history.dim() != 2:
            raise ValueError("history must be [B, H]")
        H = history.shape[1]
        _on(history, dev, i32, "history", (B, H))
        if hist_len is None:
            raise ValueError("history needs hist_len")
        _on(hist_len, dev, i32, "hist_len", (B,))
        if n_prompt is not None:
            _on(n_prompt, dev, i32, "n_prompt", (B,))
        if H:  # (an empty list is no list)
            a_hist, a_len, a_prompt = history.data_ptr(), hist_len.data_ptr(), _p(n_prompt)
    elif hist_len is not None or n_prompt is not None:
        raise ValueError("hist_len and n_prompt need history")
    if draft is not None:
        _on(draft, dev, i32, "draft", (B, m1 - 1))
        if m1 > 1:
            a_draft = draft.data_ptr()
    if (bias_tok is None) != (bias_val is None):
        raise ValueError("bias_tok and bias_val come together")
    if bias_tok is not None:
        if bias_tok.dim() != 2:
            raise ValueError("bias_tok must be [B, K]")
        K = bias_tok.shape[1]
        _on(bias_tok, dev, i32, "bias_tok", (B, K))
        _on(bias_val, dev, f32, "bias_val", (B, K))
        if K:
            a_tok, a_val = bias_tok.data_ptr(), bias_val.data_ptr()
    if allowed is not None:
        _on(allowed, dev, i32, "allowed", (B, m1, (V + 31) // 32))
        a_ok = allowed.data_ptr()
    stream = _here(dev)
    if p is None:
        p = torch.empty((B, m1, V), dtype=f32, device=logits.device)
    else:
        _on(p, dev, f32, "p", (B, m1, V))
    if workspace is None:
        workspace = logo_target_probs_workspace(logits, H, K)
    elif _given_workspace(workspace).get_device() != dev:
        raise ValueError(f"workspace is on {workspace.device}, not on cuda:{dev} as the others")
    _call("logo_target_probs", logits.data_ptr(), int(logits.dtype is torch.bfloat16), a_T, a_pen, a_hist, a_len, a_prompt,
          a_draft, a_tok, a_val, a_ok, p.data_ptr(), B, m1, V, H, K, workspace.data_ptr(), workspace.nbytes, stream)
    return p


def logo_select_noalloc(gate_p, mode: int, b_th: float = 0.5, ratio: float = 0.0, z=None, pos=None, cu_q=None,
                        row_of=None, n_sel_total=None):
    """logo_select without a workspace, for callers that cannot allocate
    scratch (its scratch is a static device array inside the library; see
    include/logo.h for the size limits).  The outputs must be given or are
    allocated here by torch.  Returns (z, pos, cu_q, row_of, n_sel_total)."""
    _need(gate_p, torch.float32, "gate_p")
    B, T = gate_p.shape
    dev = gate_p.device
    dims = Dims(B, T, 1, 1, 64)
    z = z if z is not None else torch.empty((B, T), dtype=torch.uint8, device=dev)
    pos = pos if pos is not None else torch.empty((B * T,), dtype=torch.int32, device=dev)
    cu_q = cu_q if cu_q is not None else torch.empty((B + 1,), dtype=torch.int32, device=dev)
    row_of = row_of if row_of is not None else torch.empty((B, T), dtype=torch.int32, device=dev)
    n_sel_total = n_sel_total if n_sel_total is not None else torch.empty((1,), dtype=torch.int32, device=dev)
    _call("logo_select_noalloc", _p(gate_p), dims, int(mode), float(b_th), float(ratio), _p(z), _p(pos), _p(cu_q),
          _p(row_of), _p(n_sel_total), _stream())
    return z, pos, cu_q, row_of, n_sel_total


def logo_local_attn_fwd(q, k, v, window: int, scale: float = 0.0, o=None, lse=None):
    """Eq. 6 local branch.  Returns (o [B,T,Hq,D] bf16, lse [B,Hq,T] fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, n)
    d = dims_of(q, k)
    o = o if o is not None else torch.empty_like(q)
    lse = lse if lse is not None else torch.empty((d.B, d.Hq, d.T), dtype=torch.float32, device=q.device)
    _call("logo_local_attn_fwd", _p(q), _p(k), _p(v), _p(o), _p(lse), d, int(window), float(scale), _stream())
    return o, lse


def logo_local_attn_bwd(q, k, v, o, lse, dO, window: int, scale: float = 0.0, dq=None, dk=None, dv=None,
                        workspace=None):
    """Gradients of the local branch.  Returns (dq, dk, dv)."""
    d = dims_of(q, k)
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dO, "dO")):
        _need(t, torch.bfloat16, n)
    _need(lse, torch.float32, "lse", (d.B, d.Hq, d.T))
    dq = dq if dq is not None else torch.empty_like(q)
    dk = dk if dk is not None else torch.empty_like(k)
    dv = dv if dv is not None else torch.empty_like(v)
    nbytes = workspace_bytes("local_bwd", d)
    ws = _workspace(nbytes, q.device, workspace)
    _call("logo_local_attn_bwd", _p(q), _p(k), _p(v), _p(o), _p(lse), _p(dO), _p(dq), _p(dk), _p(dv), d,
          int(window), float(scale), _p(ws), nbytes, _stream())
    return dq, dk, dv


def logo_global_sparse_attn_fwd(q, k, v, pos, cu_q, n_sel_total, scale: float = 0.0, o_c=None, lse_c=None,
                                workspace=None):
    """Eq. 8 query-sparse global branch.  Returns (o_c [B*T,Hq,D], lse_c [Hq,B*T])."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.bfloat16, n)
    for t, n in ((pos, "pos"), (cu_q, "cu_q"), (n_sel_total, "n_sel_total")):
        _need(t, torch.int32, n)
    d = dims_of(q, k)
    cap = d.B * d.T
    o_c = o_c if o_c is not None else torch.empty((cap, d.Hq, d.D), dtype=torch.bfloat16, device=q.device)
    lse_c = lse_c if lse_c is not None else torch.empty((d.Hq, cap), dtype=torch.float32, device=q.device)
    nbytes = workspace_bytes("global_fwd", d)
    ws = _workspace(nbytes, q.device, workspace)
    _call("logo_global_sparse_attn_fwd", _p(q), _p(k), _p(v), _p(pos), _p(cu_q), _p(n_sel_total), _p(o_c),
          _p(lse_c), d, float(scale), _p(ws), nbytes, _stream())
    return o_c, lse_c


def logo_global_sparse_attn_bwd(q, k, v, pos, cu_q, n_sel_total, o_c, lse_c, dO_c, scale: float = 0.0, dq=None,
                                dk=None, dv=None, workspace=None):
    """Row-sparse gradients of the global branch.  Returns (dq dense, dk, dv)."""
    d = dims_of(q, k)
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o_c, "o_c"), (dO_c, "dO_c")):
        _need(t, torch.bfloat16, n)
    _need(lse_c, torch.float32, "lse_c")
    dq = dq if dq is not None else torch.empty_like(q)
    dk = dk if dk is not None else torch.empty_like(k)
    dv = dv if dv is not None else torch.empty_like(v)
    nbytes = workspace_bytes("global_bwd", d)
    ws = _workspace(nbytes, q.device, workspace)
    _call("logo_global_sparse_attn_bwd", _p(q), _p(k), _p(v), _p(pos), _p(cu_q), _p(n_sel_total), _p(o_c),
          _p(lse_c), _p(dO_c), _p(dq), _p(dk), _p(dv), d, float(scale), _p(ws), nbytes, _stream())
    return dq, dk, dv


def logo_combine(o_l, o_c, gate_p, z, row_of, gain_l=None, gain_g=None, eps: float = 1e-6, o=None, rstd_l=None,
                 rstd_g=None):
    """Eq. 9 ContextNorm + Eq. 10 fusion.  Returns (o, rstd_l, rstd_g)."""
    _need(o_l, torch.bfloat16, "o_l")
    _need(o_c, torch.bfloat16, "o_c")
    B, T, H, D = o_l.shape
    d = Dims(B, T, H, H, D)
    o = o if o is not None else torch.empty_like(o_l)
    rstd_l = rstd_l if rstd_l is not None else torch.empty((B, T, H), dtype=torch.float32, device=o_l.device)
    rstd_g = rstd_g if rstd_g is not None else torch.empty((B * T, H), dtype=torch.float32, device=o_l.device)
    _call("logo_combine", _p(o_l), _p(o_c), _p(gate_p), _p(z), _p(row_of), _p(gain_l), _p(gain_g), float(eps),
          _p(o), _p(rstd_l), _p(rstd_g), d, _stream())
    return o, rstd_l, rstd_g


def logo_combine_bwd(dO, o_l, o_c, gate_p, z, row_of, gain_l=None, gain_g=None, eps: float = 1e-6, dO_l=None,
                     dO_c=None, dgate_p=None):
    """Backward of logo_combine with z fixed.  Returns (dO_l, dO_c, dgate_p)."""
    _need(dO, torch.bfloat16, "dO")
    B, T, H, D = o_l.shape
    d = Dims(B, T, H, H, D)
    dO_l = dO_l if dO_l is not None else torch.empty_like(o_l)
    dO_c = dO_c if dO_c is not None else torch.empty((B * T, H, D), dtype=torch.bfloat16, device=o_l.device)
    dgate_p = dgate_p if dgate_p is not None else torch.empty((B, T), dtype=torch.float32, device=o_l.device)
    _call("logo_combine_bwd", _p(dO), _p(o_l), _p(o_c), _p(gate_p), _p(z), _p(row_of), _p(gain_l), _p(gain_g),
          float(eps), _p(dO_l), _p(dO_c), _p(dgate_p), d, _stream())
    return dO_l, dO_c, dgate_p


def logo_combine_bwd_gains(dO, o_l, o_c, gate_p, z, row_of, gain_l=None, gain_g=None, eps: float = 1e-6,
                           dO_l=None, dO_c=None, dgate_p=None, dgain_l=None, dgain_g=None, workspace=None):
    """logo_combine_bwd plus the ContextNorm gain gradients (Eq. 9).
    Returns (dO_l, dO_c, dgate_p, dgain_l, dgain_g); the gain gradients are
    [Hq, D] float32."""
    _need(dO, torch.bfloat16, "dO")
    B, T, H, D = o_l.shape
    d = Dims(B, T, H, H, D)
    dev = o_l.device
    dO_l = dO_l if dO_l is not None else torch.empty_like(o_l)
    dO_c = dO_c if dO_c is not None else torch.empty((B * T, H, D), dtype=torch.bfloat16, device=dev)
    dgate_p = dgate_p if dgate_p is not None else torch.empty((B, T), dtype=torch.float32, device=dev)
    dgain_l = dgain_l if dgain_l is not None else torch.empty((H, D), dtype=torch.float32, device=dev)
    dgain_g = dgain_g if dgain_g is not None else torch.empty((H, D), dtype=torch.float32, device=dev)
    nbytes = int(lib().logo_combine_bwd_workspace_size(d))
    ws = _workspace(nbytes, dev, workspace)
    _call("logo_combine_bwd_gains", _p(dO), _p(o_l), _p(o_c), _p(gate_p), _p(z), _p(row_of), _p(gain_l),
          _p(gain_g), float(eps), _p(dO_l), _p(dO_c), _p(dgate_p), _p(dgain_l), _p(dgain_g), d, _p(ws),
          ws.numel(), _stream())
    return dO_l, dO_c, dgate_p, dgain_l, dgain_g

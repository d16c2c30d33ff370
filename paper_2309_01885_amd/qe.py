"""ctypes binding of libqe.so (include/qe.h) on torch device tensors.

Argument marshalling only: every step of the QuantEase hot path runs in the
HIP kernels behind the C ABI; torch provides device memory and the stream.
There is no fallback: if libqe.so is missing or no GPU is present, the calls
raise.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqe.so")

QE_OK = 0
QE_ERR_ARG = 1
QE_ERR_DIAG = 2
QE_ERR_SCALE = 3
QE_ERR_WORKSPACE = 4
QE_ERR_HIP = 5
QE_ERR_UNSUPPORTED = 6
QE_ERR_TOO_LARGE = 7
QE_ERR_NONFINITE = 8
QE_NOALLOC_SCRATCH_BYTES = 64 << 20

QE_LAYOUT_PN = 0
QE_LAYOUT_NP = 1
QE_GRAM_FP32 = 0x100
QE_GRAM_BF16X3 = 0x200

QE_INIT_FROM_W = 0x1
QE_R_VALID = 0x2
QE_CODES_VALID = 0x4
QE_RELAX_MASK = 0xff00
QE_OUTLIER_COLUMNS = 0x10
QE_CD_FP32 = 0x20
QE_CD_DENSE = 0x10000
QE_DEBUG_CHECKS = 0x40
QE_OBJ_IN = 0x80

QE_F32 = 0
QE_F16 = 1
QE_BF16 = 2


def QE_RELAX_PERIOD(k: int) -> int:
    """Flag bits for relaxed sweeps every k-th sweep of a call (qe.h)."""
    return (int(k) & 0xff) << 8

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_int = ctypes.c_int
_f32 = ctypes.c_float
_sz = ctypes.c_size_t

# name -> (restype, argtypes); mirrors include/qe.h
SIGNATURES = {
    "qe_status_string": (ctypes.c_char_p, [_int]),
    "qe_version": (_int, []),
    "qe_sync_status": (_int, [_vp, _vp]),
    "qe_gram_workspace_size": (_sz, [_i64, _i64]),
    "qe_gram": (_int, [_vp, _i64, _i64, _int, _vp, _int, _f32, _vp, _sz, _vp]),
    "qe_grid_minmax": (_int, [_vp, _vp, _i64, _i64, _int, _vp, _vp, _vp]),
    "qe_cd_workspace_size": (_sz, [_i64, _i64, _int]),
    "qe_cd_sweep": (_int, [_vp, _vp, _i64, _i64, _int, _vp, _vp, _vp, _vp, _vp, _int, _int,
                           ctypes.c_uint32, _vp, _vp, _sz, _vp]),
    "qe_cd_sweep_noalloc": (_int, [_vp, _vp, _i64, _i64, _int, _vp, _vp, _vp, _vp, _vp, _int,
                                   _int, ctypes.c_uint32, _vp, _vp, _vp]),
    "qe_outlier_workspace_size": (_sz, [_i64, _i64, _int, _i64]),
    "qe_cd_outlier_sweep": (_int, [_vp, _vp, _i64, _i64, _int, _vp, _vp, _vp, _vp, _vp, _vp,
                                   _i64, _f32, _vp, _vp, _int, _int, ctypes.c_uint32, _vp, _vp,
                                   _sz, _vp]),
    "qe_topk_workspace_size": (_sz, [_i64, _i64]),
    "qe_topk_abs": (_int, [_vp, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "qe_topk_columns_workspace_size": (_sz, [_i64, _i64]),
    "qe_topk_columns": (_int, [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "qe_packed_row_bytes": (_i64, [_i64, _int]),
    "qe_pack_codes": (_int, [_vp, _i64, _i64, _int, _vp, _vp]),
    "qe_outliers_csr": (_int, [_vp, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _vp]),
    "qe_objective_workspace_size": (_sz, [_i64, _i64]),
    "qe_objective": (_int, [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "qe_lambda_workspace_size": (_sz, [_i64]),
    "qe_lambda_max": (_int, [_vp, _i64, _int, _f32, ctypes.POINTER(_f32), _vp, _sz, _vp]),
    "qe_kv_page_bytes": (_i64, [_int, _int, _int, _int]),
    "qe_kv_write": (_int, [_vp, _vp, _int, _i64, _int, _int, _i64, _i64, _i64, _i64, _vp, _int, _vp, _i64,
                           _int, _vp, _vp]),
    "qe_kv_read": (_int, [_vp, _i64, _int, _vp, _i64, _int, _int, _int, _vp, _vp, _int, _i64, _i64, _i64,
                          _i64, _vp, _vp]),
    "qe_kv_extend_workspace_size": (_sz, [_i64]),
    "qe_kv_extend": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _int, _i64, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "qe_kv_append": (_int, [_vp, _vp, _vp, _int, _i64, _int, _int, _int, _i64, _i64, _i64, _i64, _i64, _i64, _vp, _vp,
                            ctypes.c_double, _vp, _vp, _vp, _i64, _int, _int, _vp, _int, _vp, _i64, _int, _vp, _i64, _i64,
                            _vp, _vp]),
    "qe_kv_attn_workspace_size": (_sz, [_i64, _i64, _i64, _int, _int, _int]),
    "qe_kv_attn": (_int, [_vp, _int, _i64, _int, _int, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _int, _int,
                          _int, _vp, _i64, _vp, _f32, _int, _int, _vp, _vp, _i64, _i64, _vp, _vp, _sz,
                          _vp]),
    "qe_kv_attn_sinks": (_int, [_vp, _int, _i64, _int, _int, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _int, _int,
                                _int, _vp, _i64, _vp, _f32, _int, _int, _int, _vp, _vp, _i64, _i64, _vp, _vp, _sz,
                                _vp]),
    "qe_kv_attn_shared_workspace_size": (_sz, [_i64, _i64, _i64, _int, _int, _int, _i64]),
    "qe_kv_attn_shared": (_int, [_vp, _int, _i64, _int, _int, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _int, _int,
                                 _int, _vp, _i64, _vp, _vp, _vp, _i64, _f32, _int, _vp, _vp, _i64, _i64, _vp, _vp, _sz,
                                 _vp]),
}

_lib = None


class QEError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


def load() -> ctypes.CDLL:
    """Loads libqe.so (built in-tree by paper_2309_01885_amd/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python paper_2309_01885_amd/build.py` (no CPU fallback exists)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def status_string(code: int) -> str:
    return load().qe_status_string(code).decode()


def _stream(stream=None) -> _vp:
    s = torch.cuda.current_stream() if stream is None else stream
    return _vp(s.cuda_stream)


def _ptr(t: Optional[torch.Tensor], dtype, name: str, numel: Optional[int] = None) -> _vp:
    if t is None:
        return _vp(None)
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, got {t.numel()}")
    return _vp(t.data_ptr())


def _check(code: int, where: str):
    if code != QE_OK:
        raise QEError(code, where)


def workspace(nbytes: int, device) -> torch.Tensor:
    """A device workspace; zero-filled, so that its status word reads QE_OK
    before any call has used it."""
    return torch.zeros(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _on(stream, make):
    """make() with `stream` as torch's current stream (None: as it is).  A call's own buffers are made there, so that
    their filling comes before the call's work and their memory is reused after it."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


def sync_status(ws: torch.Tensor, stream=None) -> int:
    """Waits for the stream; returns (and clears) the workspace's device status word."""
    return load().qe_sync_status(_vp(ws.data_ptr()), _stream(stream))


def _finish(ws, check, where, stream=None):
    if check:
        _check(sync_status(ws, stream), where)


# ---------------------------------------------------------------------------- Gram
def gram(X: torch.Tensor, layout: int = QE_LAYOUT_PN, Sigma: Optional[torch.Tensor] = None,
         accumulate: bool = False, damp: float = 0.0, ws: Optional[torch.Tensor] = None,
         check: bool = True, stream=None, fp32: bool = False,
         bf16x3: bool = False) -> torch.Tensor:
    """Sigma (+)= X X^T (qe_gram).  fp32=True selects the fp32 matrix-core
    products (QE_GRAM_FP32), bf16x3=True the three-way bf16 split on every
    tile (QE_GRAM_BF16X3), instead of the default split products."""
    lib = load()
    if X.dim() != 2:
        raise ValueError("X must be 2-D")
    p, n = (X.shape if layout == QE_LAYOUT_PN else X.shape[::-1])
    if fp32:
        layout |= QE_GRAM_FP32
    if bf16x3:
        layout |= QE_GRAM_BF16X3
    if Sigma is None:
        Sigma = _on(stream, lambda: torch.empty((p, p), dtype=torch.float32, device=X.device))
    need = lib.qe_gram_workspace_size(p, n)
    if ws is None:
        ws = _on(stream, lambda: workspace(need, X.device))
    _check(lib.qe_gram(_ptr(X, torch.float32, "X"), p, n, layout,
                       _ptr(Sigma, torch.float32, "Sigma", p * p), 1 if accumulate else 0,
                       float(damp), _vp(ws.data_ptr()), ws.numel(), _stream(stream)), "qe_gram")
    _finish(ws, check, "qe_gram", stream)
    return Sigma


# ---------------------------------------------------------------------------- grid
def grid_minmax(W: torch.Tensor, bits: int, H: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    lib = load()
    q, p = W.shape
    scale = _on(stream, lambda: torch.empty(q, dtype=torch.float32, device=W.device))
    zero = _on(stream, lambda: torch.empty(q, dtype=torch.float32, device=W.device))
    _check(lib.qe_grid_minmax(_ptr(W, torch.float32, "W"), _ptr(H, torch.float32, "H", q * p)
                              if H is not None else _vp(None), q, p, bits,
                              _ptr(scale, torch.float32, "scale"), _ptr(zero, torch.float32, "zero"),
                              _stream(stream)), "qe_grid_minmax")
    return scale, zero


# ---------------------------------------------------------------------------- CD
def cd_workspace_size(q: int, p: int, block: int = 0) -> int:
    return int(load().qe_cd_workspace_size(q, p, block))


def cd_sweep(W, Sigma, bits, scale, zero, W_hat, codes, R, sweeps, block: int = 0,
             flags: int = QE_INIT_FROM_W, obj: Optional[torch.Tensor] = None,
             ws: Optional[torch.Tensor] = None, check: bool = True, stream=None):
    """In place on W_hat (fp32), codes (uint8) and R (fp32), all q x p."""
    lib = load()
    q, p = W.shape
    if ws is None:
        ws = _on(stream, lambda: workspace(cd_workspace_size(q, p, block), W.device))
    if obj is not None and (obj.dtype != torch.float64 or obj.numel() < sweeps):
        raise ValueError("obj must be a float64 device tensor with >= sweeps entries")
    _check(lib.qe_cd_sweep(_ptr(W, torch.float32, "W"), _ptr(Sigma, torch.float32, "Sigma", p * p),
                           q, p, bits, _ptr(scale, torch.float32, "scale", q),
                           _ptr(zero, torch.float32, "zero", q),
                           _ptr(W_hat, torch.float32, "W_hat", q * p),
                           _ptr(codes, torch.uint8, "codes", q * p),
                           _ptr(R, torch.float32, "R", q * p), sweeps, block, flags,
                           _ptr(obj, torch.float64, "obj") if obj is not None else _vp(None),
                           _vp(ws.data_ptr()), ws.numel(), _stream(stream)), "qe_cd_sweep")
    _finish(ws, check, "qe_cd_sweep", stream)
    return W_hat, codes, R


def cd_sweep_noalloc(W, Sigma, bits, scale, zero, W_hat, codes, R, sweeps, block: int = 0,
                     flags: int = QE_INIT_FROM_W, obj: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None):
    """qe_cd_sweep_noalloc: as cd_sweep, with the library's fixed scratch in
    place of a workspace (nothing is allocated).  status: None or an int32
    device tensor of one element receiving the call's data-error status in
    stream order.  Calls that overlap on one GPU race (one shared scratch)."""
    lib = load()
    q, p = W.shape
    if obj is not None and (obj.dtype != torch.float64 or obj.numel() < sweeps):
        raise ValueError("obj must be a float64 device tensor with >= sweeps entries")
    _check(lib.qe_cd_sweep_noalloc(
        _ptr(W, torch.float32, "W"), _ptr(Sigma, torch.float32, "Sigma", p * p), q, p, bits,
        _ptr(scale, torch.float32, "scale", q), _ptr(zero, torch.float32, "zero", q),
        _ptr(W_hat, torch.float32, "W_hat", q * p), _ptr(codes, torch.uint8, "codes", q * p),
        _ptr(R, torch.float32, "R", q * p), sweeps, block, flags,
        _ptr(obj, torch.float64, "obj") if obj is not None else _vp(None),
        _ptr(status, torch.int32, "status", 1) if status is not None else _vp(None),
        _stream(stream)), "qe_cd_sweep_noalloc")
    return W_hat, codes, R


# ---------------------------------------------------------------------------- outlier-aware CD
def outlier_workspace_size(q: int, p: int, block: int, s: int) -> int:
    return int(load().qe_outlier_workspace_size(q, p, block, s))


def cd_outlier_sweep(W, Sigma, bits, scale, zero, W_hat, codes, H, E, s, lambda_max, support,
                     support_nnz, sweeps, block: int = 0, flags: int = QE_INIT_FROM_W,
                     obj: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                     check: bool = True, stream=None):
    """In place on W_hat, codes, H, E, support (int64[s]) and support_nnz (int64[1])."""
    lib = load()
    q, p = W.shape
    if ws is None:
        ws = _on(stream, lambda: workspace(outlier_workspace_size(q, p, block, s), W.device))
    if obj is not None and (obj.dtype != torch.float64 or obj.numel() < 2 * sweeps):
        raise ValueError("obj must be a float64 device tensor with >= 2*sweeps entries")
    _check(lib.qe_cd_outlier_sweep(
        _ptr(W, torch.float32, "W"), _ptr(Sigma, torch.float32, "Sigma", p * p), q, p, bits,
        _ptr(scale, torch.float32, "scale", q), _ptr(zero, torch.float32, "zero", q),
        _ptr(W_hat, torch.float32, "W_hat", q * p), _ptr(codes, torch.uint8, "codes", q * p),
        _ptr(H, torch.float32, "H", q * p), _ptr(E, torch.float32, "E", q * p), int(s),
        float(lambda_max), _ptr(support, torch.int64, "support") if s > 0 else _vp(None),
        _ptr(support_nnz, torch.int64, "support_nnz", 1), sweeps, block, flags,
        _ptr(obj, torch.float64, "obj") if obj is not None else _vp(None),
        _vp(ws.data_ptr()), ws.numel(), _stream(stream)), "qe_cd_outlier_sweep")
    _finish(ws, check, "qe_cd_outlier_sweep", stream)
    return W_hat, codes, H, E


# ---------------------------------------------------------------------------- P_s
def topk_abs(V: torch.Tensor, s: int, ws: Optional[torch.Tensor] = None, check: bool = True,
             stream=None):
    """P_s(V) over all entries of V: returns (dense P_s(V), support int64[s], nnz int64[1])."""
    lib = load()
    count = V.numel()
    out = _on(stream, lambda: torch.empty_like(V))
    support = _on(stream, lambda: torch.zeros(max(int(s), 1), dtype=torch.int64, device=V.device))
    nnz = _on(stream, lambda: torch.zeros(1, dtype=torch.int64, device=V.device))
    if ws is None:
        ws = _on(stream, lambda: workspace(lib.qe_topk_workspace_size(count, s), V.device))
    _check(lib.qe_topk_abs(_ptr(V, torch.float32, "V"), count, int(s),
                           _ptr(out, torch.float32, "out"), _vp(support.data_ptr()),
                           _ptr(nnz, torch.int64, "nnz"), _vp(ws.data_ptr()), ws.numel(),
                           _stream(stream)), "qe_topk_abs")
    _finish(ws, check, "qe_topk_abs", stream)
    return out, support, nnz


def topk_columns(V: torch.Tensor, c: int, ws: Optional[torch.Tensor] = None,
                 check: bool = True, stream=None):
    """Structured projection of the q x p matrix V (c whole columns of largest
    l2 norm): returns (dense result, kept columns int64[c], support int64[q*c],
    nnz int64[1])."""
    lib = load()
    q, p = V.shape
    out = _on(stream, lambda: torch.empty_like(V))
    cols = _on(stream, lambda: torch.full((max(int(c), 1),), -1, dtype=torch.int64, device=V.device))
    support = _on(stream, lambda: torch.zeros(max(int(q * c), 1), dtype=torch.int64, device=V.device))
    nnz = _on(stream, lambda: torch.zeros(1, dtype=torch.int64, device=V.device))
    if ws is None:
        ws = _on(stream, lambda: workspace(lib.qe_topk_columns_workspace_size(q, p), V.device))
    _check(lib.qe_topk_columns(_ptr(V, torch.float32, "V"), q, p, int(c),
                               _ptr(out, torch.float32, "out"), _vp(cols.data_ptr()),
                               _vp(support.data_ptr()), _ptr(nnz, torch.int64, "nnz"),
                               _vp(ws.data_ptr()), ws.numel(), _stream(stream)),
           "qe_topk_columns")
    _finish(ws, check, "qe_topk_columns", stream)
    return out, cols, support, nnz


# ---------------------------------------------------------------------------- export
def pack_codes(codes: torch.Tensor, bits: int, stream=None) -> torch.Tensor:
    """q x p uint8 codes -> q x qe_packed_row_bytes(p, bits) uint8 bit streams."""
    lib = load()
    q, p = codes.shape
    out = _on(stream, lambda: torch.empty((q, int(lib.qe_packed_row_bytes(p, bits))), dtype=torch.uint8,
                                          device=codes.device))
    _check(lib.qe_pack_codes(_ptr(codes, torch.uint8, "codes"), q, p, int(bits),
                             _vp(out.data_ptr()), _stream(stream)), "qe_pack_codes")
    return out


def outliers_csr(H: torch.Tensor, support: torch.Tensor, nnz: torch.Tensor, stream=None):
    """CSR (rowptr int64[q+1], cols int32[cap], vals float32[cap]) of the
    support entries of H; the first nnz entries of cols / vals are valid."""
    lib = load()
    q, p = H.shape
    cap = support.numel()
    rowptr = _on(stream, lambda: torch.empty(q + 1, dtype=torch.int64, device=H.device))
    cols = _on(stream, lambda: torch.empty(max(cap, 1), dtype=torch.int32, device=H.device))
    vals = _on(stream, lambda: torch.empty(max(cap, 1), dtype=torch.float32, device=H.device))
    _check(lib.qe_outliers_csr(_ptr(H, torch.float32, "H"), q, p,
                               _ptr(support, torch.int64, "support"), _ptr(nnz, torch.int64, "nnz"),
                               cap, _vp(rowptr.data_ptr()), _vp(cols.data_ptr()),
                               _vp(vals.data_ptr()), _stream(stream)), "qe_outliers_csr")
    return rowptr, cols, vals


# ---------------------------------------------------------------------------- objective
def objective(W, W_hat, Sigma, H: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None, check: bool = True, stream=None) -> torch.Tensor:
    """Device float64[2]: (||(W_hat + H - W) X||^2, ||W X||^2) through Sigma."""
    lib = load()
    q, p = W.shape
    out = _on(stream, lambda: torch.zeros(2, dtype=torch.float64, device=W.device))
    if ws is None:
        ws = _on(stream, lambda: workspace(lib.qe_objective_workspace_size(q, p), W.device))
    _check(lib.qe_objective(_ptr(W, torch.float32, "W"), _ptr(W_hat, torch.float32, "W_hat", q * p),
                            _ptr(H, torch.float32, "H", q * p) if H is not None else _vp(None),
                            _ptr(Sigma, torch.float32, "Sigma", p * p), q, p,
                            _ptr(out, torch.float64, "out"), _vp(ws.data_ptr()), ws.numel(),
                            _stream(stream)), "qe_objective")
    _finish(ws, check, "qe_objective", stream)
    return out


# ---------------------------------------------------------------------------- lambda_max
def lambda_max(Sigma: torch.Tensor, max_iters: int = 500, tol: float = 1e-7,
               ws: Optional[torch.Tensor] = None, stream=None) -> float:
    lib = load()
    p = Sigma.shape[0]
    if ws is None:
        ws = _on(stream, lambda: workspace(lib.qe_lambda_workspace_size(p), Sigma.device))
    out = _f32(0.0)
    _check(lib.qe_lambda_max(_ptr(Sigma, torch.float32, "Sigma", p * p), p, int(max_iters),
                             float(tol), ctypes.byref(out), _vp(ws.data_ptr()), ws.numel(),
                             _stream(stream)), "qe_lambda_max")
    return float(out.value)


# ---------------------------------------------------------------------------- key/value cache in 4 bits
# These calls come once a layer and token, so their checks are kept short: one read of each
# attribute, plain integers for pointers, the raw stream handle.
_DTYPES = {torch.float32: QE_F32, torch.float16: QE_F16, torch.bfloat16: QE_BF16}
_kv_layouts = {}    # (kv_heads, page / 32, record bytes, dim, group) of caches that fit together


def _bad(name: str, t: torch.Tensor, want: str):
    raise ValueError(f"{name} must be {want}, got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")


def _pages(pages: torch.Tensor, dim: int, group: int):
    """Checks a cache made by kv_pages: (pages, tokens of a page, kv heads, device index)."""
    shape = pages.shape
    if len(shape) != 4 or pages.dtype != torch.uint8 or not pages.is_cuda or not pages.is_contiguous():
        _bad("pages", pages, "a contiguous uint8 device tensor, pages x kv_heads x page / 32 x record bytes (kv_pages)")
    num, kv, per, rec = shape
    key = (kv, per, rec, dim, group)
    if key not in _kv_layouts:
        need = load().qe_kv_page_bytes(kv, dim, group, 32 * per)
        if need == 0 or need != kv * per * rec:
            raise ValueError(f"pages {tuple(shape)} do not fit dim {dim} and group {group}")
        _kv_layouts[key] = True
    return num, 32 * per, kv, pages.get_device()


def _heads(t: torch.Tensor, name: str, shape: tuple, dtype, dev: int):
    """Checks a tokens x heads x dim tensor whose channels are contiguous: (stride of a token, of a head)."""
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or (st[2] != 1 and shape[2] > 1 and t.numel()):
        _bad(name, t, f"{shape} {dtype} on GPU {dev} with contiguous channels")
    return st[0], st[1]


def _flat(t: Optional[torch.Tensor], name: str, dtype, dev: int, numel: Optional[int] = None):
    """Pointer of a contiguous tensor, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != dev or not t.is_contiguous() or (numel is not None and t.numel() != numel):
        _bad(name, t, f"contiguous {dtype}{'' if numel is None else f' of {numel} elements'} on GPU {dev}")
    return t.data_ptr()


def _gpu(t: torch.Tensor, name: str) -> int:
    """Index of a device tensor's GPU."""
    if not t.is_cuda:
        _bad(name, t, "a device tensor")
    return t.get_device()


def _elsewhere(dev: int) -> bool:
    """Whether a call's tensors lie on another GPU than the current one: the call is then made with theirs as the current one."""
    return dev >= 0 and dev != torch._C._cuda_getDevice()


def _raw_stream(dev: int, stream):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def kv_page_bytes(kv_heads: int, dim: int, group: int = 64, page: int = 64) -> int:
    return int(load().qe_kv_page_bytes(kv_heads, dim, group, page))


def kv_pages(num_pages: int, kv_heads: int, dim: int, group: int = 64, page: int = 64,
             device="cuda") -> torch.Tensor:
    """An empty 4-bit key/value cache: uint8, pages x kv_heads x page / 32 x record bytes (qe.h)."""
    nbytes = kv_page_bytes(kv_heads, dim, group, page)
    if nbytes == 0 or num_pages < 1:
        raise ValueError("dim must be a multiple of 8 up to 256, group 32, 64 or 128, page a multiple of 32")
    return torch.zeros((num_pages, kv_heads, page // 32, nbytes // kv_heads // (page // 32)),
                       dtype=torch.uint8, device=device)


def kv_write(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, pages: torch.Tensor, group: int = 64,
             status: Optional[torch.Tensor] = None, stream=None):
    """Quantizes K and V (tokens x kv_heads x dim; any token and head strides) into the
    slots (int64) of the cache (qe_kv_write).  status: None or an int32 device tensor of one element,
    set to QE_ERR_ARG by a slot past the cache (never cleared)."""
    shape, dtype = K.shape, K.dtype
    if len(shape) != 3 or dtype not in _DTYPES:
        _bad("K", K, "tokens x kv_heads x dim in float32, float16 or bfloat16")
    n, _, dim = shape
    num, page, heads, dev = _pages(pages, dim, group)
    shape = (n, heads, dim)
    kt, kh = _heads(K, "K", shape, dtype, dev)
    vt, vh = _heads(V, "V", shape, dtype, dev)
    code = load().qe_kv_write(K.data_ptr(), V.data_ptr(), _DTYPES[dtype], n, heads, dim, kt, kh, vt, vh,
                              _flat(slots, "slots", torch.int64, dev, n), group, pages.data_ptr(), num, page,
                              _flat(status, "status", torch.int32, dev, 1), _raw_stream(dev, stream))
    if code:
        raise QEError(code, "qe_kv_write")
    return pages


def kv_read(pages: torch.Tensor, slots: torch.Tensor, dim: int, group: int = 64, dtype=torch.float32,
            K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None,
            status: Optional[torch.Tensor] = None, stream=None):
    """The keys and values (tokens x kv_heads x dim) that the cache holds at the slots
    (qe_kv_read); into K and V where given (otherwise they are tensors of `stream`: record_stream
    them before they are used on another)."""
    num, page, heads, dev = _pages(pages, dim, group)
    n = slots.numel()
    shape = (n, heads, dim)
    if K is not None or V is not None:
        dtype = (K if K is not None else V).dtype
    if dtype not in _DTYPES:
        raise ValueError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
    if K is None:
        K = _on(stream, lambda: torch.empty(shape, dtype=dtype, device=pages.device))
    if V is None:
        V = _on(stream, lambda: torch.empty(shape, dtype=dtype, device=pages.device))
    kt, kh = _heads(K, "K", shape, dtype, dev)
    vt, vh = _heads(V, "V", shape, dtype, dev)
    code = load().qe_kv_read(pages.data_ptr(), num, page, _flat(slots, "slots", torch.int64, dev), n, heads, dim, group,
                             K.data_ptr(), V.data_ptr(), _DTYPES[dtype], kt, kh, vt, vh,
                             _flat(status, "status", torch.int32, dev, 1), _raw_stream(dev, stream))
    if code:
        raise QEError(code, "qe_kv_read")
    return K, V


def kv_extend_workspace_size(batch: int) -> int:
    return int(load().qe_kv_extend_workspace_size(batch))


def kv_extend(counts: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, free: torch.Tensor,
              free_count: torch.Tensor, page: int, total: int, keep: Optional[torch.Tensor] = None,
              slots: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
              q_start: Optional[torch.Tensor] = None, lacking: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None, check: bool = False, stream=None):
    """Pages and slots for counts[b] (int32; negative: taken back) more tokens of each sequence (qe_kv_extend).

    Updates table (int32, sequences x pages), lengths (int32), free (int32, one entry for each page of the cache: the
    free pages' numbers are its first free_count entries) and free_count (int32, one element) in place.
    Returns slots (int64) and positions (int32) of the call's `total` rows, -1 for rows that are no token's,
    and q_start (int32, sequences + 1), into the tensors given or new ones of `stream`.  keep (int32): so many of each
    sequence's first pages are the caller's.  lacking: None or int32 of one element, the pages that were
    not there; a sequence without its pages stays as it is and its slots are -1.  To take a step back, give the next call the
    lengths before it less those after it (two tensors of the device, no wait): the opposite counts would take tokens from a
    sequence that was refused its own.  The call does not wait for the device; check=True does, and raises if it met lengths that do
    not fit the table."""
    if table.dim() != 2:
        _bad("table", table, "sequences x pages")
    batch, width = table.shape
    dev = _gpu(table, "table")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return kv_extend(counts, table, lengths, free, free_count, page, total, keep, slots, positions, q_start, lacking, ws, check,
                             stream)
    i32 = torch.int32

    def made(t, name, dtype, n):
        """An output, given (checked) or new, and its pointer."""
        if t is None:
            t = _on(stream, lambda: table.new_empty(n, dtype=dtype))
            return t, t.data_ptr()
        return t, _flat(t, name, dtype, dev, n)

    slots, to_slots = made(slots, "slots", torch.int64, total)
    positions, to_positions = made(positions, "positions", i32, total)
    q_start, to_start = made(q_start, "q_start", i32, batch + 1)
    if ws is None:
        ws = _on(stream, lambda: workspace(kv_extend_workspace_size(batch), table.device))
    code = load().qe_kv_extend(_flat(counts, "counts", i32, dev, batch), batch, _flat(table, "table", i32, dev), width,
                               _flat(lengths, "lengths", i32, dev, batch), None if keep is None else _flat(keep, "keep", i32, dev, batch),
                               _flat(free, "free", i32, dev), free.numel(), _flat(free_count, "free_count", i32, dev, 1),
                               page, total, to_slots, to_positions, to_start,
                               None if lacking is None else _flat(lacking, "lacking", i32, dev, 1), _flat(ws, "ws", torch.uint8, dev),
                               ws.numel(), _raw_stream(dev, stream))
    if code:
        raise QEError(code, "qe_kv_extend")
    if check:
        _finish(ws, check, "qe_kv_extend", stream)
    return slots, positions, q_start


def kv_append(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, pages: torch.Tensor,
              group: int = 64, positions: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None,
              sin: Optional[torch.Tensor] = None, interleaved: bool = False, q_weight: Optional[torch.Tensor] = None,
              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, out: Optional[torch.Tensor] = None,
              status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Norm and rotation of Q (tokens x heads x dim) and K (tokens x kv_heads x dim), and the write of K and V into the
    slots of the cache, in one pass (qe_kv_append); returns the queries, in `out` (Q itself is allowed) or a
    new tensor of `stream`.

    q_weight, k_weight: float32 of dim elements, or None for no norm.  cos, sin: float32, positions x rot / 2,
    or None for no rotation; positions (int32) names each token's row, a negative one skips the token, whose row of the
    output is not written.  interleaved pairs channels 2 i and 2 i + 1 instead of i and i + rot / 2.  status:
    None or an int32 device tensor of one element, set to QE_ERR_ARG by a slot past the cache or a position past
    the tables (never cleared).  No gradient: the output has no graph."""
    shape, dtype = Q.shape, Q.dtype
    if len(shape) != 3 or dtype not in _DTYPES:
        _bad("Q", Q, "tokens x heads x dim in float32, float16 or bfloat16")
    n, heads, dim = shape
    num, page, kv, dev = _pages(pages, dim, group)
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return kv_append(Q, K, V, slots, pages, group, positions, cos, sin, interleaved, q_weight, k_weight, eps, out, status, stream)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    rows = half = 0
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape:
            _bad("cos", cos, "positions x rot / 2, as sin")
        if positions is None:
            raise ValueError("a rotation needs positions")
        rows, half = cos.shape
    qt, qh = _heads(Q, "Q", shape, dtype, dev)
    kt, kh = _heads(K, "K", (n, kv, dim), dtype, dev)
    vt, vh = _heads(V, "V", (n, kv, dim), dtype, dev)
    if out is None:
        out = _on(stream, lambda: Q.new_empty(shape))
        ot, oh = heads * dim, dim
    else:
        ot, oh = _heads(out, "out", shape, dtype, dev)
    f32 = torch.float32
    code = load().qe_kv_append(Q.data_ptr(), K.data_ptr(), V.data_ptr(), _DTYPES[dtype], n, heads, kv, dim, qt, qh, kt, kh, vt, vh,
                               _flat(q_weight, "q_weight", f32, dev, dim), _flat(k_weight, "k_weight", f32, dev, dim), eps,
                               _flat(positions, "positions", torch.int32, dev, n), _flat(cos, "cos", f32, dev),
                               _flat(sin, "sin", f32, dev), rows, 2 * half, 1 if interleaved else 0,
                               _flat(slots, "slots", torch.int64, dev, n), group, pages.data_ptr(), num, page, out.data_ptr(),
                               ot, oh, None if status is None else _flat(status, "status", torch.int32, dev, 1), _raw_stream(dev, stream))
    if code:
        raise QEError(code, "qe_kv_append")
    return out


def kv_attn_workspace_size(total: int, batch: int, max_q: int, heads: int, kv_heads: int, dim: int) -> int:
    return int(load().qe_kv_attn_workspace_size(total, batch, max_q, heads, kv_heads, dim))


def _attn(Q, pages, table, lengths, group, q_start, max_q, scale, causal, window, sinks, slopes, out, lse, ws, check, stream, groups,
          shared):
    """kv_attn, and kv_attn_shared where `shared` is given."""
    shape, dtype = Q.shape, Q.dtype
    if len(shape) != 3 or dtype not in _DTYPES:
        _bad("Q", Q, "total x heads x dim in float32, float16 or bfloat16")
    if table.dim() != 2:
        _bad("table", table, "sequences x pages")
    total, heads, dim = shape
    batch, width = table.shape
    num, page, kv, dev = _pages(pages, dim, group)
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return _attn(Q, pages, table, lengths, group, q_start, max_q, scale, causal, window, sinks, slopes, out, lse, ws, check,
                         stream, groups, shared)
    if q_start is None:
        if max_q is None:
            max_q = total // batch if batch else 0
        if total != batch * max_q:
            raise ValueError(f"{total} queries are not {max_q} for each of {batch} sequences: give q_start")
    elif max_q is None:
        raise ValueError("q_start needs max_q, the largest number of queries of a sequence")
    shape = (total, heads, dim)
    if not -0x80000000 <= window <= 0x7fffffff:      # (a C int would take its low bits: 2^32 as no window)
        window = 0x7fffffff if window > 0 else -1
    qt, qh = _heads(Q, "Q", shape, dtype, dev)
    if out is None:
        out = _on(stream, lambda: torch.empty(shape, dtype=dtype, device=pages.device))
        ot, oh = heads * dim, dim
    else:
        ot, oh = _heads(out, "out", shape, dtype, dev)
    if ws is None:
        need = (kv_attn_workspace_size(total, batch, max_q, heads, kv, dim) if shared is None else
                kv_attn_shared_workspace_size(total, batch, max_q, heads, kv, dim, shared.numel()))
        ws = _on(stream, lambda: workspace(need, pages.device))
    queries = (Q.data_ptr(), _DTYPES[dtype], total, heads, dim, qt, qh,
               None if q_start is None else _flat(q_start, "q_start", torch.int32, dev, batch + 1), batch, max_q, pages.data_ptr(),
               num, page, kv, group, _flat(table, "table", torch.int32, dev), width,
               _flat(lengths, "lengths", torch.int32, dev, batch))
    scale = dim ** -0.5 if scale is None else scale
    rest = (None if slopes is None else _flat(slopes, "slopes", torch.float32, dev, heads), out.data_ptr(), ot, oh,
            None if lse is None else _flat(lse, "lse", torch.float32, dev, total * heads),
            _flat(ws, "ws", torch.uint8, dev), ws.numel(), _raw_stream(dev, stream))
    if shared is not None:
        code = load().qe_kv_attn_shared(*queries, _flat(groups, "groups", torch.int32, dev, shared.numel() + 1),
                                        _flat(shared, "shared", torch.int32, dev), shared.numel(), scale, 1 if causal else 0, *rest)
    elif sinks:
        sinks = min(max(sinks, -1), 0x7fffffff)
        code = load().qe_kv_attn_sinks(*queries, scale, 1 if causal else 0, window, sinks, *rest)
    else:
        code = load().qe_kv_attn(*queries, scale, 1 if causal else 0, window, *rest)
    if code:
        raise QEError(code, "qe_kv_attn" if shared is None else "qe_kv_attn_shared")
    if check:
        _finish(ws, check, "qe_kv_attn" if shared is None else "qe_kv_attn_shared", stream)
    return out


def kv_attn(Q: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
            group: int = 64, q_start: Optional[torch.Tensor] = None, max_q: Optional[int] = None,
            scale: Optional[float] = None, causal: bool = True, window: int = 0,
            slopes: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
            lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, check: bool = False,
            stream=None, sinks: int = 0) -> torch.Tensor:
    """Attention of Q (total x heads x dim) over the 4-bit cache (qe_kv_attn, qe_kv_attn_sinks).

    table (int32, sequences x pages) and lengths (int32) describe the sequences; q_start (int32,
    sequences + 1) and max_q their queries, without them total / sequences queries each.
    scale: 1 / sqrt(dim) unless given.  window: 0 for none; one wider than every sequence hides nothing.  sinks: so many
    first tokens stay visible beside the window.  lse: None or float32, total x heads, written.  The call does
    not wait for the device; check=True does, and raises if it met a bad page number, length or
    query range (sync_status(ws) tells later otherwise).  An output or a workspace that the call makes is
    a tensor of `stream`; rows of it that are no sequence's are not written.  The kernels cut their work for
    sequences that fill the table, so a table much wider than they are costs time.  No gradient:
    the output has no graph."""
    return _attn(Q, pages, table, lengths, group, q_start, max_q, scale, causal, window, sinks, slopes, out, lse, ws, check, stream, None,
                 None)


def kv_attn_sinks(Q: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, window: int,
                  sinks: int, **more) -> torch.Tensor:
    """kv_attn with a window beside which the first `sinks` tokens stay visible (qe_kv_attn_sinks)."""
    return kv_attn(Q, pages, table, lengths, window=window, sinks=sinks, **more)


def kv_attn_shared_workspace_size(total: int, batch: int, max_q: int, heads: int, kv_heads: int, dim: int,
                                  groups: int) -> int:
    return int(load().qe_kv_attn_shared_workspace_size(total, batch, max_q, heads, kv_heads, dim, groups))


def kv_attn_shared(Q: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                   groups: torch.Tensor, shared: torch.Tensor, group: int = 64, q_start: Optional[torch.Tensor] = None,
                   max_q: Optional[int] = None, scale: Optional[float] = None, causal: bool = True,
                   slopes: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, check: bool = False,
                   stream=None) -> torch.Tensor:
    """kv_attn of sequences that begin with the same pages, which are read once for a group (qe_kv_attn_shared).

    The sequences groups[g] .. groups[g + 1] - 1 (int32, groups + 1 ascending entries) have the same first shared[g]
    (int32) entries in their rows of table; a row's lengths count the shared tokens.  The result is kv_attn's up to
    the rounding of sums.  Worth it behind long prefixes; in a table much wider than the sequences are, kv_attn is the faster
    call for short ones (its own rule only sees the table's width).  Up to 1024 groups; more are kv_attn's.  The other arguments are
    kv_attn's; kv_attn_shared_workspace_size gives the workspace."""
    return _attn(Q, pages, table, lengths, group, q_start, max_q, scale, causal, 0, 0, slopes, out, lse, ws, check, stream, groups, shared)

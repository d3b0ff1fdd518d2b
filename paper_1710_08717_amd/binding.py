"""Binding of ``libla_mi355x.so``: argument marshalling only, by ctypes, and for plain calls by ``_la_host.so``.

Each function mirrors one ``la_*`` entry point of ``include/la.h``.  Tensors must live on
the GPU, be contiguous and be float32 or float64; all leading axes are flattened into the
batch ("batch mode", section 4.1 of the paper).  Work is enqueued on torch's current
stream.
"""
import contextlib
import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libla_mi355x.so")
_lib = None
_host = None  # the module of csrc/host_call.cpp, once load() has run

SYMBOLS = [
    "la_potrf_batched", "la_potrf_backward", "la_trsm_batched", "la_trmm_batched", "la_syrk_batched",
    "la_sumlogdiag", "la_gp_glue", "la_gemm2_batched", "la_trsm_backward", "la_trmm_backward", "la_syrk_backward",
    "la_gemm2_backward", "la_potri", "la_potri_backward", "la_sgp_workspace_bytes", "la_sgp_criterion",
    "la_kalman_filter", "la_gp_workspace_bytes", "la_gp_criterion",
    "la_last_error", "la_version",
    "la_workspace_bytes", "la_potrf_batched_ws", "la_potrf_backward_ws", "la_trsm_batched_ws", "la_trmm_batched_ws",
    "la_syrk_batched_ws", "la_gemm2_batched_ws", "la_trsm_backward_ws", "la_trmm_backward_ws", "la_syrk_backward_ws",
    "la_gemm2_backward_ws", "la_potri_ws", "la_potri_backward_ws", "la_potrf_batched_noalloc",
    "la_delta_rule_workspace_bytes", "la_delta_rule_saved_bytes", "la_delta_rule", "la_delta_rule_backward_workspace_bytes",
    "la_delta_rule_backward", "la_delta_rule_step", "la_layer_norm", "la_layer_norm_backward_workspace_bytes", "la_layer_norm_backward",
    "la_clip_gradients_workspace_bytes", "la_clip_gradients",
]

# la_op of include/la.h
OP_POTRF, OP_POTRF_BACKWARD, OP_TRSM, OP_TRMM, OP_SYRK, OP_GEMM2 = 0, 1, 2, 3, 4, 5
OP_TRSM_BACKWARD, OP_TRMM_BACKWARD, OP_SYRK_BACKWARD, OP_GEMM2_BACKWARD, OP_POTRI, OP_POTRI_BACKWARD = 6, 7, 8, 9, 10, 11


class LaError(RuntimeError):
    pass


def lib_path():
    return _LIB_PATH


def load():
    """Load the HIP library (built beforehand by ``paper_1710_08717_amd.build``); raises if absent."""
    global _lib, _host
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise LaError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_1710_08717_amd.build` "
            "(there is no fallback path)"
        )
    from . import _la_host

    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double
    lib.la_potrf_batched.argtypes = [i32, i32, i64, i32, vp, vp, vp, vp]
    lib.la_potrf_backward.argtypes = [i32, i32, i64, i32, vp, vp, vp, vp]
    lib.la_trsm_batched.argtypes = [i32, i32, i32, i32, f64, i64, i32, i32, vp, vp, vp, vp]
    lib.la_trmm_batched.argtypes = [i32, i32, i32, i32, f64, i64, i32, i32, vp, vp, vp, vp]
    lib.la_syrk_batched.argtypes = [i32, i32, f64, i64, i32, i32, vp, vp, vp]
    lib.la_sumlogdiag.argtypes = [i32, i64, i32, vp, vp, vp]
    lib.la_gp_glue.argtypes = [i32, i64, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.la_gemm2_batched.argtypes = [i32, i32, i32, f64, i64, i32, i32, i32, vp, vp, vp, vp]
    lib.la_gemm2_batched.restype = i32
    lib.la_trsm_backward.argtypes = [i32, i32, i32, i32, f64, i64, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.la_trmm_backward.argtypes = [i32, i32, i32, i32, f64, i64, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.la_syrk_backward.argtypes = [i32, i32, f64, i64, i32, i32, vp, vp, vp, vp]
    lib.la_gemm2_backward.argtypes = [i32, i32, i32, f64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.la_potri.argtypes = [i32, i32, i64, i32, vp, vp, vp]
    lib.la_potri_backward.argtypes = [i32, i32, i64, i32, vp, vp, vp, vp, vp]
    for name in ("la_trsm_backward", "la_trmm_backward", "la_syrk_backward", "la_gemm2_backward", "la_potri",
                 "la_potri_backward"):
        getattr(lib, name).restype = i32
    lib.la_sgp_workspace_bytes.argtypes = [i32, i32, i32]
    lib.la_sgp_workspace_bytes.restype = ctypes.c_size_t
    lib.la_sgp_criterion.argtypes = [i32, i32, i32, vp, vp, vp, vp, f64, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.la_sgp_criterion.restype = i32
    lib.la_kalman_filter.argtypes = [i32, i64, i32, i32, i32, i32] + [vp] * 12
    lib.la_kalman_filter.restype = i32
    lib.la_gp_workspace_bytes.argtypes = [i32, i64, i32]
    lib.la_gp_workspace_bytes.restype = ctypes.c_size_t
    lib.la_gp_criterion.argtypes = [i32, i64, i32, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.la_gp_criterion.restype = i32
    lib.la_last_error.restype = ctypes.c_char_p
    lib.la_version.restype = i32
    for name in SYMBOLS[:7]:
        getattr(lib, name).restype = i32
    lib.la_potrf_batched_noalloc.argtypes = lib.la_potrf_batched.argtypes
    lib.la_potrf_batched_noalloc.restype = i32
    lib.la_workspace_bytes.argtypes = [i32, i32, i64, i32, i32, i32]
    lib.la_workspace_bytes.restype = ctypes.c_size_t
    rule, sz = [i32, i64, i64, i32, i32, i32, i32], ctypes.c_size_t
    rows = rule + [vp, vp, i64, vp, i64, vp, i64, vp, vp, f64, vp]  # offsets, q, k, v, g, beta, scale, initial_state
    for name, args in (
        ("la_delta_rule_workspace_bytes", rule + [i32]), ("la_delta_rule_saved_bytes", rule + [i32]),
        ("la_delta_rule_backward_workspace_bytes", rule + [i32, i32]),
        ("la_layer_norm_backward_workspace_bytes", [i32, i64, i32]), ("la_clip_gradients_workspace_bytes", [i32, vp]),
        ("la_delta_rule", rows + [vp, vp, vp, sz, vp, sz, vp]),
        ("la_delta_rule_backward", rows + [vp, vp, vp, sz] + [vp] * 6 + [vp, sz, vp]),
        ("la_delta_rule_step", [i32, i64, i32, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, vp, f64, vp, i64, vp, vp, vp]),
        ("la_layer_norm", [i32, i32, i64, i32, i64, vp, vp, vp, f64, vp, vp, vp, vp]),
        ("la_layer_norm_backward", [i32, i32, i64, i32, i64] + [vp] * 8 + [vp, sz, vp]),
        ("la_clip_gradients", [i32, vp, vp, vp, vp, f64, i32, vp, vp, sz, vp]),
    ):
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = sz if name.endswith("_bytes") else i32
    # the _ws form of an entry point: its arguments with (workspace, workspace_bytes) before the stream
    for name in SYMBOLS:
        if name.endswith("_ws"):
            plain = getattr(lib, name[:-3])
            f = getattr(lib, name)
            f.argtypes = plain.argtypes[:-1] + [vp, ctypes.c_size_t, vp]
            f.restype = i32
    _la_host.bind(_LIB_PATH)
    _lib = lib
    _host = _la_host
    return lib


_STATUS = {1: "LA_ERR_INVALID_ARG", 2: "LA_ERR_UNSUPPORTED", 3: "LA_ERR_RUNTIME", 4: "LA_ERR_WORKSPACE"}


def _check(rc, name):
    if rc != 0:
        msg = f"{name}: {_STATUS.get(rc, rc)}"
        if rc in (3, 4):
            msg += f" ({load().la_last_error().decode()})"
        raise LaError(msg)


def _dt(t):
    if t.dtype == torch.float32:
        return 0
    if t.dtype == torch.float64:
        return 1
    raise LaError(f"unsupported dtype {t.dtype}")


def _chk(*ts):
    d = ts[0]
    for t in ts:
        if not t.is_cuda:
            raise LaError("tensors must be on the GPU")
        if not t.is_contiguous():
            raise LaError("tensors must be contiguous")
        if t.dtype != d.dtype or t.device != d.device:
            raise LaError("tensors must share dtype and device")


# The calls on small matrices take a few microseconds of GPU time, so what the host does per call counts.  A call with
# no tensor of the caller's for results, info or scratch goes through csrc/host_call.cpp first, which makes it or answers
# None where it is not a plain one (potrf, trsm, potrf_backward and sumlogdiag of 16 matrices of 32 x 32: 8.6, 10.5, 9.3 and
# 8.3 us of host time through ctypes, 4.8, 5.0, 4.9 and 4.3 through it, 3 of them the launch).
# What comes here hands pointers to ctypes as plain integers, switches the device only where it is another one, and asks
# for the stream's handle without building a Stream object.
_HERE = contextlib.nullcontext()


def _on_device(t):
    d = t.get_device()
    return _HERE if d == torch.cuda.current_device() else torch.cuda.device(d)


def _stream(t):
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _batch(t, trailing=2):
    b = 1
    for s in t.shape[: t.dim() - trailing]:
        b *= s
    return b


_ws_sizes = {}


def workspace_bytes(op, t, batch, n=0, m=0, k=0):
    """la_workspace_bytes for tensors of t's dtype (the answers are remembered: they depend on the sizes only)."""
    key = (op, t.dtype, batch, n, m, k)
    need = _ws_sizes.get(key)
    if need is None:
        need = _ws_sizes[key] = int(load().la_workspace_bytes(op, _dt(t), batch, n, m, k))
    return need


def _ws(workspace, op, t, batch, n=0, m=0, k=0):
    """(tensor, pointer, bytes) of the scratch memory of one call: the caller's uint8 device tensor, or, when the call
    needs one and none was given, a fresh one from torch's allocator (stream-ordered on the current stream)."""
    if workspace is not None:
        assert workspace.dtype == torch.uint8 and workspace.is_cuda and workspace.is_contiguous()
        return workspace, workspace.data_ptr(), workspace.numel()
    need = workspace_bytes(op, t, batch, n, m, k)
    if need == 0:
        return None, 0, 0
    buf = torch.empty(need, dtype=torch.uint8, device=t.device)
    return buf, buf.data_ptr(), need  # the caller keeps buf until the call is enqueued


def potrf(A, lower=True, out=None, info=None, workspace=None):
    """la_potrf_batched.  ``out`` may be ``A`` itself (in place).  ``info``: int32 [batch] or None."""
    if _host is not None and out is None and info is None and workspace is None:
        r = _host.potrf(A, lower)
        if r is not None:
            return r
    _chk(A)
    n = A.shape[-1]
    assert A.shape[-2] == n
    L = torch.empty_like(A) if out is None else out
    _chk(A, L)
    if info is not None:
        assert info.dtype == torch.int32 and info.is_cuda and info.numel() == _batch(A)
    with _on_device(A):
        keep, wp, wb = _ws(workspace, OP_POTRF, A, _batch(A), n)
        _check(load().la_potrf_batched_ws(_dt(A), int(lower), _batch(A), n, _ptr(A), _ptr(L), _ptr(info), wp, wb,
                                          _stream(A)), "la_potrf_batched_ws")
    return L


NOALLOC_SCRATCH_BYTES = 64 << 20  # LA_NOALLOC_SCRATCH_BYTES of include/la.h


def potrf_noalloc(A, out, lower=True, info=None):
    """la_potrf_batched_noalloc: potrf on the library's static scratch array; the caller supplies ``out``
    (which may be ``A``), nothing is allocated here or in the library."""
    _chk(A, out)
    n = A.shape[-1]
    assert A.shape[-2] == n and out.shape == A.shape
    if info is not None:
        assert info.dtype == torch.int32 and info.is_cuda and info.numel() == _batch(A)
    with _on_device(A):
        _check(load().la_potrf_batched_noalloc(_dt(A), int(lower), _batch(A), n, _ptr(A), _ptr(out), _ptr(info),
                                               _stream(A)), "la_potrf_batched_noalloc")
    return out


def potrf_backward(L, Lbar, lower=True, out=None, workspace=None):
    """la_potrf_backward.  ``out`` may be ``Lbar`` itself."""
    if _host is not None and out is None and workspace is None:
        r = _host.potrf_backward(L, Lbar, lower)
        if r is not None:
            return r
    _chk(L, Lbar)
    n = L.shape[-1]
    assert L.shape == Lbar.shape and L.shape[-2] == n
    Abar = torch.empty_like(Lbar) if out is None else out
    _chk(L, Abar)
    with _on_device(L):
        keep, wp, wb = _ws(workspace, OP_POTRF_BACKWARD, L, _batch(L), n)
        _check(load().la_potrf_backward_ws(_dt(L), int(lower), _batch(L), n, _ptr(L), _ptr(Lbar), _ptr(Abar), wp, wb,
                                           _stream(L)), "la_potrf_backward_ws")
    return Abar


def _tri(op, name, L, A, lower, trans, rightside, alpha, out, workspace):
    if _host is not None and out is None and workspace is None:
        r = _host.tri(op == OP_TRSM, L, A, lower, trans, rightside, alpha)
        if r is not None:
            return r
    _chk(L, A)
    n = L.shape[-1]
    assert L.shape[-2] == n
    m = A.shape[-2] if rightside else A.shape[-1]
    assert (A.shape[-1] if rightside else A.shape[-2]) == n
    assert _batch(L) == _batch(A)
    B = torch.empty_like(A) if out is None else out
    _chk(A, B)
    with _on_device(L):
        keep, wp, wb = _ws(workspace, op, L, _batch(L), n, m)
        _check(getattr(load(), name)(_dt(L), int(lower), int(trans), int(rightside), float(alpha), _batch(L), n, m,
                                     _ptr(L), _ptr(A), _ptr(B), wp, wb, _stream(L)), name)
    return B


def trsm(L, A, lower=True, trans=False, rightside=False, alpha=1.0, out=None, workspace=None):
    return _tri(OP_TRSM, "la_trsm_batched_ws", L, A, lower, trans, rightside, alpha, out, workspace)


def trmm(L, A, lower=True, trans=False, rightside=False, alpha=1.0, out=None, workspace=None):
    return _tri(OP_TRMM, "la_trmm_batched_ws", L, A, lower, trans, rightside, alpha, out, workspace)


def _tri_backward(op, name, L, X, Bbar, lower, trans, rightside, alpha, out_a, out_l, workspace):
    if _host is not None and out_a is None and out_l is None and workspace is None:
        r = _host.tri_backward(op == OP_TRSM_BACKWARD, L, X, Bbar, lower, trans, rightside, alpha)
        if r is not None:
            return r
    _chk(L, X)
    _chk(L, Bbar)
    n = L.shape[-1]
    assert L.shape[-2] == n and X.shape == Bbar.shape
    m = X.shape[-2] if rightside else X.shape[-1]
    assert (X.shape[-1] if rightside else X.shape[-2]) == n and _batch(L) == _batch(X)
    Abar = torch.empty_like(Bbar) if out_a is None else out_a
    Lbar = torch.empty_like(L) if out_l is None else out_l
    _chk(L, Abar)
    _chk(L, Lbar)
    with _on_device(L):
        keep, wp, wb = _ws(workspace, op, L, _batch(L), n, m)
        _check(getattr(load(), name)(_dt(L), int(lower), int(trans), int(rightside), float(alpha), _batch(L), n, m,
                                     _ptr(L), _ptr(X), _ptr(Bbar), _ptr(Abar), _ptr(Lbar), wp, wb, _stream(L)), name)
    return Abar, Lbar


def trsm_backward(L, B, Bbar, lower=True, trans=False, rightside=False, alpha=1.0, out_a=None, out_l=None,
                  workspace=None):
    """la_trsm_backward: (Abar, Lbar) from the forward OUTPUT B.  out_a may be Bbar, out_l may be L."""
    return _tri_backward(OP_TRSM_BACKWARD, "la_trsm_backward_ws", L, B, Bbar, lower, trans, rightside, alpha, out_a,
                         out_l, workspace)


def trmm_backward(L, A, Bbar, lower=True, trans=False, rightside=False, alpha=1.0, out_a=None, out_l=None,
                  workspace=None):
    """la_trmm_backward: (Abar, Lbar) from the forward INPUT A.  out_a may be Bbar."""
    return _tri_backward(OP_TRMM_BACKWARD, "la_trmm_backward_ws", L, A, Bbar, lower, trans, rightside, alpha, out_a,
                         out_l, workspace)


def syrk_backward(A, Bbar, trans=False, alpha=1.0, out=None, workspace=None):
    """la_syrk_backward: Abar = alpha (Bbar + Bbar^T) A  or  alpha A (Bbar + Bbar^T)."""
    if _host is not None and out is None and workspace is None:
        r = _host.syrk_backward(A, Bbar, trans, alpha)
        if r is not None:
            return r
    _chk(A, Bbar)
    n, k = (A.shape[-1], A.shape[-2]) if trans else (A.shape[-2], A.shape[-1])
    assert Bbar.shape[-2:] == (n, n) and _batch(A) == _batch(Bbar)
    Abar = torch.empty_like(A) if out is None else out
    _chk(A, Abar)
    with _on_device(A):
        keep, wp, wb = _ws(workspace, OP_SYRK_BACKWARD, A, _batch(A), n, 0, k)
        _check(load().la_syrk_backward_ws(_dt(A), int(trans), float(alpha), _batch(A), n, k, _ptr(A), _ptr(Bbar),
                                          _ptr(Abar), wp, wb, _stream(A)), "la_syrk_backward_ws")
    return Abar


def gemm2_backward(A, B, Cbar, ta=False, tb=False, alpha=1.0, workspace=None):
    """la_gemm2_backward: (Abar, Bbar) of C = alpha t_a(A) t_b(B)."""
    if _host is not None and workspace is None:
        r = _host.gemm2_backward(A, B, Cbar, ta, tb, alpha)
        if r is not None:
            return r
    _chk(A, B)
    _chk(A, Cbar)
    m, k = (A.shape[-1], A.shape[-2]) if ta else (A.shape[-2], A.shape[-1])
    n = B.shape[-2] if tb else B.shape[-1]
    assert Cbar.shape[-2:] == (m, n) and _batch(A) == _batch(B) == _batch(Cbar)
    Abar, Bbar = torch.empty_like(A), torch.empty_like(B)
    with _on_device(A):
        keep, wp, wb = _ws(workspace, OP_GEMM2_BACKWARD, A, _batch(A), n, m, k)
        _check(load().la_gemm2_backward_ws(_dt(A), int(ta), int(tb), float(alpha), _batch(A), m, n, k, _ptr(A), _ptr(B),
                                           _ptr(Cbar), _ptr(Abar), _ptr(Bbar), wp, wb, _stream(A)),
               "la_gemm2_backward_ws")
    return Abar, Bbar


def potri(L, lower=True, out=None, workspace=None):
    """la_potri: A^-1 from the Cholesky factor of A.  ``out`` may be ``L`` itself."""
    if _host is not None and out is None and workspace is None:
        r = _host.potri(L, lower)
        if r is not None:
            return r
    _chk(L)
    n = L.shape[-1]
    assert L.shape[-2] == n
    B = torch.empty_like(L) if out is None else out
    _chk(L, B)
    with _on_device(L):
        keep, wp, wb = _ws(workspace, OP_POTRI, L, _batch(L), n)
        _check(load().la_potri_ws(_dt(L), int(lower), _batch(L), n, _ptr(L), _ptr(B), wp, wb, _stream(L)), "la_potri_ws")
    return B


def potri_backward(L, B, Bbar, lower=True, out=None, workspace=None):
    """la_potri_backward: gradient of the factor from B = A^-1 and Bbar."""
    if _host is not None and out is None and workspace is None:
        r = _host.potri_backward(L, B, Bbar, lower)
        if r is not None:
            return r
    _chk(L, B)
    _chk(L, Bbar)
    n = L.shape[-1]
    assert L.shape == B.shape == Bbar.shape
    Lbar = torch.empty_like(L) if out is None else out
    _chk(L, Lbar)
    with _on_device(L):
        keep, wp, wb = _ws(workspace, OP_POTRI_BACKWARD, L, _batch(L), n)
        _check(load().la_potri_backward_ws(_dt(L), int(lower), _batch(L), n, _ptr(L), _ptr(B), _ptr(Bbar), _ptr(Lbar),
                                           wp, wb, _stream(L)), "la_potri_backward_ws")
    return Lbar


def sgp_criterion(Kuu, Kuf, Kff_diag, y, noise_var, workspace=None):
    """la_sgp_criterion: dict with phi, Kuu_bar, Kuf_bar, Kff_diag_bar, y_bar, noise_bar (device tensors).
    ``workspace``: a uint8 device tensor of at least la_sgp_workspace_bytes bytes (allocated here if absent)."""
    _chk(Kuu, Kuf)
    _chk(Kuu, Kff_diag)
    _chk(Kuu, y)
    U, n = Kuf.shape
    assert Kuu.shape == (U, U) and Kff_diag.shape == (n,) and y.shape == (n,)
    need = int(load().la_sgp_workspace_bytes(_dt(Kuu), U, n))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=Kuu.device)
    out = {"phi": torch.empty(1, dtype=Kuu.dtype, device=Kuu.device), "Kuu_bar": torch.empty_like(Kuu),
           "Kuf_bar": torch.empty_like(Kuf), "Kff_diag_bar": torch.empty_like(Kff_diag), "y_bar": torch.empty_like(y),
           "noise_bar": torch.empty(1, dtype=Kuu.dtype, device=Kuu.device)}
    with _on_device(Kuu):
        _check(load().la_sgp_criterion(_dt(Kuu), U, n, _ptr(Kuu), _ptr(Kuf), _ptr(Kff_diag), _ptr(y), float(noise_var),
                                       _ptr(out["phi"]), _ptr(out["Kuu_bar"]), _ptr(out["Kuf_bar"]),
                                       _ptr(out["Kff_diag_bar"]), _ptr(out["y_bar"]), _ptr(out["noise_bar"]),
                                       workspace.data_ptr(), workspace.numel(), _stream(Kuu)), "la_sgp_criterion")
    return out


def gp_criterion(A, y, out=None, loss=None, info=None, workspace=None):
    """la_gp_criterion: (loss [batch], Abar [batch, n, n]).  ``out`` may be ``A`` itself."""
    if _host is not None and out is None and loss is None and info is None and workspace is None:
        r = _host.gp_criterion(A, y)
        if r is not None:
            return r
    _chk(A, y)
    n = A.shape[-1]
    batch = _batch(A)
    assert A.shape[-2] == n and y.shape[-1] == n and _batch(y, 1) == batch
    Abar = torch.empty_like(A) if out is None else out
    _chk(A, Abar)
    if loss is None:
        loss = torch.empty(A.shape[:-2], dtype=A.dtype, device=A.device)
    _chk(A, loss)
    need = int(load().la_gp_workspace_bytes(_dt(A), batch, n))
    if need and workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=A.device)
    if info is not None:
        assert info.dtype == torch.int32 and info.is_cuda and info.numel() == batch
    with _on_device(A):
        _check(load().la_gp_criterion(_dt(A), batch, n, _ptr(A), _ptr(y), _ptr(loss), _ptr(Abar), _ptr(info),
                                      workspace.data_ptr() if need else 0,
                                      workspace.numel() if need else 0, _stream(A)), "la_gp_criterion")
    return loss, Abar


def kalman_filter(A, B, Sh, Sv, mu0, S0, v, want_states=True, info=None):
    """la_kalman_filter.  Parameters without a batch axis are shared by all sequences of v [batch, T, dv];
    otherwise they carry v's batch axis.  Returns (nll [batch], f [batch, T, dh] or None, F [batch, T, dh, dh] or None)."""
    for x in (B, Sh, Sv, mu0, S0, v):
        _chk(A, x)
    batch, T, dv = v.shape
    shared = A.dim() == 2
    dh = A.shape[-1]
    pb = () if shared else (batch,)
    assert tuple(A.shape) == pb + (dh, dh) and tuple(B.shape) == pb + (dv, dh) and tuple(Sh.shape) == pb + (dh, dh)
    assert tuple(Sv.shape) == pb + (dv, dv) and tuple(mu0.shape) == pb + (dh,) and tuple(S0.shape) == pb + (dh, dh)
    nll = torch.empty(batch, dtype=v.dtype, device=v.device)
    f = torch.empty((batch, T, dh), dtype=v.dtype, device=v.device) if want_states else None
    F = torch.empty((batch, T, dh, dh), dtype=v.dtype, device=v.device) if want_states else None
    if info is not None:
        assert info.dtype == torch.int32 and info.is_cuda and info.numel() == batch
    with _on_device(v):
        _check(load().la_kalman_filter(_dt(v), batch, T, dh, dv, int(shared), _ptr(A), _ptr(B), _ptr(Sh), _ptr(Sv),
                                       _ptr(mu0), _ptr(S0), _ptr(v), _ptr(f), _ptr(F), _ptr(nll), _ptr(info),
                                       _stream(v)), "la_kalman_filter")
    return nll, f, F


def syrk(A, trans=False, alpha=1.0, out=None, workspace=None):
    if _host is not None and out is None and workspace is None:
        r = _host.syrk(A, trans, alpha)
        if r is not None:
            return r
    _chk(A)
    n, k = (A.shape[-1], A.shape[-2]) if trans else (A.shape[-2], A.shape[-1])
    B = torch.empty(A.shape[:-2] + (n, n), dtype=A.dtype, device=A.device) if out is None else out
    _chk(A, B)
    with _on_device(A):
        keep, wp, wb = _ws(workspace, OP_SYRK, A, _batch(A), n, 0, k)
        _check(load().la_syrk_batched_ws(_dt(A), int(trans), float(alpha), _batch(A), n, k, _ptr(A), _ptr(B), wp, wb,
                                         _stream(A)), "la_syrk_batched_ws")
    return B


def gemm2(A, B, ta=False, tb=False, alpha=1.0, out=None, workspace=None):
    """la_gemm2_batched: C = alpha * t_a(A) t_b(B)."""
    if _host is not None and out is None and workspace is None:
        r = _host.gemm2(A, B, ta, tb, alpha)
        if r is not None:
            return r
    _chk(A, B)
    m, k = (A.shape[-1], A.shape[-2]) if ta else (A.shape[-2], A.shape[-1])
    n = B.shape[-2] if tb else B.shape[-1]
    assert (B.shape[-1] if tb else B.shape[-2]) == k and _batch(A) == _batch(B)
    C = torch.empty(A.shape[:-2] + (m, n), dtype=A.dtype, device=A.device) if out is None else out
    _chk(A, C)
    with _on_device(A):
        keep, wp, wb = _ws(workspace, OP_GEMM2, A, _batch(A), n, m, k)
        _check(load().la_gemm2_batched_ws(_dt(A), int(ta), int(tb), float(alpha), _batch(A), m, n, k, _ptr(A), _ptr(B),
                                          _ptr(C), wp, wb, _stream(A)), "la_gemm2_batched_ws")
    return C


def sumlogdiag(L, out=None):
    if _host is not None and out is None:
        r = _host.sumlogdiag(L)
        if r is not None:
            return r
    _chk(L)
    n = L.shape[-1]
    o = torch.empty(L.shape[:-2], dtype=L.dtype, device=L.device) if out is None else out
    with _on_device(L):
        _check(load().la_sumlogdiag(_dt(L), _batch(L), n, _ptr(L), _ptr(o), _stream(L)), "la_sumlogdiag")
    return o


def gp_glue(L, y, z, alpha, loss=None, Lbar=None):
    _chk(L, y, z, alpha)
    n = L.shape[-1]
    loss = torch.empty(L.shape[:-2], dtype=L.dtype, device=L.device) if loss is None else loss
    Lbar = torch.empty_like(L) if Lbar is None else Lbar
    with _on_device(L):
        _check(load().la_gp_glue(_dt(L), _batch(L), n, _ptr(L), _ptr(y), _ptr(z), _ptr(alpha), _ptr(loss), _ptr(Lbar),
                                 _stream(L)), "la_gp_glue")
    return loss, Lbar


# A recurrent sequence layer and its training step.  These take float32, bfloat16 and float16 (layer norm and clipping float64 as well); gates,
# states, statistics and norms are float32 (float64 beside float64).
_LAYER_TYPES = {torch.float32: 0, torch.float64: 1, torch.bfloat16: 2, torch.float16: 3}


def _layer_dt(t):
    if t.dtype not in _LAYER_TYPES:
        raise LaError(f"unsupported dtype {t.dtype}")
    return _LAYER_TYPES[t.dtype]


def _on_gpu(device, dtype, **tensors):
    """Each tensor that is not None: on `device`, of `dtype`, contiguous."""
    for name, t in tensors.items():
        if t is None:
            continue
        if t.device != device:
            raise LaError(f"{name}: tensors must be on the same GPU")
        if t.dtype != dtype:
            raise LaError(f"{name}: {dtype} is wanted, got {t.dtype}")
        if not t.is_contiguous():
            raise LaError(f"{name}: tensors must be contiguous")


def _shape(name, t, want):
    if t is not None and tuple(t.shape) != tuple(want):
        raise LaError(f"{name}: shape {tuple(want)} is wanted, got {tuple(t.shape)}")


def _sizes_fit(**sizes):
    """ctypes takes an int modulo 2^32: what the C entries' own ints do not hold ends here."""
    for name, n in sizes.items():
        if n > 0x7FFFFFFF:
            raise LaError(f"{name}: sizes of up to 2^31 - 1 are taken, got {n} (LA_ERR_UNSUPPORTED)")


def _rows(name, t, inner):
    """Elements from one row to the next of a tensor whose last `inner` axes are dense and whose leading axes are rows one distance apart."""
    want = 1
    if t.numel() == 0:
        for i in range(t.dim() - inner, t.dim()):
            want *= t.shape[i]
        return want
    for i in range(t.dim() - 1, t.dim() - 1 - inner, -1):
        if t.shape[i] != 1 and t.stride(i) != want:
            raise LaError(f"{name}: the last {inner} axes must be contiguous")
        want *= t.shape[i]
    ld, count = None, 1
    for i in range(t.dim() - 1 - inner, -1, -1):
        if t.shape[i] == 1:
            continue
        if ld is None:
            ld = t.stride(i)
            if ld < want:
                raise LaError(f"{name}: rows must not overlap")
        elif t.stride(i) != ld * count:
            raise LaError(f"{name}: rows must be one distance apart")
        count *= t.shape[i]
    return want if ld is None else ld


def _written(*tensors):
    """Tensors of the caller's that a call has written: autograd is told, as of torch's own operators in place."""
    torch.autograd.graph.increment_version([t for t in tensors if t is not None])


def _scratch(workspace, need, t):
    """(tensor, pointer, bytes): the caller's uint8 device tensor, or a fresh one where the call needs some and none was given."""
    if workspace is not None:
        if workspace.dtype != torch.uint8 or workspace.device != t.device or not workspace.is_contiguous():
            raise LaError("a workspace is a contiguous uint8 tensor on the same GPU")
        return workspace, workspace.data_ptr(), workspace.numel()
    if need == 0:
        return None, 0, 0
    buf = torch.empty(need, dtype=torch.uint8, device=t.device)
    return buf, buf.data_ptr(), need  # the caller keeps buf until the call is enqueued


class _Delta:
    """Checked operands of the gated delta rule: q, k [batch, tokens, hk, dk], v [batch, tokens, hv, dv], g, beta [batch, tokens, hv]."""

    def __init__(self, q, k, v, g, beta, offsets, lead=2):
        if not q.is_cuda:
            raise LaError("tensors must be on the GPU")
        self.dt = _layer_dt(q)
        if q.dtype == torch.float64:
            raise LaError("the delta rule takes float32, bfloat16 and float16")
        for name, t in (("q", q), ("k", k), ("v", v)):
            if t.dim() != lead + 2:
                raise LaError(f"{name}: {lead + 2} axes are wanted, got {t.dim()}")
            if t.dtype != q.dtype or t.device != q.device:
                raise LaError("q, k and v must share dtype and device")
        self.hk, self.dk, self.hv, self.dv = q.shape[-2], q.shape[-1], v.shape[-2], v.shape[-1]
        _sizes_fit(hk=self.hk, dk=self.dk, hv=self.hv, dv=self.dv)
        self.lead = tuple(q.shape[:lead])
        _shape("k", k, q.shape)
        if tuple(v.shape[:lead]) != self.lead:
            raise LaError("q and v: the same sequences and tokens are wanted")
        if self.hk < 1 or self.hv < 1 or self.hv % self.hk:
            raise LaError("the value heads must be a multiple of the key heads")
        for name, t in (("g", g), ("beta", beta)):
            _shape(name, t, self.lead + (self.hv,))
        _on_gpu(q.device, torch.float32, g=g, beta=beta)
        self.ld = tuple(_rows(name, t, 2) for name, t in (("q", q), ("k", k), ("v", v)))
        self.batch, self.tokens = (self.lead + (1,))[:2]
        if offsets is not None:
            _on_gpu(q.device, torch.int32, offsets=offsets)
            if offsets.dim() != 1 or offsets.numel() < 2 or self.lead[0] != 1:
                raise LaError("offsets: one axis of at least two, with one row of packed tokens, is wanted")
            self.batch = offsets.numel() - 1
        self.sizes = (self.dt, self.batch, self.tokens, self.hk, self.hv, self.dk, self.dv)
        self.states = (self.batch, self.hv, self.dk, self.dv)
        self.inputs = (_ptr(q), self.ld[0], _ptr(k), self.ld[1], _ptr(v), self.ld[2], _ptr(g), _ptr(beta))

    def scale(self, scale):
        return float(self.dk ** -0.5 if scale is None else scale)


def delta_rule(q, k, v, g, beta, scale=None, initial_state=None, offsets=None, want_state=False, keep=False, out=None, workspace=None):
    """la_delta_rule: the gated delta rule over whole sequences.  q, k [batch, tokens, hk, dk], v [batch, tokens, hv, dv] (views whose tokens
    are one distance apart, as of a wider projection, are taken as they are), g (log decay) and beta [batch, tokens, hv] in float32,
    initial_state [batch, hv, dk, dv] in float32.  ``offsets``: int32 [sequences + 1] on the GPU, with batch = 1: packed sequences of different
    lengths.  ``scale``: dk ** -0.5 where None.  Returns (o, final state or None, saved or None); ``keep``: what delta_rule_backward takes as
    ``saved`` instead of running the forward pass again."""
    d = _Delta(q, k, v, g, beta, offsets)
    o = torch.empty(v.shape, dtype=v.dtype, device=v.device) if out is None else out
    _shape("out", o, v.shape)
    _on_gpu(v.device, v.dtype, out=o)
    _shape("initial_state", initial_state, d.states)
    _on_gpu(v.device, torch.float32, initial_state=initial_state)
    state = torch.empty(d.states, dtype=torch.float32, device=v.device) if want_state else None
    lib, packed = load(), int(offsets is not None)
    with _on_device(q):
        saved = torch.empty(int(lib.la_delta_rule_saved_bytes(*d.sizes, packed)), dtype=torch.uint8, device=v.device) if keep else None
        buf, wp, wb = (None, 0, 0) if keep else _scratch(workspace, int(lib.la_delta_rule_workspace_bytes(*d.sizes, packed)), q)
        _check(lib.la_delta_rule(*d.sizes, _ptr(offsets), *d.inputs, d.scale(scale), _ptr(initial_state), _ptr(o), _ptr(state), _ptr(saved),
                                 saved.numel() if keep else 0, wp, wb, _stream(q)), "la_delta_rule")
    _written(out)
    return o, state, saved


def delta_rule_backward(q, k, v, g, beta, o_bar, scale=None, initial_state=None, state_bar=None, offsets=None, saved=None, workspace=None):
    """la_delta_rule_backward: (q_bar, k_bar, v_bar, g_bar, beta_bar, initial_state_bar) from the gradients of delta_rule's results.
    initial_state_bar is None where initial_state is.  ``saved``: what delta_rule(..., keep=True) gave for the same arguments."""
    d = _Delta(q, k, v, g, beta, offsets)
    _shape("o_bar", o_bar, v.shape)
    _on_gpu(v.device, v.dtype, o_bar=o_bar)
    for name, t in (("initial_state", initial_state), ("state_bar", state_bar)):
        _shape(name, t, d.states)
        _on_gpu(v.device, torch.float32, **{name: t})
    _on_gpu(v.device, torch.uint8, saved=saved)
    new = lambda t, dt=None: torch.empty(t.shape, dtype=dt or t.dtype, device=t.device)  # noqa: E731
    bars = [new(q), new(k), new(v), new(g), new(beta), None if initial_state is None else new(initial_state)]
    lib = load()
    with _on_device(q):
        need = int(lib.la_delta_rule_backward_workspace_bytes(*d.sizes, int(offsets is not None), int(saved is not None)))
        buf, wp, wb = _scratch(workspace, need, q)
        _check(lib.la_delta_rule_backward(*d.sizes, _ptr(offsets), *d.inputs, d.scale(scale), _ptr(initial_state), _ptr(o_bar), _ptr(state_bar),
                                          _ptr(saved), 0 if saved is None else saved.numel(), *[_ptr(t) for t in bars], wp, wb, _stream(q)),
               "la_delta_rule_backward")
    return tuple(bars)


def delta_rule_step(q, k, v, g, beta, state, slots=None, scale=None, out=None):
    """la_delta_rule_step: one token of every sequence: q, k [batch, hk, dk], v [batch, hv, dv], g, beta [batch, hv].  ``state``
    [rows, hv, dk, dv] in float32 is updated in place; sequence n has row ``slots[n]`` (int32, on the GPU), or n.  A slot outside the rows
    gives zeros and updates nothing.  Returns o [batch, hv, dv]."""
    if _host is not None and out is None:
        r = _host.delta_rule_step(q, k, v, g, beta, state, slots, scale)
        if r is not None:
            return r
    d = _Delta(q, k, v, g, beta, None, lead=1)
    o = torch.empty(v.shape, dtype=v.dtype, device=v.device) if out is None else out
    _shape("out", o, v.shape)
    _on_gpu(v.device, v.dtype, out=o)
    _shape("state", state, (*state.shape[:1], d.hv, d.dk, d.dv))
    _on_gpu(v.device, torch.float32, state=state)
    _on_gpu(v.device, torch.int32, slots=slots)
    _shape("slots", slots, (d.batch,))
    with _on_device(q):
        _check(load().la_delta_rule_step(d.dt, d.batch, d.hk, d.hv, d.dk, d.dv, *d.inputs, d.scale(scale), _ptr(state), state.shape[0], _ptr(slots),
                                         _ptr(o), _stream(q)), "la_delta_rule_step")
    _written(state, out)
    return o


def _weights(x, weight, bias):
    """The la_dtype of weight and bias: x's own, or float32 beside 16 bits."""
    w = weight if weight is not None else bias
    dt = x.dtype if w is None else w.dtype
    if dt != x.dtype and not (dt == torch.float32 and x.element_size() == 2):
        raise LaError("weight and bias: x's dtype, or float32 beside 16 bits, is wanted")
    for name, t in (("weight", weight), ("bias", bias)):
        _shape(name, t, x.shape[-1:])
        _on_gpu(x.device, dt, **{name: t})
    return dt


def _norm_input(x):
    if not x.is_cuda:
        raise LaError("tensors must be on the GPU")
    if x.dim() < 1:
        raise LaError("x: at least one axis is wanted")
    _sizes_fit(x=x.shape[-1])
    return _layer_dt(x), _batch(x, 1), x.shape[-1], _rows("x", x, 1)


def layer_norm(x, weight=None, bias=None, eps=1e-5, want_stats=False, out=None):
    """la_layer_norm over the last axis of x (whose rows may be a view's, one distance apart).  Returns (y, mean, rstd), the statistics None
    unless ``want_stats``: layer_norm_backward takes them."""
    if _host is not None and out is None:
        r = _host.layer_norm(x, weight, bias, eps, want_stats)
        if r is not None:
            return r
    dt, rows, n, ld = _norm_input(x)
    wdt = _weights(x, weight, bias)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    _shape("out", y, x.shape)
    _on_gpu(x.device, x.dtype, out=y)
    stat = torch.float64 if x.dtype == torch.float64 else torch.float32
    mean, rstd = (torch.empty(x.shape[:-1], dtype=stat, device=x.device) for _ in range(2)) if want_stats else (None, None)
    with _on_device(x):
        _check(load().la_layer_norm(dt, _LAYER_TYPES[wdt], rows, n, ld, _ptr(x), _ptr(weight), _ptr(bias), float(eps), _ptr(y), _ptr(mean), _ptr(rstd),
                                    _stream(x)), "la_layer_norm")
    _written(out)
    return y, mean, rstd


def layer_norm_backward(x, y_bar, mean, rstd, weight=None, want_weights=True, out=None, workspace=None):
    """la_layer_norm_backward: (x_bar, weight_bar, bias_bar) from layer_norm's input and statistics; the last two None unless
    ``want_weights``, in weight's dtype (x's where weight is None).  ``out`` may be ``y_bar`` itself."""
    if _host is not None and out is None and workspace is None:
        r = _host.layer_norm_backward(x, y_bar, mean, rstd, weight, want_weights)
        if r is not None:
            return r
    dt, rows, n, ld = _norm_input(x)
    wdt = _weights(x, weight, None)
    _shape("y_bar", y_bar, x.shape)
    _on_gpu(x.device, x.dtype, y_bar=y_bar)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _shape(name, t, x.shape[:-1])
        _on_gpu(x.device, torch.float64 if x.dtype == torch.float64 else torch.float32, **{name: t})
    x_bar = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    _shape("out", x_bar, x.shape)
    _on_gpu(x.device, x.dtype, out=x_bar)
    wb, bb = (torch.empty(n, dtype=wdt, device=x.device) for _ in range(2)) if want_weights else (None, None)
    lib = load()
    with _on_device(x):
        buf, wp, wbytes = _scratch(workspace, int(lib.la_layer_norm_backward_workspace_bytes(dt, rows, n)), x)
        _check(lib.la_layer_norm_backward(dt, _LAYER_TYPES[wdt], rows, n, ld, _ptr(x), _ptr(y_bar), _ptr(mean), _ptr(rstd), _ptr(weight), _ptr(x_bar),
                                          _ptr(wb), _ptr(bb), wp, wbytes, _stream(x)), "la_layer_norm_backward")
    _written(out)
    return x_bar, wb, bb


def clip_gradients(grads, max_norm, out=None, workspace=None):
    """la_clip_gradients: scales all tensors of ``grads`` by min(1, max_norm / norm) over all of them, into ``out`` (as many tensors of the same
    shapes and dtypes) or in place; no output overlaps another gradient or output, so that a tensor is not there twice in place.  Returns the norm before it, on the
    GPU (float64 where a gradient is, else float32); where it is not finite the gradients are passed on unchanged."""
    if _host is not None and workspace is None:
        r = _host.clip_gradients(grads, max_norm, out)
        if r is not None:
            return r
    grads = list(grads)
    outs = grads if out is None else list(out)
    if not grads:
        raise LaError("no gradients")
    if len(outs) != len(grads):
        raise LaError("out: as many tensors as gradients are wanted")
    first = grads[0]
    if not first.is_cuda:
        raise LaError("tensors must be on the GPU")
    count = len(grads)
    for x, y in zip(grads, outs):
        if x.device != first.device or not x.is_contiguous():
            raise LaError("gradients must be contiguous and on the same GPU")
        _layer_dt(x)
        if y is not x:
            _shape("out", y, x.shape)
            _on_gpu(first.device, x.dtype, out=y)
    types = (ctypes.c_int * count)(*[_LAYER_TYPES[x.dtype] for x in grads])
    sizes = (ctypes.c_int64 * count)(*[x.numel() for x in grads])
    src = (ctypes.c_void_p * count)(*[x.data_ptr() for x in grads])
    dst = src if out is None else (ctypes.c_void_p * count)(*[y.data_ptr() for y in outs])
    wide = any(x.dtype == torch.float64 for x in grads)
    norm = torch.empty((), dtype=torch.float64 if wide else torch.float32, device=first.device)
    lib = load()
    with _on_device(first):
        buf, wp, wb = _scratch(workspace, int(lib.la_clip_gradients_workspace_bytes(count, sizes)), first)
        _check(lib.la_clip_gradients(count, types, sizes, src, dst, float(max_norm), int(wide), _ptr(norm), wp, wb, _stream(first)),
               "la_clip_gradients")
    _written(*outs)
    return norm

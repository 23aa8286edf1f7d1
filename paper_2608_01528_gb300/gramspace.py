"""Thin Python binding of libgramspace.so (include/gramspace.h).

Argument marshalling only: tensors are passed to the C ABI as raw device
pointers, outputs are allocated with torch (device memory and streams are
PyTorch's plumbing), and every step of the computation runs in the library's
CUDA kernels.  There is no CPU fallback: if the library is not built, or no
sm_103 device is present, calls raise.

Names follow the C ABI (gs_ prefix dropped): build_basis, build_basis_grouped,
basis_groups, import_basis, project_similarity, project_similarity_host (with
reserve_staging), project_similarity_static, similarity_coeffs, group_argmax,
prob_vectorize, reconstruct, reconstruct_bind, bind, attention_scores,
cross_attention, cross_attention_backward, window_attention,
window_attention_backward, page_slots, page_store, paged_attention, sample_scores,
verify_drafts, stream_status, selftest_wait_timeout.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import warnings

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_build", "libgramspace.so")

GS_OK, GS_ERR_INVALID_ARG, GS_ERR_ALIGNMENT, GS_ERR_SHAPE, GS_ERR_NOMEM = 0, 1, 2, 3, 4
GS_ERR_CUDA, GS_ERR_TIMEOUT, GS_ERR_RANGE, GS_ERR_UNSUPPORTED = 5, 6, 7, 8
GS_F32, GS_BF16 = 0, 1
MODES = {"raw": 0, "cosine": 1, "softmax": 2}
PATHS = {"auto": 0, "simt": 1, "tensor": 2}
GS_BUILD_NORMALIZE_ROWS = 1

# Every symbol include/gramspace.h declares (checked by the CPU tests).
EXPORTS = ("gs_build_basis", "gs_basis_info", "gs_basis_destroy", "gs_project_similarity",
           "gs_prob_vectorize", "gs_reconstruct", "gs_attention_scores", "gs_stream_status",
           "gs_status_string", "gs_version", "gs_project_similarity_static", "gs_similarity_coeffs",
           "gs_selftest_wait_timeout", "gs_basis_import", "gs_basis_reserve_staging",
           "gs_project_similarity_host", "gs_build_basis_grouped", "gs_basis_groups", "gs_group_argmax",
           "gs_bind", "gs_reconstruct_bind", "gs_cross_attention_workspace", "gs_cross_attention",
           "gs_cross_attention_backward", "gs_sample_scores", "gs_window_attention_workspace", "gs_window_attention",
           "gs_window_attention_backward", "gs_page_slots", "gs_page_store", "gs_paged_attention_workspace",
           "gs_paged_attention", "gs_verify_drafts")


class GramSpaceError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Heads(ctypes.Structure):  # gs_heads
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_longlong), ("row", ctypes.c_longlong),
                ("head", ctypes.c_longlong)]


class _Attn(ctypes.Structure):  # gs_attn
    _fields_ = [("dtype", ctypes.c_int), ("B", ctypes.c_int), ("Lq", ctypes.c_int), ("Lk", ctypes.c_int),
                ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int), ("dk", ctypes.c_int), ("dv", ctypes.c_int),
                ("scale", ctypes.c_float), ("key_lens", ctypes.c_void_p), ("key_mask", ctypes.c_void_p),
                ("ld_mask", ctypes.c_longlong), ("flags", ctypes.c_uint)]


class _Window(ctypes.Structure):  # gs_window
    _fields_ = [("window", ctypes.c_int), ("sinks", ctypes.c_int), ("start", ctypes.c_int), ("starts", ctypes.c_void_p)]


class _Paged(ctypes.Structure):  # gs_paged
    _fields_ = [("dtype", ctypes.c_int), ("B", ctypes.c_int), ("Lq", ctypes.c_int), ("Hq", ctypes.c_int),
                ("Hkv", ctypes.c_int), ("dk", ctypes.c_int), ("dv", ctypes.c_int), ("scale", ctypes.c_float),
                ("pages", ctypes.c_int), ("page_size", ctypes.c_int), ("columns", ctypes.c_int), ("table", ctypes.c_void_p),
                ("ld_table", ctypes.c_longlong), ("lens", ctypes.c_void_p), ("q_lens", ctypes.c_void_p),
                ("window", ctypes.c_int), ("sinks", ctypes.c_int), ("flags", ctypes.c_uint)]


class _Sampling(ctypes.Structure):  # gs_sampling
    _fields_ = [("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("top_k", ctypes.c_int), ("temperature_rows", ctypes.c_void_p), ("top_p_rows", ctypes.c_void_p),
                ("min_p_rows", ctypes.c_void_p), ("top_k_rows", ctypes.c_void_p)]


_lib = None


def load_library(path=LIB_PATH):
    """Loads (once) and returns the ctypes handle of libgramspace.so."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libgramspace.so is not built ({path}); run __graft_entry__.build()")
    L = ctypes.CDLL(path)
    vp, ip, i64, f32, u32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_uint
    L.gs_build_basis.argtypes = [vp, ip, ip, ip, f32, u32, vp, ctypes.POINTER(vp)]
    L.gs_basis_info.argtypes = [vp, ctypes.POINTER(ip), ctypes.POINTER(ip), ctypes.POINTER(ip),
                                ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
    L.gs_basis_destroy.argtypes = [vp]
    L.gs_basis_reserve_staging.argtypes = [vp, i64]
    L.gs_project_similarity_host.argtypes = [vp, vp, i64, ip, ip, f32, u32, vp, vp, vp]
    L.gs_basis_import.argtypes = [vp, ip, ip, ip, vp, ip, ip, vp, vp, ctypes.POINTER(vp)]
    L.gs_build_basis_grouped.argtypes = [vp, ip, ip, ip, vp, ip, f32, u32, vp, ctypes.POINTER(vp)]
    L.gs_basis_groups.argtypes = [vp, ctypes.POINTER(ip), vp, vp]
    L.gs_group_argmax.argtypes = [vp, i64, ip, vp, ip, vp, vp, vp]
    L.gs_bind.argtypes = [vp, i64, ip, ip, vp, i64, ip, ip, vp, ip, vp]
    L.gs_reconstruct_bind.argtypes = [vp, vp, ip, i64, ip, vp, i64, ip, ip, vp, ip, u32, vp]
    L.gs_project_similarity.argtypes = [vp, vp, i64, ip, ip, f32, u32, vp, ip, vp, ip, vp, vp, vp]
    L.gs_similarity_coeffs.argtypes = [vp, vp, i64, ip, ip, f32, u32, vp, ip, vp, vp, vp]
    L.gs_prob_vectorize.argtypes = [vp, vp, i64, ip, vp, ip, ip, u32, vp]
    L.gs_reconstruct.argtypes = [vp, vp, ip, i64, ip, vp, ip, u32, vp]
    L.gs_attention_scores.argtypes = [vp, vp, ip, ip, ip, ip, ip, ip, f32, ip, vp, u32, vp]
    hp, ap = ctypes.POINTER(_Heads), ctypes.POINTER(_Attn)
    L.gs_cross_attention_workspace.argtypes = [ap, ip, ctypes.POINTER(i64)]
    L.gs_cross_attention.argtypes = [ap, hp, hp, hp, hp, vp, vp, i64, vp]
    L.gs_cross_attention_backward.argtypes = [ap, hp, hp, hp, hp, vp, hp, hp, hp, hp, vp, i64, vp]
    wp, pp = ctypes.POINTER(_Window), ctypes.POINTER(_Paged)
    L.gs_window_attention_workspace.argtypes = [ap, wp, ip, ctypes.POINTER(i64)]
    L.gs_window_attention.argtypes = [ap, wp, hp, hp, hp, hp, vp, vp, i64, vp]
    L.gs_window_attention_backward.argtypes = [ap, wp, hp, hp, hp, hp, vp, hp, hp, hp, hp, vp, i64, vp]
    L.gs_page_slots.argtypes = [vp, vp, ip, ip, ip, ip, vp, ip, vp, vp, i64, ip, vp, vp, vp, vp]
    L.gs_page_store.argtypes = [ip, ip, ip, ip, ip, ip, hp, hp, vp, i64, ip, ip, hp, hp, vp]
    L.gs_paged_attention_workspace.argtypes = [pp, ctypes.POINTER(i64)]
    L.gs_paged_attention.argtypes = [pp, hp, hp, hp, hp, vp, vp, i64, vp]
    L.gs_verify_drafts.argtypes = [vp, vp, ip, ip, ip, ip, i64, i64, i64, i64, vp, vp, vp, vp, vp, vp]
    L.gs_sample_scores.argtypes = [vp, ip, i64, ip, i64, ctypes.POINTER(_Sampling), vp, vp, vp, vp]
    L.gs_stream_status.argtypes = [vp]
    L.gs_selftest_wait_timeout.argtypes = [vp]
    L.gs_project_similarity_static.argtypes = [vp, ip, ip, vp, ip, vp, vp, i64, ip, ip, f32, vp, vp, vp]
    L.gs_project_similarity_static.restype = ctypes.c_int
    L.gs_status_string.argtypes = [ip]
    L.gs_status_string.restype = ctypes.c_char_p
    L.gs_version.restype = ctypes.c_int
    for name in ("gs_build_basis", "gs_basis_info", "gs_basis_destroy", "gs_project_similarity",
                 "gs_similarity_coeffs", "gs_prob_vectorize", "gs_reconstruct", "gs_attention_scores",
                 "gs_stream_status", "gs_selftest_wait_timeout", "gs_basis_import",
                 "gs_basis_reserve_staging", "gs_project_similarity_host", "gs_build_basis_grouped",
                 "gs_basis_groups", "gs_group_argmax", "gs_bind", "gs_reconstruct_bind",
                 "gs_cross_attention_workspace", "gs_cross_attention", "gs_cross_attention_backward",
                 "gs_sample_scores", "gs_window_attention_workspace", "gs_window_attention",
                 "gs_window_attention_backward", "gs_page_slots", "gs_page_store", "gs_paged_attention_workspace",
                 "gs_paged_attention", "gs_verify_drafts"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def status_string(status):
    return load_library().gs_status_string(int(status)).decode()


def _check(status, where):
    if status != GS_OK:
        raise GramSpaceError(status, where)


# A small call is mostly its host time, so the helpers below take the shortest way that torch offers:
# plain integers for the pointer arguments (ctypes converts them itself), the raw stream handle (a
# Stream object costs more than the launch), and no device switch when the device is current already.
# A 1,024-query similarity_coeffs went from 16.5 to 11 us a call, of which the kernel takes 5.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)
_STAY = contextlib.nullcontext()


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stream(stream, device=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and device is not None and device.type == "cuda" and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _on(device):
    """torch.cuda.device(device), or nothing to do when it is the current device."""
    if _get_device is not None and device.type == "cuda" and device.index is not None and torch.cuda.is_initialized() \
            and _get_device() == device.index:
        return _STAY
    return torch.cuda.device(device)


def _ld(t):
    st = t.stride()
    if len(st) != 2 or st[1] != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    return st[0]


def _dtype_code(t):
    if t.dtype == torch.float32:
        return GS_F32
    if t.dtype == torch.bfloat16:
        return GS_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


class _DevArray:
    """__cuda_array_interface__ view of memory owned by a basis handle."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr,
                                         "data": (int(ptr or 0), False), "version": 3, "strides": None}


class Basis:
    """A built Gram-Space basis (owns the C handle): Q (r x D), R (M x r), cnorm (M)."""

    def __init__(self, handle, device):
        self._h = handle
        self.device = device
        L = load_library()
        M, D, r = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        q, rr, cn = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        _check(L.gs_basis_info(handle, ctypes.byref(M), ctypes.byref(D), ctypes.byref(r), ctypes.byref(q),
                               ctypes.byref(rr), ctypes.byref(cn)), "gs_basis_info")
        self.M, self.D, self.r = M.value, D.value, r.value
        self._q, self._R, self._cn = q.value, rr.value, cn.value

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("basis already destroyed")
        return self._h

    def _view(self, ptr, shape):
        if 0 in shape:
            return torch.zeros(shape, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            return torch.as_tensor(_DevArray(ptr, shape, "<f4"), device=self.device)

    @property
    def Q(self):
        return self._view(self._q, (self.r, self.D))

    @property
    def R(self):
        return self._view(self._R, (self.M, self.r))

    @property
    def cnorm(self):
        return self._view(self._cn, (self.M,))

    def destroy(self):
        if self._h is not None:
            load_library().gs_basis_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def build_basis(C, rank_tol=1e-6, normalize_rows=False, stream=None):
    """Gram-Schmidt basis of the rows of C (M x D fp32 on the GPU); see gs_build_basis."""
    if not C.is_cuda or C.dtype != torch.float32:
        raise TypeError("C must be a float32 CUDA tensor")
    L = load_library()
    h = ctypes.c_void_p()
    with _on(C.device):
        st = L.gs_build_basis(_ptr(C), C.shape[0], C.shape[1], _ld(C), float(rank_tol),
                              GS_BUILD_NORMALIZE_ROWS if normalize_rows else 0, _stream(stream, C.device),
                              ctypes.byref(h))
    _check(st, "gs_build_basis")
    return Basis(h, C.device)


def _offsets(group_offsets):
    off = [int(o) for o in group_offsets]
    return (ctypes.c_int * len(off))(*off), len(off) - 1


def build_basis_grouped(C, group_offsets, rank_tol=1e-6, normalize_rows=False, stream=None):
    """One Gram-Schmidt basis per group of rows of C (rows [off[g], off[g+1])), stacked in one
    handle; see gs_build_basis_grouped."""
    if not C.is_cuda or C.dtype != torch.float32:
        raise TypeError("C must be a float32 CUDA tensor")
    off, G = _offsets(group_offsets)
    L = load_library()
    h = ctypes.c_void_p()
    with _on(C.device):
        st = L.gs_build_basis_grouped(_ptr(C), C.shape[0], C.shape[1], _ld(C), off, G, float(rank_tol),
                                      GS_BUILD_NORMALIZE_ROWS if normalize_rows else 0, _stream(stream, C.device),
                                      ctypes.byref(h))
    _check(st, "gs_build_basis_grouped")
    return Basis(h, C.device)


def basis_groups(basis):
    """(row_offsets, coeff_offsets) of the basis' groups; see gs_basis_groups."""
    L = load_library()
    G = ctypes.c_int()
    _check(L.gs_basis_groups(basis.handle, ctypes.byref(G), None, None), "gs_basis_groups")
    rows = (ctypes.c_int * (G.value + 1))()
    coeffs = (ctypes.c_int * (G.value + 1))()
    _check(L.gs_basis_groups(basis.handle, ctypes.byref(G), rows, coeffs), "gs_basis_groups")
    return list(rows), list(coeffs)


def group_argmax(S, group_offsets, want_maxval=True, out=None, stream=None):
    """Per-row, per-group argmax (index within the group) and max of scores S (N x M fp32, CUDA);
    see gs_group_argmax.  Returns {"argmax": N x G int32, "maxval": N x G fp32}."""
    if not S.is_cuda or S.dtype != torch.float32:
        raise TypeError("S must be a float32 CUDA tensor")
    off, G = _offsets(group_offsets)
    N = S.shape[0]
    out = dict(out or {})
    if "argmax" not in out:
        out["argmax"] = torch.empty((N, G), dtype=torch.int32, device=S.device)
    if want_maxval and "maxval" not in out:
        out["maxval"] = torch.empty((N, G), dtype=torch.float32, device=S.device)
    L = load_library()
    with _on(S.device):
        st = L.gs_group_argmax(_ptr(S), N, _ld(S) if N else S.shape[1], off, G, _ptr(out.get("argmax")),
                               _ptr(out.get("maxval")), _stream(stream, S.device))
    _check(st, "gs_group_argmax")
    return out


def import_basis(Q, R, cnorm=None, stream=None):
    """Restore a basis saved from Basis.Q / Basis.R / Basis.cnorm (fp32 CUDA tensors, Q: r x D,
    R: M x r); see gs_basis_import.  The restored basis gives bit-identical results."""
    for t in (Q, R) + ((cnorm,) if cnorm is not None else ()):
        if not t.is_cuda or t.dtype != torch.float32:
            raise TypeError("Q, R and cnorm must be float32 CUDA tensors")
    r, D = Q.shape
    M = R.shape[0]
    L = load_library()
    h = ctypes.c_void_p()
    with _on(R.device):
        st = L.gs_basis_import(_ptr(Q) if r else None, r, D, _ld(Q) if r else D, _ptr(R) if r else None, M,
                               _ld(R) if r else 1, _ptr(cnorm), _stream(stream, R.device), ctypes.byref(h))
    _check(st, "gs_basis_import")
    return Basis(h, R.device)


def reserve_staging(basis, rows):
    """Device staging for project_similarity_host (rows queries); see gs_basis_reserve_staging."""
    L = load_library()
    with _on(basis.device):
        _check(L.gs_basis_reserve_staging(basis.handle, int(rows)), "gs_basis_reserve_staging")


def project_similarity_host(basis, X, mode="raw", scale=1.0, path="auto", want_argmax=True, want_maxval=True,
                            out=None, stream=None):
    """Project + similarity of host queries X (N x D float32 CPU tensor, ideally pinned) into host
    outputs; see gs_project_similarity_host.  Asynchronous on `stream`: synchronise before reading
    the outputs, and keep X referenced (and unchanged) until then -- a pinned tensor freed earlier
    returns its block to torch's host allocator, which can reuse it while the copy is queued."""
    if X.is_cuda or X.dtype != torch.float32:
        raise TypeError("X must be a float32 CPU tensor")
    if X.dim() != 2 or X.shape[1] != basis.D:
        raise ValueError(f"X must be N x {basis.D}")
    N = X.shape[0]
    out = dict(out or {})
    pin = X.is_pinned()
    if want_argmax and "argmax" not in out:
        out["argmax"] = torch.empty(N, dtype=torch.int32, pin_memory=pin)
    if want_maxval and "maxval" not in out:
        out["maxval"] = torch.empty(N, dtype=torch.float32, pin_memory=pin)
    L = load_library()
    with _on(basis.device):
        st = L.gs_project_similarity_host(basis.handle, _ptr(X), N, _ld(X), MODES[mode], float(scale),
                                          PATHS[path], _ptr(out.get("argmax")), _ptr(out.get("maxval")),
                                          _stream(stream, basis.device))
    _check(st, "gs_project_similarity_host")
    return out


def project_similarity(basis, X, mode="raw", scale=1.0, path="auto", want_Y=False, want_S=False,
                       want_argmax=True, want_maxval=True, out=None, stream=None):
    """Fused Y = X Q^T and scores against the codebook in Gram-loc; see gs_project_similarity.

    Returns a dict with the requested outputs ("Y", "S", "argmax", "maxval").
    `out` may supply preallocated output tensors under the same keys.
    """
    N = X.shape[0]
    dev = X.device
    out = dict(out or {})
    if want_Y and "Y" not in out:
        out["Y"] = torch.empty((N, basis.r), dtype=torch.float32, device=dev)
    if want_S and "S" not in out:
        out["S"] = torch.empty((N, basis.M), dtype=torch.float32, device=dev)
    if want_argmax and "argmax" not in out:
        out["argmax"] = torch.empty(N, dtype=torch.int32, device=dev)
    if want_maxval and "maxval" not in out:
        out["maxval"] = torch.empty(N, dtype=torch.float32, device=dev)
    Y, S = out.get("Y"), out.get("S")
    L = load_library()
    # the handle's calls switch to the basis' device themselves: only the stream is looked up here
    st = L.gs_project_similarity(basis.handle, _ptr(X), N, _ld(X), MODES[mode], float(scale), PATHS[path],
                                 _ptr(Y), _ld(Y) if Y is not None and Y.numel() else max(basis.r, 1),
                                 _ptr(S), _ld(S) if S is not None and S.numel() else max(basis.M, 1),
                                 _ptr(out.get("argmax")), _ptr(out.get("maxval")), _stream(stream, dev))
    _check(st, "gs_project_similarity")
    return out


def similarity_coeffs(basis, Y, mode="raw", scale=1.0, path="auto", want_S=False, want_argmax=True,
                      want_maxval=True, out=None, stream=None):
    """Scores of Gram-loc queries Y (N x r fp32) against the codebook, S = Y R^T; see
    gs_similarity_coeffs.  Returns a dict with the requested outputs ("S", "argmax", "maxval")."""
    N = Y.shape[0]
    dev = Y.device
    out = dict(out or {})
    if want_S and "S" not in out:
        out["S"] = torch.empty((N, basis.M), dtype=torch.float32, device=dev)
    if want_argmax and "argmax" not in out:
        out["argmax"] = torch.empty(N, dtype=torch.int32, device=dev)
    if want_maxval and "maxval" not in out:
        out["maxval"] = torch.empty(N, dtype=torch.float32, device=dev)
    S = out.get("S")
    L = load_library()
    st = L.gs_similarity_coeffs(basis.handle, _ptr(Y) if Y.numel() else None, N,
                                _ld(Y) if Y.numel() else max(basis.r, 1), MODES[mode], float(scale),
                                PATHS[path], _ptr(S), _ld(S) if S is not None and S.numel() else max(basis.M, 1),
                                _ptr(out.get("argmax")), _ptr(out.get("maxval")), _stream(stream, dev))
    _check(st, "gs_similarity_coeffs")
    return out


def prob_vectorize(basis, P, dtype=torch.float32, path="auto", out=None, stream=None):
    """V = P R (Gram-loc of P C); see gs_prob_vectorize."""
    N = P.shape[0]
    V = out if out is not None else torch.empty((N, basis.r), dtype=dtype, device=P.device)
    L = load_library()
    with _on(P.device):
        st = L.gs_prob_vectorize(basis.handle, _ptr(P), N, _ld(P), _ptr(V), _dtype_code(V),
                                 _ld(V) if V.numel() else max(basis.r, 1), PATHS[path], _stream(stream, P.device))
    _check(st, "gs_prob_vectorize")
    return V


def reconstruct(basis, T, path="auto", out=None, stream=None):
    """Xhat = T Q (x = U t); see gs_reconstruct."""
    N = T.shape[0]
    X = out if out is not None else torch.empty((N, basis.D), dtype=torch.float32, device=T.device)
    L = load_library()
    with _on(T.device):
        st = L.gs_reconstruct(basis.handle, _ptr(T), _dtype_code(T), N, _ld(T) if T.numel() else max(basis.r, 1),
                              _ptr(X), _ld(X), PATHS[path], _stream(stream, T.device))
    _check(st, "gs_reconstruct")
    return X


BIND_OPS = {"bind": 0, "unbind": 1}
BIND_METHODS = {"auto": 0, "direct": 2, "spectral": 4}


def _partner(Y, N, D):
    if not Y.is_cuda or Y.dtype != torch.float32 or Y.dim() != 2 or Y.shape[1] != D:
        raise ValueError(f"Y must be a float32 CUDA tensor with {D} columns")
    if Y.shape[0] == 1 and N != 1:
        return 0  # one partner for every row
    if Y.shape[0] != N:
        raise ValueError("Y must have one row or one row per input row")
    return _ld(Y)


def bind(X, Y, L, op="bind", method="auto", out=None, stream=None):
    """Block circular convolution (op="bind") or correlation ("unbind") of the rows of X with
    those of Y (or with Y's single row), blocks of L; method "direct" (the sum per output),
    "spectral" (block transforms) or "auto"; see gs_bind."""
    N, D = X.shape
    ldy = _partner(Y, N, D)
    Z = out if out is not None else torch.empty((N, D), dtype=torch.float32, device=X.device)
    L_ = load_library()
    with _on(X.device):
        st = L_.gs_bind(_ptr(X), N, D, _ld(X) if N else D, _ptr(Y), ldy, int(L), BIND_OPS[op] | BIND_METHODS[method],
                        _ptr(Z), _ld(Z) if N else D, _stream(stream, X.device))
    _check(st, "gs_bind")
    return Z


def reconstruct_bind(basis, T, Y, L, op="bind", path="auto", method="auto", out=None, stream=None):
    """op(T Q, Y): reconstruction then binding, chunk by chunk through the basis' scratch; see gs_reconstruct_bind
    (path: the reconstruction's kernels, method: the binding's, as in bind)."""
    N = T.shape[0]
    ldy = _partner(Y, N, basis.D)
    Z = out if out is not None else torch.empty((N, basis.D), dtype=torch.float32, device=T.device)
    L_ = load_library()
    with _on(basis.device):
        st = L_.gs_reconstruct_bind(basis.handle, _ptr(T), _dtype_code(T), N, _ld(T) if N else basis.r, _ptr(Y),
                                    ldy, int(L), BIND_OPS[op] | BIND_METHODS[method], _ptr(Z),
                                    _ld(Z) if N else basis.D, PATHS[path], _stream(stream, basis.device))
    _check(st, "gs_reconstruct_bind")
    return Z


def attention_scores(Yq, Yk, scale, apply_softmax=True, path="auto", out=None, stream=None):
    """softmax_row(scale * Yq Yk^T) per sequence; Yq: B x Lq x r, Yk: B x Lk x r."""
    B, Lq, r = Yq.shape
    Lk = Yk.shape[1]
    if Yk.shape[0] != B or Yk.shape[2] != r or Yq.dtype != Yk.dtype:
        raise ValueError("Yq and Yk must agree in batch, width and dtype")
    if not (Yq.is_contiguous() and Yk.is_contiguous()):
        raise ValueError("Yq and Yk must be contiguous (row stride r)")
    A = out if out is not None else torch.empty((B, Lq, Lk), dtype=torch.float32, device=Yq.device)
    L = load_library()
    with _on(Yq.device):
        st = L.gs_attention_scores(_ptr(Yq), _ptr(Yk), _dtype_code(Yq), B, Lq, Lk, r, max(r, 1), float(scale),
                                   1 if apply_softmax else 0, _ptr(A), PATHS[path], _stream(stream, Yq.device))
    _check(st, "gs_attention_scores")
    return A


def _on_stream(device, stream):
    """The context of a call that runs on `stream`, or nothing to do.  The call's device is current in it, and so is its
    stream: memory from torch's allocator belongs to the stream that is current when it is taken, so outputs and
    workspaces are taken under the stream that writes them."""
    if stream is None:
        return _on(device)
    if stream.device != device:
        raise ValueError(f"the tensors are on {device}, the stream on {stream.device}")
    return torch.cuda.stream(stream)


def _c_int(*sizes):
    """Refuses sizes that a C int does not hold (ctypes would cut them)."""
    if max(sizes) > 0x7fffffff:
        raise ValueError(f"sizes above 2^31 - 1: {sizes}")


def _heads(t, name, shape, like):
    """gs_heads of a B x L x H x w tensor with a dense last axis."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {' x '.join(map(str, shape))}, got {tuple(t.shape)}")
    if t.dtype is not like.dtype or t.device != like.device:
        raise TypeError(f"{name} must be {like.dtype} on {like.device}, got {t.dtype} on {t.device}")
    s = t.stride()
    if s[3] != 1 and shape[3] > 1:
        raise ValueError(f"{name} must have unit stride along its last axis")
    return _Heads(t.data_ptr(), s[0], s[1], s[2])


def _attn(Q, K, V, scale, key_lens, key_mask, path):
    """gs_attn and the gs_heads of the inputs, after the checks that need no device."""
    if Q.dim() != 4 or K.dim() != 4 or V.dim() != 4:
        raise ValueError("Q, K and V must be 4-D (batch, length, heads, width)")
    code = _dtype_code(Q)
    B, Lq, Hq, dk = Q.shape
    _, Lk, Hkv, dv = V.shape
    _c_int(B, Lq, Lk, Hq, Hkv, dk, dv)
    hs = (_heads(Q, "Q", Q.shape, Q), _heads(K, "K", (B, Lk, Hkv, dk), Q), _heads(V, "V", (B, Lk, Hkv, dv), Q))
    if scale is None:
        scale = dk ** -0.5 if dk else 1.0
    a = _Attn(code, B, Lq, Lk, Hq, Hkv, dk, dv, scale, None, None, 0, PATHS[path])
    if key_lens is not None:
        if key_lens.dtype is not torch.int32 or key_lens.shape != (B,) or not key_lens.is_contiguous():
            raise ValueError(f"key_lens must be a contiguous int32 vector of {B} lengths")
        if key_lens.device != Q.device:
            raise TypeError(f"key_lens must be on {Q.device}")
        a.key_lens = key_lens.data_ptr()
    if key_mask is not None:
        if key_mask.dtype not in (torch.bool, torch.uint8) or key_mask.shape != (B, Lk) \
                or (Lk > 1 and key_mask.stride(1) != 1):
            raise ValueError(f"key_mask must be a {B} x {Lk} bool (or uint8) tensor with unit column stride")
        if key_mask.device != Q.device:
            raise TypeError(f"key_mask must be on {Q.device}")
        a.key_mask = key_mask.data_ptr()
        a.ld_mask = key_mask.stride(0) if B > 1 else Lk
    if not Q.is_cuda:
        raise TypeError("Q, K and V must be CUDA tensors")
    return a, hs


def _attn_workspace(L, a, backward, device, w=None):
    """(tensor to keep until the call has been made, its address, its bytes)"""
    n = ctypes.c_longlong()
    if w is None:
        _check(L.gs_cross_attention_workspace(ctypes.byref(a), backward, ctypes.byref(n)), "gs_cross_attention_workspace")
    else:
        _check(L.gs_window_attention_workspace(ctypes.byref(a), ctypes.byref(w), backward, ctypes.byref(n)),
               "gs_window_attention_workspace")
    if n.value == 0:
        return None, None, 0
    ws = torch.empty(n.value, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), n.value


def _attn_lse(lse, shape, device):
    if lse.dtype is not torch.float32 or lse.shape != shape or not lse.is_contiguous() or lse.device != device:
        raise ValueError(f"lse must be a contiguous float32 {' x '.join(map(str, shape))} tensor on {device}")
    return lse.data_ptr()


def cross_attention(Q, K, V, scale=None, key_lens=None, key_mask=None, want_lse=False, path="auto", out=None,
                    stream=None):
    """softmax(scale * Q K^T over the valid keys) V per head; see gs_cross_attention.

    Q: B x Lq x Hq x dk, K: B x Lk x Hkv x dk, V: B x Lk x Hkv x dv (float32 or bfloat16, any
    strides with a dense last axis; Hkv divides Hq, head h reads key head h // (Hq // Hkv)).
    scale: dk ** -0.5 by default.  key_lens: int32 [B], keys to read of each sequence.  key_mask:
    bool B x Lk, False = not read.  Returns {"O": B x Lq x Hq x dv, "lse": B x Hq x Lq float32 with want_lse};
    `out` may supply them.  Like every call of this module it is not recorded by autograd: a graph's backward step calls
    cross_attention_backward (there is a warning where an input asks for its gradient)."""
    _warn_unrecorded("cross_attention", Q, K, V)
    a, hs = _attn(Q, K, V, scale, key_lens, key_mask, path)
    return _forward(a, hs, Q, want_lse, out, stream)


def _warn_unrecorded(name, *inputs):
    if torch.is_grad_enabled() and any(t.requires_grad for t in inputs):
        warnings.warn(f"{name} is not recorded by autograd, gradients do not pass through it: take them from "
                      f"{name}_backward, and call it under torch.no_grad() or on detached tensors", stacklevel=3)


def _forward(a, hs, Q, want_lse, out, stream, w=None):
    """cross_attention, or through a window window_attention."""
    L, dev, ref = load_library(), Q.device, ctypes.byref
    out = dict(out) if out else {}
    with _on_stream(dev, stream):
        if "O" not in out:
            out["O"] = torch.empty((a.B, a.Lq, a.Hq, a.dv), dtype=Q.dtype, device=dev)
        if want_lse and out.get("lse") is None:
            out["lse"] = torch.empty((a.B, a.Hq, a.Lq), dtype=torch.float32, device=dev)
        o = _heads(out["O"], "O", (a.B, a.Lq, a.Hq, a.dv), Q)
        lse = _attn_lse(out["lse"], (a.B, a.Hq, a.Lq), dev) if out.get("lse") is not None else None
        keep, ws, size = _attn_workspace(L, a, 0, dev, w)
        rest = (ref(hs[0]), ref(hs[1]), ref(hs[2]), ref(o), lse, ws, size, _stream(stream, dev))
        st = L.gs_cross_attention(ref(a), *rest) if w is None else L.gs_window_attention(ref(a), ref(w), *rest)
    _check(st, "gs_cross_attention" if w is None else "gs_window_attention")
    return out


def cross_attention_backward(Q, K, V, O, lse, dO, scale=None, key_lens=None, key_mask=None, path="auto", out=None,
                             stream=None):
    """The gradient of cross_attention; see gs_cross_attention_backward.  O and lse are the forward
    call's (want_lse=True), dO the gradient of O; the other arguments as there.  Returns {"dQ", "dK", "dV"} with
    the shapes and type of Q, K and V; `out` may supply them."""
    a, hs = _attn(Q, K, V, scale, key_lens, key_mask, path)
    return _backward(a, hs, Q, K, V, O, lse, dO, out, stream)


def _backward(a, hs, Q, K, V, O, lse, dO, out, stream, w=None):
    """cross_attention_backward, or through a window window_attention_backward."""
    L, dev, ref = load_library(), Q.device, ctypes.byref
    out = dict(out) if out else {}
    shape = (a.B, a.Lq, a.Hq, a.dv)
    o, do = _heads(O, "O", shape, Q), _heads(dO, "dO", shape, Q)
    logs = _attn_lse(lse, (a.B, a.Hq, a.Lq), dev)  # (the tensor stays in its name: its last reference may be this call's)
    with _on_stream(dev, stream):
        for name, t in (("dQ", Q), ("dK", K), ("dV", V)):
            if name not in out:
                out[name] = torch.empty(t.shape, dtype=t.dtype, device=dev)
        gq, gk, gv = _heads(out["dQ"], "dQ", Q.shape, Q), _heads(out["dK"], "dK", K.shape, Q), _heads(out["dV"], "dV", V.shape, Q)
        keep, ws, size = _attn_workspace(L, a, 1, dev, w)
        rest = (ref(hs[0]), ref(hs[1]), ref(hs[2]), ref(o), logs, ref(do), ref(gq), ref(gk), ref(gv), ws, size, _stream(stream, dev))
        st = L.gs_cross_attention_backward(ref(a), *rest) if w is None else L.gs_window_attention_backward(ref(a), ref(w), *rest)
    _check(st, "gs_cross_attention_backward" if w is None else "gs_window_attention_backward")
    return out


def _window(window, sinks, start, B, device):
    """gs_window; start is a number or an int32 vector of B."""
    window = 0x7fffffff if window is None else int(window)
    if window < 1 or int(sinks) < 0:
        raise ValueError(f"window must be at least 1 and sinks at least 0, got {window} and {sinks}")
    w = _Window(min(window, 0x7fffffff), min(int(sinks), 0x7fffffff), 0, None)
    if isinstance(start, torch.Tensor):
        w.starts = _int_vector(start, "start", B, device)
    else:
        if abs(int(start)) > 0x7fffffff:
            raise ValueError(f"start is no 32-bit position: {start}")
        w.start = int(start)
    return w


def _int_vector(t, name, n, device):
    if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 vector of {n}")
    if t.device != device:
        raise TypeError(f"{name} must be on {device}")
    return t.data_ptr()


def window_attention(Q, K, V, window, sinks=0, start=0, scale=None, key_lens=None, key_mask=None, want_lse=False, path="auto",
                     out=None, stream=None):
    """Causal attention over a sliding window; see gs_window_attention.

    As cross_attention, where query row i stands at position start + i (start: a number, or an int32 CUDA vector with one per
    sequence) and sees the keys up to it, the last `window` of them (None: all) and the first `sinks`."""
    _warn_unrecorded("window_attention", Q, K, V)
    a, hs = _attn(Q, K, V, scale, key_lens, key_mask, path)
    return _forward(a, hs, Q, want_lse, out, stream, _window(window, sinks, start, a.B, Q.device))


def window_attention_backward(Q, K, V, O, lse, dO, window, sinks=0, start=0, scale=None, key_lens=None, key_mask=None,
                              path="auto", out=None, stream=None):
    """The gradient of window_attention, as cross_attention_backward is of cross_attention; see
    gs_window_attention_backward."""
    a, hs = _attn(Q, K, V, scale, key_lens, key_mask, path)
    return _backward(a, hs, Q, K, V, O, lse, dO, out, stream, _window(window, sinks, start, a.B, Q.device))


def _table(table, device):
    """(address, requests, columns, row stride) of a block table."""
    if table.dim() != 2 or table.dtype is not torch.int32 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be a 2-D int32 tensor (requests x columns) with unit column stride")
    if table.device != device:
        raise TypeError(f"table must be on {device}")
    B, columns = table.shape
    _c_int(B, columns)
    return table.data_ptr(), B, columns, table.stride(0) if B > 1 else columns


def page_slots(lens, added, table, free, page_size, max_new, pages, free_from=None, want_lens=True, want_taken=True, out=None,
               stream=None):
    """Slots of new tokens in a paged cache; see gs_page_slots.

    lens, added: int32 CUDA vectors, tokens that each request holds and gets.  table: int32 requests x columns, the block table,
    whose next columns are filled in place.  free: int32 vector, the free pages, taken from entry free_from (an int32 CUDA
    tensor of one; None: 0) on.  max_new: columns of the result, pages: of the cache.  Returns {"slots": requests x max_new, "lens": the
    requests' new lengths, "taken": pages asked for, one number}, int32.  free_from of the next call is free_from + taken, or the list's
    length where that is less: free_from.add_(taken).clamp_(max=free.numel())."""
    dev = lens.device
    t, B, columns, ld = _table(table, dev)
    _c_int(abs(int(page_size)), abs(int(max_new)), abs(int(pages)), free.numel())
    if int(max_new) < 0:
        raise ValueError(f"max_new must be at least 0, got {max_new}")
    if free.dim() != 1:
        raise ValueError("free must be a vector")
    args = (_int_vector(lens, "lens", B, dev), _int_vector(added, "added", B, dev))
    fr = _int_vector(free, "free", free.shape[0], dev)
    ff = _int_vector(free_from.view(-1), "free_from", 1, dev) if free_from is not None else None
    out = dict(out) if out else {}
    for name, shape in (("slots", (B, max_new)), ("lens", (B,)), ("taken", (1,))):
        x = out.get(name)
        if x is not None and (x.dtype is not torch.int32 or x.shape != shape or not x.is_contiguous() or x.device != dev):
            raise ValueError(f"out[{name!r}] must be a contiguous int32 {' x '.join(map(str, shape))} tensor on {dev}")
    if not lens.is_cuda:
        raise TypeError("lens, added, table and free must be CUDA tensors")
    L = load_library()
    with _on_stream(dev, stream):
        for name, shape, want in (("slots", (B, max_new), True), ("lens", (B,), want_lens), ("taken", (1,), want_taken)):
            if want and out.get(name) is None:
                out[name] = torch.empty(shape, dtype=torch.int32, device=dev)
        st = L.gs_page_slots(*args, B, int(max_new), int(page_size), int(pages), fr, free.shape[0], ff, t, ld, columns,
                             _ptr(out["slots"]), _ptr(out.get("lens")), _ptr(out.get("taken")), _stream(stream, dev))
    _check(st, "gs_page_slots")
    return out


def _cache(Kc, Vc, like):
    """gs_heads of a cache's two arrays, its pages and page size."""
    if Kc.dim() != 4 or Vc.dim() != 4:
        raise ValueError("Kc and Vc must be 4-D (pages, page size, heads, width)")
    pages, size, H, dk = Kc.shape
    _c_int(pages, size, H, dk, Vc.shape[3])
    return _heads(Kc, "Kc", Kc.shape, like), _heads(Vc, "Vc", (pages, size, H, Vc.shape[3]), like), pages, size


def page_store(K, V, slots, Kc, Vc, stream=None):
    """New keys and values (requests x tokens x heads x width) into the slots (int32 requests x tokens, negative: skipped) of the
    cache Kc, Vc (pages x page size x heads x width), in place; see gs_page_store."""
    if K.dim() != 4 or V.dim() != 4:
        raise ValueError("K and V must be 4-D (requests, tokens, heads, width)")
    code = _dtype_code(K)
    kc, vc, pages, size = _cache(Kc, Vc, K)
    B, n, H, dk = K.shape
    dv = Vc.shape[3]
    _c_int(B, n)
    if Kc.shape[2] != H or Kc.shape[3] != dk:
        raise ValueError(f"Kc must hold {H} heads of {dk}, got {Kc.shape[2]} of {Kc.shape[3]}")
    k, v = _heads(K, "K", K.shape, K), _heads(V, "V", (B, n, H, dv), K)
    dev = K.device
    if slots.dtype is not torch.int32 or slots.shape != (B, n) or (n > 1 and slots.stride(1) != 1):
        raise ValueError(f"slots must be an int32 {B} x {n} tensor with unit column stride")
    if slots.device != dev:
        raise TypeError(f"slots must be on {dev}")
    if not K.is_cuda:
        raise TypeError("K, V and the cache must be CUDA tensors")
    L, ref = load_library(), ctypes.byref
    with _on_stream(dev, stream):
        st = L.gs_page_store(code, B, n, H, dk, dv, ref(k), ref(v), slots.data_ptr(), slots.stride(0) if B > 1 else n, pages, size,
                             ref(kc), ref(vc), _stream(stream, dev))
    _check(st, "gs_page_store")


def paged_attention(Q, Kc, Vc, table, lens, scale=None, q_lens=None, window=None, sinks=0, want_lse=False, path="auto", out=None,
                    stream=None):
    """Attention of the requests' newest tokens over a paged cache; see gs_paged_attention.

    Q: B x Lq x Hq x dk, the last q_lens[b] (int32 [B]; None: Lq) tokens of each request, Kc and Vc: the cache (pages x page size x
    Hkv x width), table: int32 B x columns, lens: int32 [B], keys of each request with the newest ones.  A token sees the keys up to
    itself, the last `window` (None: all) and the first `sinks`.  Returns {"O": B x Lq x Hq x dv, "lse": B x Hq x Lq float32 with
    want_lse}; `out` may supply them."""
    if Q.dim() != 4:
        raise ValueError("Q must be 4-D (requests, tokens, heads, width)")
    code = _dtype_code(Q)
    B, Lq, Hq, dk = Q.shape
    _c_int(B, Lq, Hq, dk)
    q = _heads(Q, "Q", Q.shape, Q)
    kc, vc, pages, size = _cache(Kc, Vc, Q)
    if Kc.shape[3] != dk:
        raise ValueError(f"Kc must be {dk} wide, got {Kc.shape[3]}")
    dev = Q.device
    t, rows, columns, ld = _table(table, dev)
    if rows != B:
        raise ValueError(f"table must have {B} rows, got {rows}")
    w = _window(window, sinks, 0, B, dev)
    if scale is None:
        scale = dk ** -0.5 if dk else 1.0
    a = _Paged(code, B, Lq, Hq, Kc.shape[2], dk, Vc.shape[3], scale, pages, size, columns, t, ld, _int_vector(lens, "lens", B, dev),
               _int_vector(q_lens, "q_lens", B, dev) if q_lens is not None else None, w.window, w.sinks, PATHS[path])
    if not Q.is_cuda:
        raise TypeError("Q and the cache must be CUDA tensors")
    L, ref = load_library(), ctypes.byref
    out = dict(out) if out else {}
    with _on_stream(dev, stream):
        if "O" not in out:
            out["O"] = torch.empty((B, Lq, Hq, a.dv), dtype=Q.dtype, device=dev)
        if want_lse and out.get("lse") is None:
            out["lse"] = torch.empty((B, Hq, Lq), dtype=torch.float32, device=dev)
        o = _heads(out["O"], "O", (B, Lq, Hq, a.dv), Q)
        lse = _attn_lse(out["lse"], (B, Hq, Lq), dev) if out.get("lse") is not None else None
        n = ctypes.c_longlong()
        _check(L.gs_paged_attention_workspace(ref(a), ref(n)), "gs_paged_attention_workspace")
        ws = torch.empty(n.value, dtype=torch.uint8, device=dev) if n.value else None
        st = L.gs_paged_attention(ref(a), ref(q), ref(kc), ref(vc), ref(o), lse, _ptr(ws), n.value, _stream(stream, dev))
    _check(st, "gs_paged_attention")
    return out


def verify_drafts(P, D, drafts, U, draft_lens=None, out=None, stream=None):
    """Which drafted tokens stand, and the token behind them; see gs_verify_drafts.

    P: B x (K + 1) x M probabilities of the target (float32 or bfloat16, unit stride along M), D: B x K x M, those that the drafts
    were drawn from (None: chosen without chance), drafts: int32 B x K, U: float32 B x (K + 1) numbers of [0, 1), draft_lens: int32
    [B] or None (K each).  Returns {"accepted": int32 [B], "tokens": int32 B x (K + 1), -1 behind the drawn token}."""
    if P.dim() != 3 or P.shape[1] < 1:
        raise ValueError("P must be 3-D (requests, drafts + 1, entries)")
    code = _dtype_code(P)
    B, K, M = P.shape[0], P.shape[1] - 1, P.shape[2]
    _c_int(B, K, M)
    dev = P.device
    if P.stride(2) != 1 and M > 1:
        raise ValueError("P must have unit stride along its last axis")
    if D is not None:
        if D.shape != (B, K, M) or (D.stride(2) != 1 and M > 1):
            raise ValueError(f"D must be {B} x {K} x {M} with unit stride along its last axis")
        if D.dtype is not P.dtype or D.device != dev:
            raise TypeError(f"D must be {P.dtype} on {dev}")
    for name, t, dt, shape in (("drafts", drafts, torch.int32, (B, K)), ("U", U, torch.float32, (B, K + 1))):
        if t.dtype is not dt or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dt} tensor of {shape[0]} x {shape[1]}")
        if t.device != dev:
            raise TypeError(f"{name} must be on {dev}")
    n = _int_vector(draft_lens, "draft_lens", B, dev) if draft_lens is not None else None
    out = dict(out) if out else {}
    for name, shape in (("accepted", (B,)), ("tokens", (B, K + 1))):
        t = out.get(name)
        if t is not None and (t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous() or t.device != dev):
            raise ValueError(f"out[{name!r}] must be a contiguous int32 {' x '.join(map(str, shape))} tensor on {dev}")
    if not P.is_cuda:
        raise TypeError("P must be a CUDA tensor")
    L = load_library()
    with _on_stream(dev, stream):
        for name, shape in (("accepted", (B,)), ("tokens", (B, K + 1))):
            if name not in out:
                out[name] = torch.empty(shape, dtype=torch.int32, device=dev)
        st = L.gs_verify_drafts(P.data_ptr(), _ptr(D) if K else None, code, B, K, M, P.stride(0), P.stride(1),
                                D.stride(0) if D is not None else 0, D.stride(1) if D is not None else 0, drafts.data_ptr(), n,
                                U.data_ptr(), _ptr(out.get("accepted")), _ptr(out.get("tokens")), _stream(stream, dev))
    _check(st, "gs_verify_drafts")
    return out


def sample_scores(S, U, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, want_prob=True, out=None, stream=None):
    """One random entry of each row of the scores S (N x M, float32 or bfloat16, CUDA) from the numbers
    U (N float32 of [0, 1)); see gs_sample_scores for the rules.  temperature, top_k, top_p and min_p are
    numbers or, for one setting per row, contiguous CUDA vectors of N (float32; top_k int32).  Returns
    {"index": N int32, "prob": N float32}, neither recorded by autograd."""
    ld = _ld(S)
    N, M = S.shape
    _c_int(M)
    dev = S.device
    code = _dtype_code(S)

    def vector(t, name, dt):
        if t.dtype is not dt or t.shape != (N,) or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dt} vector of N = {N} entries")
        if t.device != dev:
            raise TypeError(f"{name} must be on {dev}")
        return t.data_ptr()

    how = _Sampling()
    for name, v, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                        ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if isinstance(v, torch.Tensor):
            setattr(how, name + "_rows", vector(v, name, dt))
        else:
            setattr(how, name, max(0, min(int(v), M)) if name == "top_k" else float(v))
    u = vector(U, "U", torch.float32)
    out = dict(out) if out else {}
    for name, dt in (("index", torch.int32), ("prob", torch.float32)):
        if out.get(name) is not None:
            vector(out[name], f"out[{name!r}]", dt)
    if not S.is_cuda:
        raise TypeError("S must be a CUDA tensor")
    L = load_library()
    with _on_stream(dev, stream):
        if "index" not in out:
            out["index"] = torch.empty(N, dtype=torch.int32, device=dev)
        if want_prob and "prob" not in out:
            out["prob"] = torch.empty(N, dtype=torch.float32, device=dev)
        st = L.gs_sample_scores(S.data_ptr(), code, N, M, ld if N > 1 else M, ctypes.byref(how), u, _ptr(out.get("index")),
                                _ptr(out.get("prob")), _stream(stream, dev))
    _check(st, "gs_sample_scores")
    return out


def project_similarity_static(Q, R, cnorm, X, mode="raw", scale=1.0, want_argmax=True, want_maxval=True,
                              out=None, stream=None):
    """Project + similarity from a caller-held basis without any device allocation by the
    library; see gs_project_similarity_static.  Q: r x D, R: M x r, cnorm: M (fp32, CUDA)."""
    # the C entry takes ld(Q) = D and ld(R) = r and reads cnorm[0..M): every shape is checked here,
    # before any pointer reaches the library
    if Q.dim() != 2 or R.dim() != 2 or X.dim() != 2 or cnorm.dim() != 1:
        raise ValueError("Q, R, X must be 2-D and cnorm 1-D")
    N = X.shape[0]
    r, D = Q.shape
    M = R.shape[0]
    if R.shape[1] != r:
        raise ValueError(f"R must be M x r with r = {r} (Q's rows), got {tuple(R.shape)}")
    if X.shape[1] != D:
        raise ValueError(f"X must be N x {D} (Q's columns), got {tuple(X.shape)}")
    if cnorm.shape[0] != M:
        raise ValueError(f"cnorm must hold M = {M} entries, got {cnorm.shape[0]}")
    for t in (Q, R):
        if t.numel() and not t.is_contiguous():
            raise ValueError("Q and R must be contiguous")
    out = dict(out or {})
    for key, dt in (("argmax", torch.int32), ("maxval", torch.float32)):
        t = out.get(key)
        if t is not None and (t.dtype != dt or t.dim() != 1 or t.shape[0] != N or not t.is_contiguous()):
            raise ValueError(f"out[{key!r}] must be a contiguous {dt} vector of N = {N} entries")
    for name, t in (("Q", Q), ("R", R), ("cnorm", cnorm), ("X", X)):
        if t.dtype != torch.float32:
            raise TypeError(f"{name} must be float32, got {t.dtype}")
    tensors = [Q, R, cnorm, X] + [t for t in out.values() if t is not None]
    if any(not t.is_cuda for t in tensors) or len({t.device for t in tensors}) != 1:
        raise TypeError("Q, R, cnorm, X and the outputs must be CUDA tensors on one device")
    if want_argmax and "argmax" not in out:
        out["argmax"] = torch.empty(N, dtype=torch.int32, device=X.device)
    if want_maxval and "maxval" not in out:
        out["maxval"] = torch.empty(N, dtype=torch.float32, device=X.device)
    L = load_library()
    with _on(X.device):
        st = L.gs_project_similarity_static(_ptr(Q) if Q.numel() else None, r, D, _ptr(R) if R.numel() else None,
                                            M, _ptr(cnorm), _ptr(X), N, _ld(X), MODES[mode], float(scale),
                                            _ptr(out.get("argmax")), _ptr(out.get("maxval")), _stream(stream, X.device))
    _check(st, "gs_project_similarity_static")
    return out


def stream_status(stream=None):
    """Synchronises and raises GramSpaceError if the device recorded an error."""
    L = load_library()
    st = L.gs_stream_status(_stream(stream) if stream is not False else None)
    _check(st, "gs_stream_status")


def selftest_wait_timeout(stream=None):
    """Enqueue a block whose bounded wait runs out (~2 s); see gs_selftest_wait_timeout.
    stream_status() afterwards raises GramSpaceError with GS_ERR_TIMEOUT."""
    _check(load_library().gs_selftest_wait_timeout(_stream(stream)), "gs_selftest_wait_timeout")

"""UltraMem memory-layer forward on AMD Instinct MI355X (gfx950).

A thin ctypes binding of ``libumem.so``, whose C ABI is declared in ``include/umem.h``.  Every
function here has the C function's name and arguments and only marshals them: device arrays may
be passed as torch tensors (contiguous, on the GPU) or as raw integer addresses, ``None`` is a
NULL pointer, and ``stream=None`` means torch's current stream.  Each returns the C status code;
:func:`check` turns a non-zero status into :class:`UmemError`.  All computation happens in the
library's HIP kernels; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

# torch first: its HIP runtime (libamdhip64.so, SONAME libamdhip64.so.7) must be the one in the
# process before libumem.so is loaded, so that libumem.so binds to it.  Loaded the other way
# round, torch would bring in a second copy of the runtime, and the two would not share
# devices, streams or allocations.
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libumem.so")

UMEM_OK = 0
UMEM_ERR_INVALID_ARG = -1
UMEM_ERR_UNSUPPORTED = -2
UMEM_ERR_WORKSPACE = -3
UMEM_ERR_HIP = -4
UMEM_ERR_SCRATCH_LIMIT = -5
UMEM_STATIC_SCRATCH_BYTES = 64 << 20
UMEM_F32, UMEM_BF16 = 0, 1
UMEM_GRID_ADD, UMEM_GRID_TUCKER = 0, 1
UMEM_W_RAW, UMEM_W_SOFTMAX = 0, 1
UMEM_NORM_LAYER, UMEM_NORM_RMS, UMEM_NORM_NONE = 0, 1, 2
UMEM_GATE_NONE, UMEM_GATE_CHANNEL, UMEM_GATE_TOKEN, UMEM_GATE_FULL = 0, 1, 2, 3
UMEM_ACT_LINEAR, UMEM_ACT_SIGMOID = 0, 1

EXPORTED = ("umem_workspace_size", "umem_axis_scores", "umem_select", "umem_score_topk",
            "umem_gather_sum", "umem_project_workspace_size", "umem_project", "umem_forward",
            "umem_forward_noalloc",
            "umem_query_workspace_size", "umem_query", "umem_key_norm",
            "umem_gather_backward_workspace_size", "umem_gather_backward", "umem_gather_backward_rows",
            "umem_score_backward_workspace_size", "umem_score_backward",
            "umem_block_in", "umem_block_out", "umem_block_backward_workspace_size",
            "umem_block_in_backward", "umem_block_out_backward",
            "umem_grad_workspace_size", "umem_grad_norm", "umem_grad_clip",
            "umem_adapter_workspace_size", "umem_adapter_add",
            "umem_query_adapted_workspace_size", "umem_query_adapted", "umem_status_string")


class umem_desc(ctypes.Structure):
    _fields_ = [
        ("heads", ctypes.c_int32), ("dk", ctypes.c_int32), ("n_keys", ctypes.c_int32),
        ("rank", ctypes.c_int32), ("topk", ctypes.c_int32), ("topm", ctypes.c_int32),
        ("grid", ctypes.c_int32), ("weight", ctypes.c_int32), ("n_values", ctypes.c_int64),
        ("dv", ctypes.c_int32), ("vdtype", ctypes.c_int32), ("expand", ctypes.c_int32),
        ("dv_virt", ctypes.c_int32), ("d_out", ctypes.c_int32), ("cores", ctypes.c_int32),
    ]


class umem_query_desc(ctypes.Structure):
    _fields_ = [
        ("d_model", ctypes.c_int32), ("conv_k", ctypes.c_int32), ("heads", ctypes.c_int32),
        ("dk", ctypes.c_int32), ("shared", ctypes.c_int32), ("eps", ctypes.c_float),
    ]


class umem_block_desc(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32), ("norm_in", ctypes.c_int32), ("norm_out", ctypes.c_int32),
        ("gate", ctypes.c_int32), ("gate_act", ctypes.c_int32), ("htype", ctypes.c_int32),
        ("ytype", ctypes.c_int32), ("eps", ctypes.c_float), ("res_scale", ctypes.c_float),
        ("out_scale", ctypes.c_float),
    ]


class umem_grad(ctypes.Structure):
    _fields_ = [
        ("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n_rows", ctypes.c_void_p),
        ("rows", ctypes.c_int64), ("row_len", ctypes.c_int64), ("dtype", ctypes.c_int64),
    ]


class umem_adapter_desc(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int32), ("rank", ctypes.c_int32), ("d_in", ctypes.c_int32),
        ("d_out", ctypes.c_int32), ("xtype", ctypes.c_int32), ("otype", ctypes.c_int32),
    ]


class UmemError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        super().__init__(f"{what}: {umem_status_string(status)} ({status})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    F32 = ctypes.c_float
    BD, AD = ctypes.POINTER(umem_block_desc), ctypes.POINTER(umem_adapter_desc)
    D = ctypes.POINTER(umem_desc)
    sig = {
        "umem_workspace_size": [D, I32, ctypes.POINTER(SZ)],
        "umem_axis_scores": [D, I32, P, P, P, P, P, P, P, SZ, P],
        "umem_select": [D, I32, P, P, P, P, P, P, P, P, P, P, P, P],
        "umem_score_topk": [D, I32, P, P, P, P, P, P, P, P, P, SZ, P],
        "umem_gather_sum": [I64, I32, I32, P, I32, I32, P, P, P, I32, I32, P, P],
        "umem_project_workspace_size": [I32, I32, I32, I32, I32, ctypes.POINTER(SZ)],
        "umem_project": [I32, I32, I32, I32, I32, P, P, P, P, P, SZ, P],
        "umem_forward": [D, I32, P, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P],
        "umem_forward_noalloc": [D, I32, P, P, P, P, P, P, P, P, P, P, P, P, P],
        "umem_query_workspace_size": [ctypes.POINTER(umem_query_desc), I32, I32, ctypes.POINTER(SZ)],
        "umem_query": [ctypes.POINTER(umem_query_desc), I32, I32, P, P, P, P, P, P, P, P, P, SZ, P],
        "umem_key_norm": [I32, I32, I32, P, P, P, ctypes.c_float, P, P],
        "umem_gather_backward_workspace_size": [I32, I32, I32, ctypes.POINTER(SZ)],
        "umem_gather_backward": [I64, I32, I32, P, I32, I32, P, P, P, I32, I32, P, P, P, P, SZ, P],
        "umem_gather_backward_rows": [I64, I32, I32, P, I32, I32, P, P, P, I32, I32, P, P, P, P, P, P,
                                      SZ, P],
        "umem_score_backward_workspace_size": [D, I32, ctypes.POINTER(SZ)],
        "umem_score_backward": [D, I32, P, P, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P],
        "umem_block_in": [BD, I32, P, P, P, P, P],
        "umem_block_out": [BD, I32, P, P, P, P, P, P, P, P, P, P],
        "umem_block_backward_workspace_size": [BD, I32, ctypes.POINTER(SZ)],
        "umem_block_in_backward": [BD, I32, P, P, P, P, P, P, P, I32, P, SZ, P],
        "umem_block_out_backward": [BD, I32, P, P, P, P, P, P, P, P, P, P, I32, P, SZ, P],
        "umem_grad_workspace_size": [I32, P, ctypes.POINTER(SZ)],
        "umem_grad_norm": [I32, P, P, P, P, SZ, P],
        "umem_grad_clip": [I32, P, F32, P, P],
        "umem_adapter_workspace_size": [AD, I32, ctypes.POINTER(SZ)],
        "umem_adapter_add": [AD, I32, P, P, P, P, P, P, P, P, SZ, P],
        "umem_query_adapted_workspace_size": [ctypes.POINTER(umem_query_desc), AD, I32, I32, ctypes.POINTER(SZ)],
        "umem_query_adapted": [ctypes.POINTER(umem_query_desc), AD, I32, I32, P, P, P, P, P, P, P, P, P, P, P, P, P,
                               SZ, P],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.umem_status_string.argtypes = [ctypes.c_int]
    lib.umem_status_string.restype = ctypes.c_char_p
    return lib


_lib = _load()


# The current device and its current stream's handle.  torch builds without a GPU lack these calls.
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda d: torch.cuda.current_stream(d).cuda_stream)


def _p(x):
    """A device address: None -> NULL, int -> itself, torch tensor -> data_ptr()."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_contiguous():
        raise ValueError("tensor arguments must be contiguous")
    if not x.is_cuda:
        raise ValueError("tensor arguments must live on the GPU")
    return x.data_ptr()


def _s(stream, like=None):
    """A stream's handle; None is torch's current stream, of the current device, on which the tensor
    ``like`` (where it is one) has to live then."""
    if stream is None:
        device = _get_device()
        if like is not None and not isinstance(like, int) and like.get_device() != device:
            raise ValueError("tensor arguments must live on the current device, or a stream be given")
        return _raw_stream(device)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _d(desc):
    return ctypes.byref(desc)


def umem_status_string(status: int) -> str:
    return _lib.umem_status_string(status).decode()


def check(status: int, what: str = "umem") -> None:
    if status != UMEM_OK:
        raise UmemError(status, what)


def umem_workspace_size(desc: umem_desc, T: int):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_workspace_size(_d(desc), T, ctypes.byref(out))
    return st, out.value


def umem_axis_scores(desc, T, q_row, q_col, k_row, k_col, core, sel, ws=None, ws_bytes=0,
                     stream=None) -> int:
    return _lib.umem_axis_scores(_d(desc), T, _p(q_row), _p(q_col), _p(k_row), _p(k_col), _p(core),
                                 _p(sel), _p(ws), ws_bytes, _s(stream))


def umem_select(desc, T, sel, q_row, q_col, k_row, k_col, core, idx, w, axis_idx=None,
                values=None, pooled=None, stream=None) -> int:
    return _lib.umem_select(_d(desc), T, _p(sel), _p(q_row), _p(q_col), _p(k_row), _p(k_col),
                            _p(core), _p(idx), _p(w), _p(axis_idx), _p(values), _p(pooled),
                            _s(stream))


def umem_score_topk(desc, T, q_row, q_col, k_row, k_col, core, idx, w, axis_idx, ws, ws_bytes,
                    stream=None) -> int:
    return _lib.umem_score_topk(_d(desc), T, _p(q_row), _p(q_col), _p(k_row), _p(k_col), _p(core),
                                _p(idx), _p(w), _p(axis_idx), _p(ws), ws_bytes, _s(stream))


def umem_gather_sum(n_values, dv, vdtype, values, T, bag, idx, w, perm, expand, cores, out,
                    stream=None) -> int:
    return _lib.umem_gather_sum(n_values, dv, vdtype, _p(values), T, bag, _p(idx), _p(w), _p(perm),
                                expand, cores, _p(out), _s(stream))


def umem_project_workspace_size(T, expand, dv, dv_virt, d_out):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_project_workspace_size(T, expand, dv, dv_virt, d_out, ctypes.byref(out))
    return st, out.value


def umem_project(T, expand, dv, dv_virt, d_out, pooled, w_proj, w_out, out, ws, ws_bytes,
                 stream=None) -> int:
    return _lib.umem_project(T, expand, dv, dv_virt, d_out, _p(pooled), _p(w_proj), _p(w_out),
                             _p(out), _p(ws), ws_bytes, _s(stream))


def umem_forward(desc, T, q_row, q_col, k_row, k_col, core, values, perm, w_proj, w_out, out,
                 idx_out, w_out_scores, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_forward(_d(desc), T, _p(q_row), _p(q_col), _p(k_row), _p(k_col), _p(core),
                             _p(values), _p(perm), _p(w_proj), _p(w_out), _p(out), _p(idx_out),
                             _p(w_out_scores), _p(ws), ws_bytes, _s(stream))


def umem_forward_noalloc(desc, T, q_row, q_col, k_row, k_col, core, values, perm, w_proj, w_out,
                         out, idx_out, w_out_scores, stream=None) -> int:
    return _lib.umem_forward_noalloc(_d(desc), T, _p(q_row), _p(q_col), _p(k_row), _p(k_col),
                                     _p(core), _p(values), _p(perm), _p(w_proj), _p(w_out), _p(out),
                                     _p(idx_out), _p(w_out_scores), _s(stream))


def umem_query_workspace_size(qd, B, L):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_query_workspace_size(ctypes.byref(qd), B, L, ctypes.byref(out))
    return st, out.value


def umem_query(qd, B, L, x, x_hist, conv_w, w_q, gamma, beta, q_row, q_col, ws, ws_bytes,
               stream=None) -> int:
    return _lib.umem_query(ctypes.byref(qd), B, L, _p(x), _p(x_hist), _p(conv_w), _p(w_q),
                           _p(gamma), _p(beta), _p(q_row), _p(q_col), _p(ws), ws_bytes, _s(stream))


def umem_key_norm(heads, n, dk, keys, gamma, beta, eps, out, stream=None) -> int:
    return _lib.umem_key_norm(heads, n, dk, _p(keys), _p(gamma), _p(beta), eps, _p(out), _s(stream))


def umem_gather_backward_workspace_size(T, bag, dv):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_gather_backward_workspace_size(T, bag, dv, ctypes.byref(out))
    return st, out.value


def umem_gather_backward(n_values, dv, vdtype, values, T, bag, idx, w, perm, expand, cores,
                         d_pooled, d_values, dw, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_gather_backward(n_values, dv, vdtype, _p(values), T, bag, _p(idx), _p(w),
                                     _p(perm), expand, cores, _p(d_pooled), _p(d_values), _p(dw),
                                     _p(ws), ws_bytes, _s(stream))


def umem_gather_backward_rows(n_values, dv, vdtype, values, T, bag, idx, w, perm, expand, cores,
                              d_pooled, rows, d_rows, n_rows, dw, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_gather_backward_rows(n_values, dv, vdtype, _p(values), T, bag, _p(idx), _p(w),
                                          _p(perm), expand, cores, _p(d_pooled), _p(rows),
                                          _p(d_rows), _p(n_rows), _p(dw), _p(ws), ws_bytes,
                                          _s(stream))


def umem_score_backward_workspace_size(desc, T):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_score_backward_workspace_size(_d(desc), T, ctypes.byref(out))
    return st, out.value


def umem_score_backward(desc, T, q_row, q_col, k_row, k_col, core, idx, w, dw, dq_row, dq_col,
                        dk_row, dk_col, dcore, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_score_backward(_d(desc), T, _p(q_row), _p(q_col), _p(k_row), _p(k_col),
                                    _p(core), _p(idx), _p(w), _p(dw), _p(dq_row), _p(dq_col),
                                    _p(dk_row), _p(dk_col), _p(dcore), _p(ws), ws_bytes, _s(stream))


def umem_block_in(bd, T, h, gamma, beta, n, stream=None) -> int:
    return _lib.umem_block_in(_d(bd), T, _p(h), _p(gamma), _p(beta), _p(n), _s(stream, h))


def umem_block_out(bd, T, h, y, gate, gamma, beta, h_out, gamma_next=None, beta_next=None,
                   n_next=None, stream=None) -> int:
    return _lib.umem_block_out(_d(bd), T, _p(h), _p(y), _p(gate), _p(gamma), _p(beta), _p(h_out),
                               _p(gamma_next), _p(beta_next), _p(n_next), _s(stream, h))


def umem_block_backward_workspace_size(bd, T):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_block_backward_workspace_size(_d(bd), T, ctypes.byref(out))
    return st, out.value


def umem_block_in_backward(bd, T, h, gamma, dn, dres, dh, dgamma, dbeta, accumulate, ws, ws_bytes,
                           stream=None) -> int:
    return _lib.umem_block_in_backward(_d(bd), T, _p(h), _p(gamma), _p(dn), _p(dres), _p(dh),
                                       _p(dgamma), _p(dbeta), accumulate, _p(ws), ws_bytes, _s(stream, h))


def umem_block_out_backward(bd, T, y, gate, gamma, beta, dh_out, dh, dy, dgate, dgamma, dbeta,
                            accumulate, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_block_out_backward(_d(bd), T, _p(y), _p(gate), _p(gamma), _p(beta), _p(dh_out),
                                        _p(dh), _p(dy), _p(dgate), _p(dgamma), _p(dbeta), accumulate,
                                        _p(ws), ws_bytes, _s(stream, y))


def _table(n, grads):
    """The host address of n gradients: an array ``(umem_grad * n)``, or a C-ordered int64 numpy array
    [n, 6] with a row of the struct's six fields for each."""
    if isinstance(grads, ctypes.Array):
        if grads._type_ is not umem_grad or len(grads) < n:
            raise ValueError("grads: an array of at least n umem_grad")
        return ctypes.addressof(grads)
    if grads is None:
        return None
    if grads.dtype != "int64" or grads.ndim != 2 or grads.shape[1] != 6 or grads.shape[0] < n or \
            not grads.flags.c_contiguous:
        raise ValueError("grads: int64 [n, 6], C-ordered")
    return grads.ctypes.data


def umem_grad_workspace_size(n, grads):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_grad_workspace_size(n, _table(n, grads), ctypes.byref(out))
    return st, out.value


def umem_grad_norm(n, grads, norm, sumsq, ws, ws_bytes, stream=None) -> int:
    return _lib.umem_grad_norm(n, _table(n, grads), _p(norm), _p(sumsq), _p(ws), ws_bytes, _s(stream, norm))


def umem_grad_clip(n, grads, max_norm, norm, stream=None) -> int:
    return _lib.umem_grad_clip(n, _table(n, grads), max_norm, _p(norm), _s(stream, norm))


def umem_adapter_workspace_size(ad, T):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_adapter_workspace_size(_d(ad), T, ctypes.byref(out))
    return st, out.value


def umem_adapter_add(ad, T, x, ids, a, b, scale, base, out, ws=None, ws_bytes=0, stream=None) -> int:
    return _lib.umem_adapter_add(_d(ad), T, _p(x), _p(ids), _p(a), _p(b), _p(scale), _p(base), _p(out),
                                 _p(ws), ws_bytes, _s(stream, x))


def umem_query_adapted_workspace_size(qd, ad, B, L):
    """Returns (status, bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.umem_query_adapted_workspace_size(_d(qd), _d(ad), B, L, ctypes.byref(out))
    return st, out.value


def umem_query_adapted(qd, ad, B, L, x, x_hist, conv_w, w_q, ids, a, b, scale, gamma, beta, q_row, q_col,
                       ws, ws_bytes, stream=None) -> int:
    return _lib.umem_query_adapted(_d(qd), _d(ad), B, L, _p(x), _p(x_hist), _p(conv_w), _p(w_q), _p(ids),
                                   _p(a), _p(b), _p(scale), _p(gamma), _p(beta), _p(q_row), _p(q_col),
                                   _p(ws), ws_bytes, _s(stream, x))

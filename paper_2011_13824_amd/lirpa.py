"""Thin ctypes binding of ``liblirpa.so`` (the C ABI declared in include/lirpa.h).

The functions below carry the C names and only marshal arguments: torch CUDA tensors become
device pointers and the current torch stream becomes the ``hipStream_t``.  Every step of the
bound computation runs in the HIP library; there is no fallback.  ``Network`` is a small
convenience owner of device weights, a net handle and a workspace.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "liblirpa.so")

LIRPA_OK, LIRPA_EINVAL, LIRPA_ENOMEM, LIRPA_EDEVICE, LIRPA_EUNSUPPORTED, LIRPA_EDATA = \
    0, -1, -2, -3, -4, -5
LINEAR, CONV2D = 0, 1
F32, BF16, F16 = 0, 1, 2
DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
GATES = {"relu": 0, "silu": 1, "gelu": 2}
KEEP_NONE, KEEP_FULL, KEEP_8 = -1, 0, 8


class lirpa_layer(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("in_c", ctypes.c_int), ("in_h", ctypes.c_int),
                ("in_w", ctypes.c_int), ("out_c", ctypes.c_int), ("out_h", ctypes.c_int),
                ("out_w", ctypes.c_int), ("k", ctypes.c_int), ("stride", ctypes.c_int),
                ("pad", ctypes.c_int), ("W", ctypes.c_void_p), ("b", ctypes.c_void_p)]


class lirpa_opt_params(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("lr", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps_adam", ctypes.c_float), ("t0", ctypes.c_int),
                ("fresh", ctypes.c_int)]


class lirpa_bab_params(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("max_domains", ctypes.c_int),
                ("max_iters", ctypes.c_int), ("root_steps", ctypes.c_int),
                ("steps", ctypes.c_int), ("lr", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps_adam", ctypes.c_float)]


class lirpa_bab_result(ctypes.Structure):
    _fields_ = [("status", ctypes.c_int), ("f_lo", ctypes.c_float), ("f_hi", ctypes.c_float),
                ("iterations", ctypes.c_int), ("domains_bounded", ctypes.c_int64),
                ("domains_left", ctypes.c_int)]


class lirpa_ffn(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("gate", ctypes.c_int), ("n_model", ctypes.c_int),
                ("n_hidden", ctypes.c_int), ("Wg", ctypes.c_void_p), ("Wu", ctypes.c_void_p),
                ("Wd", ctypes.c_void_p), ("ldg", ctypes.c_int64), ("ldu", ctypes.c_int64),
                ("ldd", ctypes.c_int64)]


class lirpa_scan(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("rows", ctypes.c_int64), ("n", ctypes.c_int),
                ("states", ctypes.c_int), ("u", ctypes.c_void_p), ("dt", ctypes.c_void_p),
                ("z", ctypes.c_void_p), ("B", ctypes.c_void_p), ("C", ctypes.c_void_p),
                ("ldu", ctypes.c_int64), ("lddt", ctypes.c_int64), ("ldz", ctypes.c_int64),
                ("ldB", ctypes.c_int64), ("ldC", ctypes.c_int64), ("A", ctypes.c_void_p),
                ("D", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("seq", ctypes.c_void_p),
                ("slots", ctypes.c_int)]


CONV_ACTS = {"linear": 0, "silu": 1}
ANY_SLOT = 2 ** 31 - 1  # where no states come with the sequences

BAB_VERIFIED, BAB_VIOLATED, BAB_UNKNOWN_STUCK, BAB_UNKNOWN_LIMIT = 1, 2, 3, 4


class lirpa_kernel_time(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("total_ms", ctypes.c_double),
                ("launches", ctypes.c_int64)]


SYMBOLS = ("lirpa_net_create", "lirpa_net_destroy", "lirpa_net_num_relu",
           "lirpa_workspace_bytes", "lirpa_bound", "lirpa_bound_child", "lirpa_bound_noalloc",
           "lirpa_bound_ul",
           "lirpa_bound_grad", "lirpa_optimize", "lirpa_optimize_ul",
           "lirpa_bab_workspace_bytes", "lirpa_bab",
           "lirpa_q8_bytes", "lirpa_q8_pack", "lirpa_q8_unpack",
           "lirpa_norm_forward", "lirpa_norm_workspace_bytes", "lirpa_norm_backward",
           "lirpa_ffn_workspace_bytes", "lirpa_ffn_forward", "lirpa_ffn_backward",
           "lirpa_embed_forward", "lirpa_embed_workspace_bytes", "lirpa_embed_backward",
           "lirpa_logprob_workspace_bytes", "lirpa_logprob_forward", "lirpa_logprob_backward",
           "lirpa_conv_forward", "lirpa_conv_step", "lirpa_conv_workspace_bytes",
           "lirpa_conv_backward", "lirpa_scan_workspace_bytes", "lirpa_scan_kept_bytes",
           "lirpa_scan_forward", "lirpa_scan_step", "lirpa_scan_backward",
           "lirpa_timing_begin", "lirpa_timing_end", "lirpa_last_error")

_lib = None


def load() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -c 'import __graft_entry__ as g; g.build()'`")
    L = ctypes.CDLL(LIB_PATH)
    P, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    L.lirpa_net_create.argtypes = [ctypes.POINTER(lirpa_layer), i, ctypes.POINTER(P)]
    L.lirpa_net_create.restype = i
    L.lirpa_net_destroy.argtypes = [P]
    L.lirpa_net_destroy.restype = None
    L.lirpa_net_num_relu.argtypes = [P]
    L.lirpa_net_num_relu.restype = ctypes.c_int64
    L.lirpa_workspace_bytes.argtypes = [P, i, i, i]
    L.lirpa_workspace_bytes.restype = sz
    L.lirpa_bound.argtypes = [P, P, f, P, i, i, P, P, P, P, P, P, P, sz, P]
    L.lirpa_bound.restype = i
    L.lirpa_bound_child.argtypes = [P, P, f, P, i, i, P, P, P, P, P, P, P, P, P, sz, P]
    L.lirpa_bound_child.restype = i
    L.lirpa_bound_noalloc.argtypes = [P, P, f, P, i, i, P, P, P, P, P, P, P]
    L.lirpa_bound_noalloc.restype = i
    L.lirpa_bound_ul.argtypes = [P, P, f, P, i, i, P, P, P, P, P, P, P, P, sz, P]
    L.lirpa_bound_ul.restype = i
    L.lirpa_optimize_ul.argtypes = [P, P, f, P, i, i, P, P, P, P, P, P, P,
                                    ctypes.POINTER(lirpa_opt_params), P, P, P, sz, P]
    L.lirpa_optimize_ul.restype = i
    L.lirpa_bab_workspace_bytes.argtypes = [P, ctypes.POINTER(lirpa_bab_params)]
    L.lirpa_bab_workspace_bytes.restype = sz
    L.lirpa_bab.argtypes = [P, P, f, P, ctypes.POINTER(lirpa_bab_params),
                            ctypes.POINTER(lirpa_bab_result), P, sz, P]
    L.lirpa_bab.restype = i
    L.lirpa_bound_grad.argtypes = [P, P, f, P, i, i, P, P, i, P, P, P, sz, P]
    L.lirpa_bound_grad.restype = i
    L.lirpa_optimize.argtypes = [P, P, f, P, i, i, P, P, P, P, ctypes.POINTER(lirpa_opt_params),
                                 P, P, P, sz, P]
    L.lirpa_optimize.restype = i
    q, block = ctypes.c_int64, ctypes.POINTER(lirpa_ffn)
    L.lirpa_q8_bytes.argtypes = [q, i]
    L.lirpa_q8_bytes.restype = sz
    L.lirpa_q8_pack.argtypes = [i, q, i, P, q, P, P]
    L.lirpa_q8_pack.restype = i
    L.lirpa_q8_unpack.argtypes = [i, q, i, P, P, q, P]
    L.lirpa_q8_unpack.restype = i
    L.lirpa_norm_forward.argtypes = [i, q, i, P, q, P, q, P, f, P, q, P, q, P, P, P]
    L.lirpa_norm_forward.restype = i
    L.lirpa_norm_workspace_bytes.argtypes = [q, i]
    L.lirpa_norm_workspace_bytes.restype = sz
    L.lirpa_norm_backward.argtypes = [i, q, i, P, q, P, q, P, q, P, P, P, q, P, P, sz, P]
    L.lirpa_norm_backward.restype = i
    L.lirpa_ffn_workspace_bytes.argtypes = [block, q, i]
    L.lirpa_ffn_workspace_bytes.restype = sz
    L.lirpa_ffn_forward.argtypes = [block, q, P, q, P, q, i, P, P, P, sz, P]
    L.lirpa_ffn_forward.restype = i
    L.lirpa_ffn_backward.argtypes = [block, q, P, q, i, P, q, P, P, P, q, P, P, P, P, sz, P]
    L.lirpa_ffn_backward.restype = i
    L.lirpa_embed_forward.argtypes = [i, q, i, i, P, P, q, f, P, q, P]
    L.lirpa_embed_forward.restype = i
    L.lirpa_embed_workspace_bytes.argtypes = [q, i]
    L.lirpa_embed_workspace_bytes.restype = sz
    L.lirpa_embed_backward.argtypes = [i, q, i, i, P, P, q, f, P, q, P, q, P, sz, P]
    L.lirpa_embed_backward.restype = i
    L.lirpa_logprob_workspace_bytes.argtypes = [q, i, i]
    L.lirpa_logprob_workspace_bytes.restype = sz
    L.lirpa_logprob_forward.argtypes = [i, q, i, P, q, f, P, P, P, P, i, P, P, P, sz, P]
    L.lirpa_logprob_forward.restype = i
    L.lirpa_logprob_backward.argtypes = [i, q, i, P, q, f, P, P, P, P, P, P, q, P]
    L.lirpa_logprob_backward.restype = i
    conv = [i, q, i, i, P, q, P, P, i, P, i, P, P, P, q, P]
    L.lirpa_conv_forward.argtypes = L.lirpa_conv_step.argtypes = conv
    L.lirpa_conv_forward.restype = L.lirpa_conv_step.restype = i
    L.lirpa_conv_workspace_bytes.argtypes = [q, i, i]
    L.lirpa_conv_workspace_bytes.restype = sz
    L.lirpa_conv_backward.argtypes = [i, q, i, i, P, q, P, q, P, P, i, P, i, P, q, P, P, P, sz, P]
    L.lirpa_conv_backward.restype = i
    scan = ctypes.POINTER(lirpa_scan)
    L.lirpa_scan_workspace_bytes.argtypes = [q, i, i, i]
    L.lirpa_scan_workspace_bytes.restype = sz
    L.lirpa_scan_kept_bytes.argtypes = [q, i, i]
    L.lirpa_scan_kept_bytes.restype = sz
    L.lirpa_scan_forward.argtypes = [scan, P, P, P, q, P, P, sz, P]
    L.lirpa_scan_forward.restype = i
    L.lirpa_scan_step.argtypes = [scan, P, P, P, q, P]
    L.lirpa_scan_step.restype = i
    L.lirpa_scan_backward.argtypes = [scan, P, q, P, *[P, q] * 5, P, P, P, P, sz, P]
    L.lirpa_scan_backward.restype = i
    L.lirpa_timing_begin.argtypes = []
    L.lirpa_timing_begin.restype = i
    L.lirpa_timing_end.argtypes = [ctypes.POINTER(lirpa_kernel_time), i, ctypes.POINTER(i)]
    L.lirpa_timing_end.restype = i
    L.lirpa_last_error.argtypes = []
    L.lirpa_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


class LirpaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"lirpa error {code}: {msg}")
        self.code = code


def _check(rc):
    if rc:
        raise LirpaError(rc, load().lirpa_last_error().decode())


def _dev(t, dtype=None, what="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:  # the raw handle: a torch.cuda.Stream object costs more than a small call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def lirpa_last_error() -> str:
    return load().lirpa_last_error().decode()


def lirpa_timing_begin():
    _check(load().lirpa_timing_begin())


def lirpa_timing_end(max_entries=256):
    """{kernel class: (total_ms, launches)} of the kernels enqueued since lirpa_timing_begin."""
    arr = (lirpa_kernel_time * max_entries)()
    n = ctypes.c_int(0)
    _check(load().lirpa_timing_end(arr, max_entries, ctypes.byref(n)))
    return {arr[i].name.decode(): (arr[i].total_ms, int(arr[i].launches))
            for i in range(min(n.value, max_entries))}


def lirpa_net_create(layers):
    """layers: list of dicts with the layer fields and device tensors ``W``, ``b``."""
    arr = (lirpa_layer * len(layers))()
    for i, t in enumerate(layers):
        arr[i] = lirpa_layer(t["kind"], t["in_c"], t["in_h"], t["in_w"], t["out_c"], t["out_h"],
                             t["out_w"], t.get("k", 0), t.get("stride", 1), t.get("pad", 0),
                             _dev(t["W"], torch.float32, "W"), _dev(t["b"], torch.float32, "b"))
    h = ctypes.c_void_p()
    _check(load().lirpa_net_create(arr, len(layers), ctypes.byref(h)))
    return h


def lirpa_net_destroy(net):
    load().lirpa_net_destroy(net)


def lirpa_net_num_relu(net) -> int:
    return int(load().lirpa_net_num_relu(net))


def lirpa_workspace_bytes(net, S, B_chunk, mode=0) -> int:
    return int(load().lirpa_workspace_bytes(net, S, B_chunk, mode))


def lirpa_bound(net, x0, eps, C, S, B, split, alpha, lb, l_out, u_out, code_out, ws,
                ws_bytes, stream=None):
    _check(load().lirpa_bound(net, _dev(x0, torch.float32, "x0"), float(eps),
                              _dev(C, torch.float32, "C"), int(S), int(B),
                              _dev(split, torch.int8, "split"),
                              _dev(alpha, torch.float32, "alpha"),
                              _dev(lb, torch.float32, "lb"), _dev(l_out, torch.float32, "l_out"),
                              _dev(u_out, torch.float32, "u_out"),
                              _dev(code_out, torch.int8, "code_out"), _dev(ws, None, "ws"),
                              int(ws_bytes), _stream(stream)))


def lirpa_bound_child(net, x0, eps, C, S, B, split, alpha, l_parent, u_parent, lb, l_out, u_out,
                      code_out, ws, ws_bytes, stream=None):
    f32 = torch.float32
    _check(load().lirpa_bound_child(net, _dev(x0, f32, "x0"), float(eps), _dev(C, f32, "C"),
                                    int(S), int(B), _dev(split, torch.int8, "split"),
                                    _dev(alpha, f32, "alpha"), _dev(l_parent, f32, "l_parent"),
                                    _dev(u_parent, f32, "u_parent"), _dev(lb, f32, "lb"),
                                    _dev(l_out, f32, "l_out"), _dev(u_out, f32, "u_out"),
                                    _dev(code_out, torch.int8, "code_out"), _dev(ws, None, "ws"),
                                    int(ws_bytes), _stream(stream)))


def lirpa_bound_noalloc(net, x0, eps, C, S, B, split, alpha, lb, l_out, u_out, code_out,
                        stream=None):
    _check(load().lirpa_bound_noalloc(net, _dev(x0, torch.float32, "x0"), float(eps),
                                      _dev(C, torch.float32, "C"), int(S), int(B),
                                      _dev(split, torch.int8, "split"),
                                      _dev(alpha, torch.float32, "alpha"),
                                      _dev(lb, torch.float32, "lb"),
                                      _dev(l_out, torch.float32, "l_out"),
                                      _dev(u_out, torch.float32, "u_out"),
                                      _dev(code_out, torch.int8, "code_out"), _stream(stream)))


def lirpa_bound_ul(net, x0, eps, C, S, B, split, alpha, lb, ub, l_out, u_out, code_out, ws,
                   ws_bytes, stream=None):
    _check(load().lirpa_bound_ul(net, _dev(x0, torch.float32, "x0"), float(eps),
                                 _dev(C, torch.float32, "C"), int(S), int(B),
                                 _dev(split, torch.int8, "split"),
                                 _dev(alpha, torch.float32, "alpha"),
                                 _dev(lb, torch.float32, "lb"), _dev(ub, torch.float32, "ub"),
                                 _dev(l_out, torch.float32, "l_out"),
                                 _dev(u_out, torch.float32, "u_out"),
                                 _dev(code_out, torch.int8, "code_out"), _dev(ws, None, "ws"),
                                 int(ws_bytes), _stream(stream)))


def lirpa_optimize_ul(net, x0, eps, C, S, B, split, alpha_lo, m_lo, v_lo, alpha_up, m_up, v_up,
                      params, lb_best, ub_best, ws, ws_bytes, stream=None):
    p = params if isinstance(params, lirpa_opt_params) else lirpa_opt_params(**params)
    f32 = torch.float32
    _check(load().lirpa_optimize_ul(net, _dev(x0, f32, "x0"), float(eps), _dev(C, f32, "C"),
                                    int(S), int(B), _dev(split, torch.int8, "split"),
                                    _dev(alpha_lo, f32, "alpha_lo"), _dev(m_lo, f32, "m_lo"),
                                    _dev(v_lo, f32, "v_lo"), _dev(alpha_up, f32, "alpha_up"),
                                    _dev(m_up, f32, "m_up"), _dev(v_up, f32, "v_up"),
                                    ctypes.byref(p), _dev(lb_best, f32, "lb_best"),
                                    _dev(ub_best, f32, "ub_best"), _dev(ws, None, "ws"),
                                    int(ws_bytes), _stream(stream)))


def lirpa_bab_workspace_bytes(net, params) -> int:
    return int(load().lirpa_bab_workspace_bytes(net, ctypes.byref(params)))


def lirpa_bab(net, x0, eps, c, params, ws, ws_bytes, stream=None):
    """Runs the search (the call synchronises the stream); returns the lirpa_bab_result."""
    res = lirpa_bab_result()
    _check(load().lirpa_bab(net, _dev(x0, torch.float32, "x0"), float(eps),
                            _dev(c, torch.float32, "c"), ctypes.byref(params),
                            ctypes.byref(res), _dev(ws, None, "ws"), int(ws_bytes),
                            _stream(stream)))
    return res


def lirpa_bound_grad(net, x0, eps, C, S, B, split, alpha, full, lb, grad, ws, ws_bytes,
                     stream=None):
    _check(load().lirpa_bound_grad(net, _dev(x0, torch.float32, "x0"), float(eps),
                                   _dev(C, torch.float32, "C"), int(S), int(B),
                                   _dev(split, torch.int8, "split"),
                                   _dev(alpha, torch.float32, "alpha"), int(full),
                                   _dev(lb, torch.float32, "lb"),
                                   _dev(grad, torch.float32, "grad"), _dev(ws, None, "ws"),
                                   int(ws_bytes), _stream(stream)))


def lirpa_optimize(net, x0, eps, C, S, B, split, alpha, adam_m, adam_v, params, lb_best,
                   lb_trace, ws, ws_bytes, stream=None):
    p = params if isinstance(params, lirpa_opt_params) else lirpa_opt_params(**params)
    _check(load().lirpa_optimize(net, _dev(x0, torch.float32, "x0"), float(eps),
                                 _dev(C, torch.float32, "C"), int(S), int(B),
                                 _dev(split, torch.int8, "split"),
                                 _dev(alpha, torch.float32, "alpha"),
                                 _dev(adam_m, torch.float32, "adam_m"),
                                 _dev(adam_v, torch.float32, "adam_v"), ctypes.byref(p),
                                 _dev(lb_best, torch.float32, "lb_best"),
                                 _dev(lb_trace, torch.float32, "lb_trace"), _dev(ws, None, "ws"),
                                 int(ws_bytes), _stream(stream)))


def _matrix(t, rows, n, dtype, what):
    """(device pointer, row distance) of a [rows, n] CUDA tensor whose rows are contiguous
    (None -> NULL)."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if t.shape != (rows, n):
        raise ValueError(f"{what} must be [{rows}, {n}], got {list(t.shape)}")
    ld, step = t.stride()
    if step != 1 and n > 1:
        raise ValueError(f"{what} must have contiguous rows")
    if rows <= 1:  # no second row: its distance is of no account, and may be any
        ld = n
    elif ld < n:
        raise ValueError(f"rows of {what} overlap")
    return t.data_ptr(), ld


def _vector(t, n, dtype, what):
    """Device pointer of a contiguous CUDA tensor of n values (None -> NULL)."""
    if t is not None and isinstance(t, torch.Tensor) and t.numel() != n:
        raise ValueError(f"{what} must have {n} values, got {t.numel()}")
    return _dev(t, dtype, what)


def _packed(t, rows, n, what):
    if t is None:
        return None
    need = rows * -(-n // 32) * 33
    if isinstance(t, torch.Tensor) and t.numel() < need:
        raise ValueError(f"{what} must have {need} bytes, got {t.numel()}")
    return _dev(t, torch.uint8, what)


def _dtype(t, what):
    if not isinstance(t, torch.Tensor) or t.dtype not in DTYPES:
        raise TypeError(f"{what} must be a float32, bfloat16 or float16 tensor")
    return t.dtype


def lirpa_q8_bytes(rows, n) -> int:
    return int(load().lirpa_q8_bytes(int(rows), int(n)))


def lirpa_q8_pack(x, q8, stream=None):
    """x [rows, n] into the uint8 tensor q8."""
    rows, n = x.shape
    dt = _dtype(x, "x")
    p, ld = _matrix(x, rows, n, dt, "x")
    _check(load().lirpa_q8_pack(DTYPES[dt], rows, n, p, ld, _packed(q8, rows, n, "q8"),
                                _stream(stream)))


def lirpa_q8_unpack(q8, x, stream=None):
    """The values of q8 into x [rows, n]."""
    rows, n = x.shape
    dt = _dtype(x, "x")
    p, ld = _matrix(x, rows, n, dt, "x")
    _check(load().lirpa_q8_unpack(DTYPES[dt], rows, n, _packed(q8, rows, n, "q8"), p, ld,
                                  _stream(stream)))


def lirpa_norm_forward(x, res, w, eps, sum, y, y8, rstd, stream=None):
    rows, n = x.shape
    dt = _dtype(x, "x")
    _check(load().lirpa_norm_forward(
        DTYPES[dt], rows, n, *_matrix(x, rows, n, dt, "x"), *_matrix(res, rows, n, dt, "res"),
        _vector(w, n, dt, "w"), float(eps), *_matrix(sum, rows, n, dt, "sum"),
        *_matrix(y, rows, n, dt, "y"), _packed(y8, rows, n, "y8"),
        _vector(rstd, rows, torch.float32, "rstd"), _stream(stream)))


def lirpa_norm_workspace_bytes(rows, n) -> int:
    return int(load().lirpa_norm_workspace_bytes(int(rows), int(n)))


def lirpa_norm_backward(dy, dsum, h, w, rstd, dh, dw, ws, ws_bytes, stream=None):
    rows, n = dy.shape
    dt = _dtype(dy, "dy")
    _check(load().lirpa_norm_backward(
        DTYPES[dt], rows, n, *_matrix(dy, rows, n, dt, "dy"), *_matrix(dsum, rows, n, dt, "dsum"),
        *_matrix(h, rows, n, dt, "h"), _vector(w, n, dt, "w"),
        _vector(rstd, rows, torch.float32, "rstd"), *_matrix(dh, rows, n, dt, "dh"),
        _vector(dw, n, dt, "dw"), _dev(ws, None, "ws"), int(ws_bytes), _stream(stream)))


def lirpa_ffn_block(Wg, Wu, Wd, gate):
    """The lirpa_ffn of device weights, which have to outlive the calls that take it."""
    dt = _dtype(Wg, "Wg")
    if Wg.dim() != 2:
        raise ValueError("Wg must be [n_hidden, n_model]")
    if gate not in GATES:
        raise ValueError(f"gate must be one of {sorted(GATES)}, got {gate!r}")
    hidden, model = Wg.shape
    g, ldg = _matrix(Wg, hidden, model, dt, "Wg")
    u, ldu = _matrix(Wu, hidden, model, dt, "Wu")
    d, ldd = _matrix(Wd, model, hidden, dt, "Wd")
    return lirpa_ffn(DTYPES[dt], GATES[gate], model, hidden, g, u, d, ldg, ldu, ldd)


def lirpa_ffn_workspace_bytes(ffn, rows, backward) -> int:
    return int(load().lirpa_ffn_workspace_bytes(ctypes.byref(ffn), int(rows), int(backward)))


def _kept(t, rows, n, dtype, keep, what):
    if keep == KEEP_8:
        return _packed(t, rows, n, what)
    return _vector(t, rows * n, dtype, what)


def lirpa_ffn_forward(ffn, x, out, keep, g, u, ws, ws_bytes, stream=None):
    rows = x.shape[0]
    dt = _dtype(x, "x")
    if DTYPES[dt] != ffn.dtype:
        raise TypeError(f"x is {dt}, the block's weights are not")
    _check(load().lirpa_ffn_forward(
        ctypes.byref(ffn), rows, *_matrix(x, rows, ffn.n_model, dt, "x"),
        *_matrix(out, rows, ffn.n_model, dt, "out"), int(keep),
        _kept(g, rows, ffn.n_hidden, dt, keep, "g"), _kept(u, rows, ffn.n_hidden, dt, keep, "u"),
        _dev(ws, None, "ws"), int(ws_bytes), _stream(stream)))


def lirpa_ffn_backward(ffn, dout, keep, x, g, u, dx, dWg, dWu, dWd, ws, ws_bytes, stream=None):
    rows = dout.shape[0]
    dt = _dtype(dout, "dout")
    if DTYPES[dt] != ffn.dtype:
        raise TypeError(f"dout is {dt}, the block's weights are not")
    D, F = ffn.n_model, ffn.n_hidden
    px, ldx = (_packed(x, rows, D, "x"), 0) if keep == KEEP_8 else _matrix(x, rows, D, dt, "x")
    _check(load().lirpa_ffn_backward(
        ctypes.byref(ffn), rows, *_matrix(dout, rows, D, dt, "dout"), int(keep), px, ldx,
        _kept(g, rows, F, dt, keep, "g"), _kept(u, rows, F, dt, keep, "u"),
        *_matrix(dx, rows, D, dt, "dx"), _vector(dWg, F * D, dt, "dWg"),
        _vector(dWu, F * D, dt, "dWu"), _vector(dWd, D * F, dt, "dWd"), _dev(ws, None, "ws"),
        int(ws_bytes), _stream(stream)))


_TORCH_TYPES = {code: t for t, code in DTYPES.items()}


def _here(stream, *tensors):
    """The stream's handle (None: torch's current one).  Refuses tensors of another device than the
    current one, whose streams the calls run on; what is no CUDA tensor is refused where its pointer
    is taken."""
    device = -1
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            if device < 0:
                device = torch._C._cuda_getDevice()
            if t.get_device() != device:
                raise ValueError(f"a tensor lies on {t.device}, the current device is "
                                 f"cuda:{device}")
    if stream is not None or device < 0:
        return None if stream is None else _stream(stream)
    return torch._C._cuda_getCurrentRawStream(device)


def _2d(t, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dim() != 2:
        raise ValueError(f"{what} must have two dimensions, got {t.dim()}")
    return t.shape


def _tokens(t, rows):
    if t is not None and isinstance(t, torch.Tensor) and t.dim() != 1:
        raise ValueError(f"tokens must have one dimension, got {t.dim()}")
    return _vector(t, rows, torch.int64, "tokens")


def lirpa_embed_forward(tokens, table, scale, out, stream=None):
    vocab, n = _2d(table, "table")
    rows = _2d(out, "out")[0]
    dt = _dtype(table, "table")
    st = _here(stream, tokens, table, out)
    _check(load().lirpa_embed_forward(
        DTYPES[dt], rows, n, vocab, _tokens(tokens, rows), *_matrix(table, vocab, n, dt, "table"),
        float(scale), *_matrix(out, rows, n, dt, "out"), st))


def lirpa_embed_workspace_bytes(rows, n) -> int:
    return int(load().lirpa_embed_workspace_bytes(int(rows), int(n)))


def lirpa_embed_backward(tokens, dout, scale, base, dtable, ws, ws_bytes, stream=None):
    rows, n = _2d(dout, "dout")
    vocab = _2d(dtable, "dtable")[0]
    dt = _dtype(dout, "dout")
    st = _here(stream, tokens, dout, base, dtable, ws)
    _check(load().lirpa_embed_backward(
        DTYPES[dt], rows, n, vocab, _tokens(tokens, rows), *_matrix(dout, rows, n, dt, "dout"),
        float(scale), *_matrix(base, vocab, n, dt, "base"),
        *_matrix(dtable, vocab, n, dt, "dtable"), _dev(ws, None, "ws"), int(ws_bytes),
        st))


def lirpa_logprob_workspace_bytes(rows, n, top) -> int:
    return int(load().lirpa_logprob_workspace_bytes(int(rows), int(n), int(top)))


def lirpa_logprob_forward(logits, scale, tokens, logp, lse, entropy, top, top_logp, top_tokens, ws,
                          ws_bytes, stream=None):
    rows, n = _2d(logits, "logits")
    dt, f32 = _dtype(logits, "logits"), torch.float32
    st = _here(stream, logits, tokens, logp, lse, entropy, top_logp, top_tokens, ws)
    _check(load().lirpa_logprob_forward(
        DTYPES[dt], rows, n, *_matrix(logits, rows, n, dt, "logits"), float(scale),
        _tokens(tokens, rows), _vector(logp, rows, f32, "logp"), _vector(lse, rows, f32, "lse"),
        _vector(entropy, rows, f32, "entropy"), int(top),
        _vector(top_logp, rows * top, f32, "top_logp"),
        _vector(top_tokens, rows * top, torch.int64, "top_tokens"), _dev(ws, None, "ws"),
        int(ws_bytes), st))


def lirpa_logprob_backward(logits, scale, tokens, lse, entropy, dlogp, dentropy, dlogits,
                           stream=None):
    rows, n = _2d(logits, "logits")
    dt, f32 = _dtype(logits, "logits"), torch.float32
    st = _here(stream, logits, tokens, lse, entropy, dlogp, dentropy, dlogits)
    _check(load().lirpa_logprob_backward(
        DTYPES[dt], rows, n, *_matrix(logits, rows, n, dt, "logits"), float(scale),
        _tokens(tokens, rows), _vector(lse, rows, f32, "lse"),
        _vector(entropy, rows, f32, "entropy"), _vector(dlogp, rows, f32, "dlogp"),
        _vector(dentropy, rows, f32, "dentropy"), *_matrix(dlogits, rows, n, dt, "dlogits"),
        st))


def _seq(seq, rows):
    return _vector(seq, rows, torch.int32, "seq")


def _state(t, rest, dtype, what):
    """(slots, device pointer) of a [slots, *rest] tensor; (None, NULL) of None."""
    if t is None:
        return None, None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a CUDA tensor")
    shape = t.shape
    if len(shape) != 3 or shape[1:] != rest or shape[0] < 1:
        raise ValueError(f"{what} must be [slots, {rest[0]}, {rest[1]}], got {list(shape)}")
    return shape[0], _dev(t, dtype, what)


def _slots(state, state_out, rest, dtype, without=ANY_SLOT):
    """(slots, pointers of state and state_out) of [slots, *rest] tensors; `without`: the slots where
    neither is given."""
    n_in, p_in = _state(state, rest, dtype, "state")
    n_out, p_out = _state(state_out, rest, dtype, "state_out")
    if n_in is not None and n_out is not None and n_in != n_out:
        raise ValueError(f"state has {n_in} slots, state_out {n_out}")
    slots = n_out if n_in is None else n_in
    return without if slots is None else slots, p_in, p_out


def _slot_count(slots):
    if not 1 <= slots <= ANY_SLOT:
        raise ValueError(f"slots must be 1 to 2^31 - 1, got {slots}")
    return slots


def _conv(call, x, w, bias, act, seq, state, state_out, y, stream):
    rows, n = _2d(x, "x")
    taps = _2d(w, "w")[0]
    dt = _dtype(x, "x")
    st = _here(stream, x, w, bias, seq, state, state_out, y)
    if act not in CONV_ACTS:
        raise ValueError(f"act must be one of {sorted(CONV_ACTS)}, got {act!r}")
    slots, s_in, s_out = _slots(state, state_out, (taps - 1, n), dt)
    _check(call(DTYPES[dt], rows, n, taps, *_matrix(x, rows, n, dt, "x"),
                _vector(w, taps * n, dt, "w"), _vector(bias, n, dt, "bias"), CONV_ACTS[act],
                _seq(seq, rows), slots, s_in, s_out, *_matrix(y, rows, n, dt, "y"),
                st))


def lirpa_conv_forward(x, w, bias, act, seq, state, state_out, y, stream=None):
    _conv(load().lirpa_conv_forward, x, w, bias, act, seq, state, state_out, y, stream)


def lirpa_conv_step(x, w, bias, act, seq, state, state_out, y, stream=None):
    _conv(load().lirpa_conv_step, x, w, bias, act, seq, state, state_out, y, stream)


def lirpa_conv_workspace_bytes(rows, n, taps) -> int:
    return int(load().lirpa_conv_workspace_bytes(int(rows), int(n), int(taps)))


def lirpa_conv_backward(dy, x, w, bias, act, seq, dx, dw, dbias, ws, ws_bytes, stream=None,
                        slots=ANY_SLOT):
    """``slots``: those of the forward pass, the number that its states had."""
    rows, n = _2d(x, "x")
    taps = _2d(w, "w")[0]
    dt = _dtype(x, "x")
    st = _here(stream, dy, x, w, bias, seq, dx, dw, dbias, ws)
    if act not in CONV_ACTS:
        raise ValueError(f"act must be one of {sorted(CONV_ACTS)}, got {act!r}")
    _check(load().lirpa_conv_backward(
        DTYPES[dt], rows, n, taps, *_matrix(dy, rows, n, dt, "dy"), *_matrix(x, rows, n, dt, "x"),
        _vector(w, taps * n, dt, "w"), _vector(bias, n, dt, "bias"), CONV_ACTS[act],
        _seq(seq, rows), _slot_count(slots), *_matrix(dx, rows, n, dt, "dx"),
        _vector(dw, taps * n, dt, "dw"), _vector(dbias, n, dt, "dbias"), _dev(ws, None, "ws"),
        int(ws_bytes), st))


def lirpa_scan_inputs(u, dt, B, C, z, A, D, bias, seq, slots=ANY_SLOT):
    """The lirpa_scan of device tensors, which have to outlive the calls that take it.  ``slots``
    holds for calls without states: rows of a number from there on are padding."""
    rows, n = _2d(u, "u")
    states = _2d(A, "A")[1]
    kind, f32 = _dtype(u, "u"), torch.float32
    _here(None, u, dt, B, C, z, A, D, bias, seq)
    pu, ldu = _matrix(u, rows, n, kind, "u")
    pdt, lddt = _matrix(dt, rows, n, kind, "dt")
    pz, ldz = _matrix(z, rows, n, kind, "z")
    pB, ldB = _matrix(B, rows, states, kind, "B")
    pC, ldC = _matrix(C, rows, states, kind, "C")
    return lirpa_scan(DTYPES[kind], rows, n, states, pu, pdt, pz, pB, pC, ldu, lddt, ldz, ldB, ldC,
                      _vector(A, n * states, f32, "A"), _vector(D, n, f32, "D"),
                      _vector(bias, n, f32, "bias"), _seq(seq, rows), _slot_count(slots))


def lirpa_scan_workspace_bytes(rows, n, states, backward) -> int:
    return int(load().lirpa_scan_workspace_bytes(int(rows), int(n), int(states), int(backward)))


def lirpa_scan_kept_bytes(rows, n, states) -> int:
    return int(load().lirpa_scan_kept_bytes(int(rows), int(n), int(states)))


def _of_scan(scan):
    return scan.rows, scan.n, scan.states, _TORCH_TYPES[scan.dtype]


def _kept_states(kept, scan):
    need = lirpa_scan_kept_bytes(scan.rows, scan.n, scan.states)
    if isinstance(kept, torch.Tensor) and kept.numel() * kept.element_size() < need:
        raise ValueError(f"kept must have {need} bytes")
    return _dev(kept, None, "kept")


def _with_slots(scan, slots):
    """The scan with other slots: a caller's struct stays as it is."""
    if slots != scan.slots:
        scan = lirpa_scan.from_buffer_copy(scan)
        scan.slots = slots
    return ctypes.byref(scan)


def lirpa_scan_forward(scan, state, state_out, y, kept, ws, ws_bytes, stream=None):
    """``scan`` is what lirpa_scan_inputs returned.  The slots are those of the states, or the scan's
    without any; ``kept`` is of these, and the scan notes them (kept_slots) for its backward pass."""
    rows, n, states, dt = _of_scan(scan)
    st = _here(stream, state, state_out, y, kept, ws)
    slots, s_in, s_out = _slots(state, state_out, (n, states), torch.float32, scan.slots)
    _check(load().lirpa_scan_forward(
        _with_slots(scan, slots), s_in, s_out, *_matrix(y, rows, n, dt, "y"),
        _kept_states(kept, scan), _dev(ws, None, "ws"), int(ws_bytes), st))
    if kept is not None:
        scan.kept_slots = slots


def lirpa_scan_step(scan, state, state_out, y, stream=None):
    rows, n, states, dt = _of_scan(scan)
    st = _here(stream, state, state_out, y)
    slots, s_in, s_out = _slots(state, state_out, (n, states), torch.float32, scan.slots)
    _check(load().lirpa_scan_step(_with_slots(scan, slots), s_in, s_out,
                                  *_matrix(y, rows, n, dt, "y"), st))


def lirpa_scan_backward(scan, dy, kept, du, ddt, dz, dB, dC, dA, dD, dbias, ws, ws_bytes,
                        stream=None, slots=None):
    """``slots``: those that ``kept`` is of; by default those of the scan's last call that kept, or
    the scan's own."""
    rows, n, states, dt = _of_scan(scan)
    f32 = torch.float32
    st = _here(stream, dy, kept, du, ddt, dz, dB, dC, dA, dD, dbias, ws)
    if slots is None:
        slots = getattr(scan, "kept_slots", scan.slots)
    _check(load().lirpa_scan_backward(
        _with_slots(scan, _slot_count(slots)), *_matrix(dy, rows, n, dt, "dy"),
        _kept_states(kept, scan), *_matrix(du, rows, n, dt, "du"),
        *_matrix(ddt, rows, n, dt, "ddt"), *_matrix(dz, rows, n, dt, "dz"),
        *_matrix(dB, rows, states, dt, "dB"), *_matrix(dC, rows, states, dt, "dC"),
        _vector(dA, n * states, f32, "dA"), _vector(dD, n, f32, "dD"),
        _vector(dbias, n, f32, "dbias"), _dev(ws, None, "ws"), int(ws_bytes), st))


class Network:
    """Device copy of a network (layer dicts with numpy W, b), its handle and a workspace."""

    def __init__(self, layers, device="cuda"):
        self.layers = []
        for t in layers:
            d = dict(t)
            d["W"] = torch.as_tensor(np.ascontiguousarray(t["W"], dtype=np.float32)).to(device)
            d["b"] = torch.as_tensor(np.ascontiguousarray(t["b"], dtype=np.float32)).to(device)
            self.layers.append(d)
        self.device = device
        self.handle = lirpa_net_create(self.layers)
        self.n_relu = lirpa_net_num_relu(self.handle)
        self._ws = None

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and _lib is not None:
            lirpa_net_destroy(h)
            self.handle = None

    def workspace(self, S, B, mode=0, max_bytes=None):
        """A workspace for up to B sub-domains per chunk (capped at max_bytes), reused."""
        need = lirpa_workspace_bytes(self.handle, S, B, mode)
        if max_bytes is not None and need > max_bytes:
            need = max_bytes
        if self._ws is None or self._ws.numel() < need:
            self._ws = None
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws, need

    def bound(self, x0, eps, C, split=None, alpha=None, B=None, want_lu=False, ws=None,
              ws_bytes=None, max_ws_bytes=16 << 30, want_codes=False):
        S = C.shape[0]
        if B is None:
            B = split.shape[0] if split is not None else (alpha.shape[0] if alpha is not None
                                                            else 1)
        lb = torch.empty((B, S), dtype=torch.float32, device=self.device)
        l = u = code = None
        if want_lu:
            l = torch.empty((B, self.n_relu), dtype=torch.float32, device=self.device)
            u = torch.empty_like(l)
        if want_codes:
            code = torch.empty((B, self.n_relu), dtype=torch.int8, device=self.device)
        if ws is None:
            ws, ws_bytes = self.workspace(S, B, 0, max_ws_bytes)
        lirpa_bound(self.handle, x0, eps, C, S, B, split, alpha, lb, l, u, code, ws, ws_bytes)
        out = (lb, l, u) if want_lu else (lb,)
        if want_codes:
            out = out + (code,)
        return out if len(out) > 1 else lb

    def bound_child(self, x0, eps, C, split, alpha, l_parent, u_parent, max_ws_bytes=16 << 30):
        """(lb, l, u, codes) with every layer's bounds intersected with the parent's."""
        S, B = C.shape[0], l_parent.shape[0]
        lb = torch.empty((B, S), dtype=torch.float32, device=self.device)
        l = torch.empty((B, self.n_relu), dtype=torch.float32, device=self.device)
        u = torch.empty_like(l)
        code = torch.empty((B, self.n_relu), dtype=torch.int8, device=self.device)
        ws, ws_bytes = self.workspace(S, B, 0, max_ws_bytes)
        lirpa_bound_child(self.handle, x0, eps, C, S, B, split, alpha, l_parent, u_parent, lb, l,
                          u, code, ws, ws_bytes)
        return lb, l, u, code

    def bound_ul(self, x0, eps, C, split=None, alpha=None, B=None, max_ws_bytes=16 << 30):
        """(lb, ub) [B, S] of the spec rows: Eq. 8's lower and upper bounds in one call."""
        S = C.shape[0]
        if B is None:
            B = split.shape[0] if split is not None else (alpha.shape[0] if alpha is not None
                                                            else 1)
        lb = torch.empty((B, S), dtype=torch.float32, device=self.device)
        ub = torch.empty_like(lb)
        ws, ws_bytes = self.workspace(S, B, 2, max_ws_bytes)
        lirpa_bound_ul(self.handle, x0, eps, C, S, B, split, alpha, lb, ub, None, None, None, ws,
                       ws_bytes)
        return lb, ub

    def optimize_ul(self, x0, eps, C, split, B=None, steps=20, lr=0.1, beta1=0.9, beta2=0.999,
                    eps_adam=1e-8, max_ws_bytes=16 << 30, state=None):
        """Optimised (lb_best, ub_best) from a fresh start (state None) or from the state dict a
        previous call returned (alpha, m, v of both sides, t0); returns (lb, ub, state)."""
        S = C.shape[0]
        B = split.shape[0] if B is None else B
        fresh = state is None
        if fresh:
            state = {k: torch.empty((B, self.n_relu), dtype=torch.float32, device=self.device)
                     for k in ("alpha_lo", "m_lo", "v_lo", "alpha_up", "m_up", "v_up")}
            state["t0"] = 0
        lb = torch.empty((B, S), dtype=torch.float32, device=self.device)
        ub = torch.empty_like(lb)
        ws, ws_bytes = self.workspace(S, B, 3, max_ws_bytes)
        lirpa_optimize_ul(self.handle, x0, eps, C, S, B, split, state["alpha_lo"], state["m_lo"],
                          state["v_lo"], state["alpha_up"], state["m_up"], state["v_up"],
                          lirpa_opt_params(steps, lr, beta1, beta2, eps_adam, state["t0"],
                                           int(fresh)), lb, ub, ws, ws_bytes)
        state = dict(state, t0=state["t0"] + steps)
        return lb, ub, state

    def bab(self, x0, eps, c, batch=64, max_domains=4000, max_iters=30, root_steps=0, steps=0,
            lr=0.1, beta1=0.9, beta2=0.999, eps_adam=1e-8):
        """Branch and bound on c^T f(x) >= 0; returns a dict of the lirpa_bab_result fields."""
        p = lirpa_bab_params(batch, max_domains, max_iters, root_steps, steps, lr, beta1, beta2,
                             eps_adam)
        need = lirpa_bab_workspace_bytes(self.handle, p)
        ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        r = lirpa_bab(self.handle, x0, eps, c, p, ws, need)
        return {k: getattr(r, k) for k, _ in lirpa_bab_result._fields_}

    def bound_grad(self, x0, eps, C, split, alpha, full=True, max_ws_bytes=16 << 30):
        S, B = C.shape[0], alpha.shape[0]
        lb = torch.empty((B, S), dtype=torch.float32, device=self.device)
        grad = torch.empty((B, self.n_relu), dtype=torch.float32, device=self.device)
        ws, ws_bytes = self.workspace(S, B, 1, max_ws_bytes)
        lirpa_bound_grad(self.handle, x0, eps, C, S, B, split, alpha, int(full), lb, grad, ws,
                         ws_bytes)
        return lb, grad

    def optimize(self, x0, eps, C, split, alpha, adam_m=None, adam_v=None, steps=20, lr=0.1,
                 beta1=0.9, beta2=0.999, eps_adam=1e-8, t0=0, trace=False, fresh=False,
                 max_ws_bytes=16 << 30):
        """In place on alpha (and adam_m, adam_v); returns lb_best (and the lb trace)."""
        S, B = C.shape[0], alpha.shape[0]
        if adam_m is None:
            adam_m = torch.zeros_like(alpha)
        if adam_v is None:
            adam_v = torch.zeros_like(alpha)
        best = torch.empty((B, S), dtype=torch.float32, device=self.device)
        tr = torch.empty((steps + 1, B, S), dtype=torch.float32, device=self.device) \
            if trace else None
        ws, ws_bytes = self.workspace(S, B, 1, max_ws_bytes)
        lirpa_optimize(self.handle, x0, eps, C, S, B, split, alpha, adam_m, adam_v,
                       lirpa_opt_params(steps, lr, beta1, beta2, eps_adam, t0, int(fresh)),
                       best, tr, ws,
                       ws_bytes)
        return (best, tr) if trace else best

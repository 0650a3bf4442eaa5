"""Thin ctypes binding of libgleam.so: argument marshalling only.

Every function has the name and argument order of its C declaration in include/gleam.h and
forwards device pointers of torch tensors (torch is used for device memory and streams only).
There is no CPU path: if the shared library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgleam.so")

GLEAM_OK = 0
GLEAM_E_NULL = -1
GLEAM_E_DIMS = -2
GLEAM_E_UNSUPPORTED_SIZE = -3
GLEAM_E_WORKSPACE = -4
GLEAM_E_DESC = -5
GLEAM_E_LAUNCH = -6


class gleam_geom(C.Structure):
    _fields_ = [("ndim_fft", C.c_int32), ("centred", C.c_int32), ("B", C.c_int64), ("C", C.c_int64), ("T", C.c_int64),
                ("D", C.c_int64), ("H", C.c_int64), ("W", C.c_int64)]


class gleam_conv(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("cin", "cout", "kt", "kd", "kh", "kw", "relu_in", "relu_out",
                                         "has_bias", "skip_src")]


class gleam_prox_desc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layers", C.POINTER(gleam_conv)), ("dtype", C.c_int32),
                ("loss_kind", C.c_int32)]


class gleam_kernel_record(C.Structure):
    _fields_ = [("name", C.c_char * 56), ("flops", C.c_double), ("bytes", C.c_double), ("mfma_flops", C.c_double),
                ("ms", C.c_float)]


class gleam_adam(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float)]


class gleam_layer_norm_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("eps", C.c_float), ("rows", C.c_int64), ("n", C.c_int64), ("ld_in", C.c_int64),
                ("ld_out", C.c_int64)]


class gleam_dropout_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("p", C.c_float), ("rows", C.c_int64), ("n", C.c_int64), ("ld_in", C.c_int64),
                ("ld_res", C.c_int64), ("ld_out", C.c_int64), ("seed", C.c_uint64), ("offset", C.c_uint64)]


class gleam_seq_strides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("b", "t", "p", "h")]


class gleam_linattn_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "heads", "q_heads", "k_heads", "v_heads", "dk", "dv")] + [("scale", C.c_float)] +
                [(n, C.c_int64) for n in ("B", "T", "P")] + [(n, gleam_seq_strides) for n in ("q", "k", "v", "o")])


class GleamError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


_lib = None


def lib() -> C.CDLL:
    """Loads libgleam.so (built by paper_2207_08393_amd/csrc/build.sh); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run paper_2207_08393_amd/csrc/build.sh "
                               "(or __graft_entry__.build()); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        pg, pp = C.POINTER(gleam_geom), C.POINTER(gleam_prox_desc)
        L.gleam_strerror.restype = C.c_char_p
        L.gleam_strerror.argtypes = [C.c_int]
        L.gleam_fft_size_supported.argtypes = [C.c_int64]
        L.gleam_set_kernel_policy.argtypes = [C.c_uint32]
        L.gleam_get_kernel_policy.argtypes = []
        L.gleam_get_kernel_policy.restype = C.c_uint32
        L.gleam_theta_count.argtypes = [pp, C.POINTER(sz)]
        L.gleam_workspace_bytes.argtypes = [pg, pp, C.POINTER(sz), C.POINTER(sz)]
        L.gleam_sense_normal.argtypes = [pg, vp, vp, vp, vp, vp, sz, vp]
        L.gleam_sense_normal_static.argtypes = [pg, vp, vp, vp, vp, vp]
        L.gleam_module_fwd.argtypes = [pg, pp, vp, vp, vp, vp, C.c_float, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.gleam_module_bwd.argtypes = [pg, pp, vp, vp, sz, vp, vp, sz, vp]
        L.gleam_module_bwd_alpha.argtypes = [pg, pp, vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, sz, vp]
        L.gleam_deep_workspace_bytes.argtypes = [pg, pp, C.c_int, C.POINTER(sz), C.POINTER(sz)]
        L.gleam_deep_module_fwd.argtypes = [pg, pp, C.c_int, vp, vp, vp, vp, C.c_float, vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.gleam_deep_module_bwd.argtypes = [pg, pp, C.c_int, vp, vp, C.c_float, vp, vp, sz, vp, vp, sz, vp]
        L.gleam_sense_adjoint.argtypes = [pg, vp, vp, vp, vp, vp, sz, vp]
        L.gleam_kspace_to_hybrid.argtypes = [pg, vp, vp, vp]
        L.gleam_mask_constant_along_outer_axis.argtypes = [pg, vp, C.POINTER(C.c_int)]
        L.gleam_modl_workspace_bytes.argtypes = [pg, pp, C.POINTER(sz), C.POINTER(sz)]
        L.gleam_modl_module_fwd.argtypes = [pg, pp, vp, vp, vp, vp, C.c_float, C.c_int, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.gleam_modl_module_bwd.argtypes = [pg, pp, vp, vp, C.c_float, C.c_int, vp, vp, sz, vp, vp, sz, vp]
        L.gleam_adam_step.argtypes = [C.POINTER(gleam_adam), C.c_int64, sz, vp, vp, vp, vp, vp]
        L.gleam_greedy_iteration.argtypes = [pg, pp, C.c_int, vp, vp, vp, vp, C.c_float, vp, vp, vp, C.POINTER(gleam_adam),
                                             C.c_int64, vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.gleam_unrolled_infer.argtypes = [pg, pp, C.c_int, vp, vp, vp, vp, C.c_float, vp, vp, vp, vp, sz, vp]
        pn, pd, pl = C.POINTER(gleam_layer_norm_desc), C.POINTER(gleam_dropout_desc), C.POINTER(gleam_linattn_desc)
        L.gleam_layer_norm_fwd.argtypes = [pn, vp, vp, vp, vp, vp, vp, vp]
        L.gleam_layer_norm_workspace_bytes.argtypes = [pn, C.POINTER(sz)]
        L.gleam_layer_norm_bwd.argtypes = [pn, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gleam_dropout_fwd.argtypes = [pd, vp, vp, vp, vp, vp]
        L.gleam_dropout_bwd.argtypes = [pd, vp, vp, vp, vp]
        L.gleam_linattn_workspace_bytes.argtypes = [pl, C.POINTER(sz), C.POINTER(sz)]
        L.gleam_linattn_fwd.argtypes = [pl, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gleam_linattn_bwd.argtypes = [pl, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.gleam_profile_begin.argtypes = []
        L.gleam_profile_end.argtypes = [C.POINTER(gleam_kernel_record), C.c_int, C.POINTER(C.c_int)]
        _lib = L
    return _lib


EXPORTS = ("gleam_strerror", "gleam_fft_size_supported", "gleam_set_kernel_policy", "gleam_get_kernel_policy", "gleam_theta_count", "gleam_workspace_bytes",
           "gleam_sense_normal", "gleam_sense_normal_static", "gleam_module_fwd", "gleam_module_bwd", "gleam_module_bwd_alpha", "gleam_deep_workspace_bytes",
           "gleam_deep_module_fwd", "gleam_deep_module_bwd", "gleam_sense_adjoint", "gleam_kspace_to_hybrid",
           "gleam_mask_constant_along_outer_axis", "gleam_modl_workspace_bytes",
           "gleam_modl_module_fwd", "gleam_modl_module_bwd", "gleam_adam_step",
           "gleam_greedy_iteration", "gleam_unrolled_infer", "gleam_layer_norm_fwd", "gleam_layer_norm_workspace_bytes", "gleam_layer_norm_bwd",
           "gleam_dropout_fwd", "gleam_dropout_bwd", "gleam_linattn_workspace_bytes", "gleam_linattn_fwd", "gleam_linattn_bwd",
           "gleam_profile_begin", "gleam_profile_end")


def strerror(status: int) -> str:
    return lib().gleam_strerror(int(status)).decode()


def make_geom(g) -> gleam_geom:
    """From any object with ndim_fft, B, C, T, D, H, W (and optionally centred) attributes."""
    return gleam_geom(int(g.ndim_fft), int(getattr(g, "centred", 0)), int(g.B), int(g.C), int(g.T), int(g.D), int(g.H), int(g.W))


def make_prox(p) -> gleam_prox_desc:
    """From any object with `layers` (cin, cout, kt, kd, kh, kw, relu_in, relu_out, has_bias, skip_src),
    `dtype` and `loss_kind`.  The returned struct keeps its layer array alive."""
    arr = (gleam_conv * len(p.layers))()
    for i, l in enumerate(p.layers):
        arr[i] = gleam_conv(l.cin, l.cout, l.kt, l.kd, l.kh, l.kw, l.relu_in, l.relu_out, l.has_bias, l.skip_src)
    d = gleam_prox_desc(len(p.layers), C.cast(arr, C.POINTER(gleam_conv)), int(p.dtype), int(p.loss_kind))
    d._keep = arr
    return d


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors passed to libgleam must be contiguous")
    return t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        # the handle itself: building a Stream object around it took 2.8 of the 14 us of a small operator call, this takes 0.3
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _check(rc: int, where: str):
    if rc != GLEAM_OK:
        raise GleamError(rc, where)


POLICY_NO_WINOGRAD, POLICY_NO_BF16_2D, POLICY_NO_THIN_MFMA, POLICY_NO_WGRAD_BALANCE, POLICY_NO_FRAME_WALK = 1, 2, 4, 8, 16


def gleam_set_kernel_policy(policy: int):
    _check(lib().gleam_set_kernel_policy(int(policy)), "gleam_set_kernel_policy")


def gleam_get_kernel_policy() -> int:
    return int(lib().gleam_get_kernel_policy())


def gleam_fft_size_supported(n: int) -> bool:
    return bool(lib().gleam_fft_size_supported(int(n)))


def gleam_theta_count(prox: gleam_prox_desc) -> int:
    n = C.c_size_t(0)
    _check(lib().gleam_theta_count(C.byref(prox), C.byref(n)), "gleam_theta_count")
    return n.value


def gleam_workspace_bytes(geom: gleam_geom, prox: Optional[gleam_prox_desc]):
    ws, saved = C.c_size_t(0), C.c_size_t(0)
    _check(lib().gleam_workspace_bytes(C.byref(geom), C.byref(prox) if prox is not None else None,
                                       C.byref(ws), C.byref(saved)), "gleam_workspace_bytes")
    return ws.value, saved.value


def gleam_sense_normal(geom, x, S, M, out, ws, stream=None):
    _check(lib().gleam_sense_normal(C.byref(geom), _ptr(x), _ptr(S), _ptr(M), _ptr(out), _ptr(ws), _nbytes(ws),
                                    _stream(stream)), "gleam_sense_normal")


STATIC_SCRATCH_BYTES = 64 << 20   # GLEAM_STATIC_SCRATCH_BYTES of include/gleam.h


def gleam_sense_normal_static(geom, x, S, M, out, stream=None):
    _check(lib().gleam_sense_normal_static(C.byref(geom), _ptr(x), _ptr(S), _ptr(M), _ptr(out), _stream(stream)),
           "gleam_sense_normal_static")


def gleam_module_fwd(geom, prox, x_in, S, M, y, alpha, theta, x_ref, x_out, loss, saved, ws, stream=None):
    _check(lib().gleam_module_fwd(C.byref(geom), C.byref(prox), _ptr(x_in), _ptr(S), _ptr(M), _ptr(y),
                                  C.c_float(alpha), _ptr(theta), _ptr(x_ref), _ptr(x_out), _ptr(loss),
                                  _ptr(saved), _nbytes(saved), _ptr(ws), _nbytes(ws), _stream(stream)),
           "gleam_module_fwd")


def gleam_module_bwd(geom, prox, theta, saved, grad_theta, ws, stream=None):
    _check(lib().gleam_module_bwd(C.byref(geom), C.byref(prox), _ptr(theta), _ptr(saved), _nbytes(saved),
                                  _ptr(grad_theta), _ptr(ws), _nbytes(ws), _stream(stream)), "gleam_module_bwd")


def gleam_module_bwd_alpha(geom, prox, x_in, S, M, y, theta, saved, grad_theta, grad_alpha, ws, stream=None):
    _check(lib().gleam_module_bwd_alpha(C.byref(geom), C.byref(prox), _ptr(x_in), _ptr(S), _ptr(M), _ptr(y), _ptr(theta),
                                        _ptr(saved), _nbytes(saved), _ptr(grad_theta), _ptr(grad_alpha), _ptr(ws),
                                        _nbytes(ws), _stream(stream)), "gleam_module_bwd_alpha")


def gleam_deep_workspace_bytes(geom, prox, n_iter):
    ws, saved = C.c_size_t(0), C.c_size_t(0)
    _check(lib().gleam_deep_workspace_bytes(C.byref(geom), C.byref(prox), int(n_iter), C.byref(ws), C.byref(saved)),
           "gleam_deep_workspace_bytes")
    return ws.value, saved.value


def gleam_deep_module_fwd(geom, prox, n_iter, x_in, S, M, y, alpha, theta, x_ref, x_out, x_tmp, loss, saved, ws, stream=None):
    _check(lib().gleam_deep_module_fwd(C.byref(geom), C.byref(prox), int(n_iter), _ptr(x_in), _ptr(S), _ptr(M), _ptr(y),
                                       C.c_float(alpha), _ptr(theta), _ptr(x_ref), _ptr(x_out), _ptr(x_tmp), _ptr(loss),
                                       _ptr(saved), _nbytes(saved), _ptr(ws), _nbytes(ws), _stream(stream)),
           "gleam_deep_module_fwd")


def gleam_deep_module_bwd(geom, prox, n_iter, S, M, alpha, theta, saved, grad_theta, ws, stream=None):
    _check(lib().gleam_deep_module_bwd(C.byref(geom), C.byref(prox), int(n_iter), _ptr(S), _ptr(M), C.c_float(alpha),
                                       _ptr(theta), _ptr(saved), _nbytes(saved), _ptr(grad_theta), _ptr(ws), _nbytes(ws),
                                       _stream(stream)), "gleam_deep_module_bwd")


def gleam_sense_adjoint(geom, S, M, y, out, ws, stream=None):
    _check(lib().gleam_sense_adjoint(C.byref(geom), _ptr(S), _ptr(M), _ptr(y), _ptr(out), _ptr(ws), _nbytes(ws),
                                     _stream(stream)), "gleam_sense_adjoint")


def gleam_kspace_to_hybrid(geom, y_in, y_out, stream=None):
    _check(lib().gleam_kspace_to_hybrid(C.byref(geom), _ptr(y_in), _ptr(y_out), _stream(stream)), "gleam_kspace_to_hybrid")


def gleam_mask_constant_along_outer_axis(geom, mask_host) -> bool:
    """mask_host: contiguous uint8 numpy array [B][T][D][H][W] in host memory."""
    import numpy as np
    m = np.ascontiguousarray(mask_host, dtype=np.uint8)
    if m.size != geom.B * geom.T * geom.D * geom.H * geom.W:
        raise ValueError("mask size does not match the geometry")
    out = C.c_int(0)
    _check(lib().gleam_mask_constant_along_outer_axis(C.byref(geom), m.ctypes.data_as(C.c_void_p), C.byref(out)),
           "gleam_mask_constant_along_outer_axis")
    return bool(out.value)


def gleam_modl_workspace_bytes(geom, prox):
    ws, saved = C.c_size_t(0), C.c_size_t(0)
    _check(lib().gleam_modl_workspace_bytes(C.byref(geom), C.byref(prox), C.byref(ws), C.byref(saved)),
           "gleam_modl_workspace_bytes")
    return ws.value, saved.value


def gleam_modl_module_fwd(geom, prox, x_in, S, M, aty, mu, n_cg, theta, x_ref, x_out, loss, saved, ws, stream=None):
    _check(lib().gleam_modl_module_fwd(C.byref(geom), C.byref(prox), _ptr(x_in), _ptr(S), _ptr(M), _ptr(aty), C.c_float(mu),
                                       int(n_cg), _ptr(theta), _ptr(x_ref), _ptr(x_out), _ptr(loss), _ptr(saved),
                                       _nbytes(saved), _ptr(ws), _nbytes(ws), _stream(stream)), "gleam_modl_module_fwd")


def gleam_modl_module_bwd(geom, prox, S, M, mu, n_cg, theta, saved, grad_theta, ws, stream=None):
    _check(lib().gleam_modl_module_bwd(C.byref(geom), C.byref(prox), _ptr(S), _ptr(M), C.c_float(mu), int(n_cg),
                                       _ptr(theta), _ptr(saved), _nbytes(saved), _ptr(grad_theta), _ptr(ws), _nbytes(ws),
                                       _stream(stream)), "gleam_modl_module_bwd")


def make_adam(lr, beta1=0.9, beta2=0.999, eps=1e-8) -> gleam_adam:
    return gleam_adam(float(lr), float(beta1), float(beta2), float(eps))


def gleam_adam_step(hyper, t, theta, grad, m, v, stream=None):
    _check(lib().gleam_adam_step(C.byref(hyper), int(t), theta.numel(), _ptr(theta), _ptr(grad), _ptr(m), _ptr(v),
                                 _stream(stream)), "gleam_adam_step")


def gleam_greedy_iteration(geom, prox, n_modules, x0, S, M, y, alpha, theta, adam_m, adam_v, hyper, t, x_ref, x_out,
                           x_tmp, losses, grad, saved, ws, stream=None):
    _check(lib().gleam_greedy_iteration(C.byref(geom), C.byref(prox), int(n_modules), _ptr(x0), _ptr(S), _ptr(M), _ptr(y),
                                        C.c_float(alpha), _ptr(theta), _ptr(adam_m), _ptr(adam_v), C.byref(hyper), int(t),
                                        _ptr(x_ref), _ptr(x_out), _ptr(x_tmp), _ptr(losses), _ptr(grad), _ptr(saved),
                                        _nbytes(saved), _ptr(ws), _nbytes(ws), _stream(stream)), "gleam_greedy_iteration")


def gleam_unrolled_infer(geom, prox, n_modules, x0, S, M, y, alpha, theta, x_out, x_tmp, ws, stream=None):
    _check(lib().gleam_unrolled_infer(C.byref(geom), C.byref(prox), int(n_modules), _ptr(x0), _ptr(S), _ptr(M), _ptr(y),
                                      C.c_float(alpha), _ptr(theta), _ptr(x_out), _ptr(x_tmp), _ptr(ws), _nbytes(ws),
                                      _stream(stream)), "gleam_unrolled_infer")


# ---- layer norm, dropout, linear attention: arrays may have strides, so what a call reads is checked against its description
def _dtype_code(dtype) -> int:
    """0 or 1 from a code or from torch.float32 / torch.bfloat16."""
    import torch
    code = {torch.float32: 0, torch.bfloat16: 1, 0: 0, 1: 1}.get(dtype)
    if code is None:
        raise ValueError(f"dtype {dtype}: float32 (0) and bfloat16 (1) have kernels")
    return code


_DTYPES = []


def _types():
    """torch types of the codes 0, 1 (activations), 2 (lengths), 3 (counters)."""
    if not _DTYPES:
        import torch
        _DTYPES.extend((torch.float32, torch.bfloat16, torch.int32, torch.int64))
    return _DTYPES


def _flat(t, code: int, count: int, what: str) -> Optional[int]:
    """Address of a contiguous device array of `count` elements of type code 0 / 1 (2: int32, 3: int64 words)."""
    if t is None or type(t) is int:
        return t
    if t.dtype is not _types()[code] or t.numel() != count or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: {t.numel()} elements of {t.dtype} on {t.device} with strides {t.stride()}, {count} contiguous ones of "
                         f"{_types()[code]} on the GPU expected")
    return t.data_ptr()


def _rows(t, code: int, rows: int, n: int, ld: int, what: str) -> Optional[int]:
    """A rows x n array with `ld` elements from row to row: contiguous (ld = n) of any shape, or two-dimensional with that stride."""
    if t is None or type(t) is int:
        return t
    if ld == n and t.is_contiguous():
        return _flat(t, code, rows * n, what)
    if (t.shape != (rows, n) or (n > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) != ld) or t.dtype is not _types()[code] or
            not t.is_cuda):
        raise ValueError(f"{what}: shape {tuple(t.shape)} with strides {t.stride()} of {t.dtype} on {t.device}, the description has {rows} rows "
                         f"of {n}, {ld} apart, of {_types()[code]} on the GPU")
    return t.data_ptr()


def make_layer_norm(dtype, rows, n, eps=1e-5, ld=None, ld_out=None) -> gleam_layer_norm_desc:
    """ld: elements from row to row of x and g_x (default n); ld_out: of y and g_y (default ld)."""
    ld = n if ld is None else ld
    return gleam_layer_norm_desc(_dtype_code(dtype), float(eps), int(rows), int(n), int(ld), int(ld if ld_out is None else ld_out))


def gleam_layer_norm_fwd(desc, x, gamma, beta, y, mean=None, rstd=None, stream=None):
    rows, n = desc.rows, desc.n
    _check(lib().gleam_layer_norm_fwd(C.byref(desc), _rows(x, desc.dtype, rows, n, desc.ld_in, "x"), _flat(gamma, 0, n, "gamma"),
                                      _flat(beta, 0, n, "beta"), _rows(y, desc.dtype, rows, n, desc.ld_out, "y"),
                                      _flat(mean, 0, rows, "mean"), _flat(rstd, 0, rows, "rstd"), _stream(stream)),
           "gleam_layer_norm_fwd")


def gleam_layer_norm_workspace_bytes(desc) -> int:
    n = C.c_size_t(0)
    _check(lib().gleam_layer_norm_workspace_bytes(C.byref(desc), C.byref(n)), "gleam_layer_norm_workspace_bytes")
    return n.value


def gleam_layer_norm_bwd(desc, x, gamma, mean, rstd, g_y, g_x, g_gamma, g_beta, ws, stream=None):
    rows, n = desc.rows, desc.n
    _check(lib().gleam_layer_norm_bwd(C.byref(desc), _rows(x, desc.dtype, rows, n, desc.ld_in, "x"), _flat(gamma, 0, n, "gamma"),
                                      _flat(mean, 0, rows, "mean"), _flat(rstd, 0, rows, "rstd"),
                                      _rows(g_y, desc.dtype, rows, n, desc.ld_out, "g_y"),
                                      _rows(g_x, desc.dtype, rows, n, desc.ld_in, "g_x"), _flat(g_gamma, 0, n, "g_gamma"),
                                      _flat(g_beta, 0, n, "g_beta"), _ptr(ws), _nbytes(ws), _stream(stream)), "gleam_layer_norm_bwd")


def make_dropout(dtype, rows, n, p, seed, offset=0, ld=None, ld_res=None, ld_out=None) -> gleam_dropout_desc:
    """ld: elements from row to row of x and g_x (default n); ld_res, ld_out: of residual, of out and g_out (default ld)."""
    ld = n if ld is None else ld
    return gleam_dropout_desc(_dtype_code(dtype), float(p), int(rows), int(n), int(ld), int(ld if ld_res is None else ld_res),
                              int(ld if ld_out is None else ld_out), int(seed), int(offset))


def gleam_dropout_fwd(desc, x, residual, out, step=None, stream=None):
    """step: int64 tensor of one element on the device, added to the offset, or None."""
    rows, n = desc.rows, desc.n
    _check(lib().gleam_dropout_fwd(C.byref(desc), _rows(x, desc.dtype, rows, n, desc.ld_in, "x"),
                                   _rows(residual, desc.dtype, rows, n, desc.ld_res, "residual"),
                                   _rows(out, desc.dtype, rows, n, desc.ld_out, "out"), _flat(step, 3, 1, "step"), _stream(stream)),
           "gleam_dropout_fwd")


def gleam_dropout_bwd(desc, g_out, g_x, step=None, stream=None):
    rows, n = desc.rows, desc.n
    _check(lib().gleam_dropout_bwd(C.byref(desc), _rows(g_out, desc.dtype, rows, n, desc.ld_out, "g_out"),
                                   _rows(g_x, desc.dtype, rows, n, desc.ld_in, "g_x"), _flat(step, 3, 1, "step"), _stream(stream)),
           "gleam_dropout_bwd")


def make_linattn(q, k, v, o, scale=1.0) -> gleam_linattn_desc:
    """From the arrays of a call, or others of their shapes and strides: [B][T][P][heads][width] with any strides but the last.
    Gradients have the strides of the arrays they belong to."""
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if t.dim() != 5 or t.dtype is not o.dtype or t.shape[:3] != o.shape[:3] or (t.shape[4] > 1 and t.stride(4) != 1):
            raise ValueError(f"{name}: [B][T][P][heads][width] of one type with contiguous widths expected, got {tuple(t.shape)} with strides "
                             f"{t.stride()} of {t.dtype}")
    if q.shape[4] != k.shape[4] or v.shape[4] != o.shape[4]:
        raise ValueError("q and k, and v and o, have the same width")
    B, T, P, H, dv = o.shape
    return gleam_linattn_desc(_dtype_code(o.dtype), H, q.shape[3], k.shape[3], v.shape[3], q.shape[4], dv, float(scale), B, T, P,
                              *(gleam_seq_strides(*t.stride()[:4]) for t in (q, k, v, o)))


def _want(desc):
    """What the arrays of a call have to be: {name: (shape, strides, type)} of q, k, v and o, kept with the description it was made for."""
    key, (made_for, want) = bytes(desc), getattr(desc, "_want", (None, None))
    if made_for != key:
        want = {}
        for name, heads, width in (("q", desc.q_heads, desc.dk), ("k", desc.k_heads, desc.dk), ("v", desc.v_heads, desc.dv), ("o", desc.heads, desc.dv)):
            s = getattr(desc, name)
            want[name] = ((desc.B, desc.T, desc.P, heads, width), (s.b, s.t, s.p, s.h, 1), _types()[desc.dtype])
        desc._want = key, want
    return want


def _seq(t, want, what: str) -> Optional[int]:
    if t is None or type(t) is int:
        return t
    shape, strides, dtype = want
    got = t.stride()
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or (
            got != strides and any(n > 1 and x != y for n, x, y in zip(shape, got, strides))):
        raise ValueError(f"{what}: shape {tuple(t.shape)} with strides {got} of {t.dtype} on {t.device}, the description has {shape} with strides "
                         f"{strides} of {dtype} on the GPU")
    return t.data_ptr()


def gleam_linattn_workspace_bytes(desc):
    """(forward, backward) bytes; 0: no workspace needed."""
    fwd, bwd = C.c_size_t(0), C.c_size_t(0)
    _check(lib().gleam_linattn_workspace_bytes(C.byref(desc), C.byref(fwd), C.byref(bwd)), "gleam_linattn_workspace_bytes")
    return fwd.value, bwd.value


def gleam_linattn_fwd(desc, q, k, v, log_decay, lengths, state_in, o, state_out, ws, stream=None):
    H, want = desc.heads, _want(desc)
    state = desc.B * desc.P * H * desc.dk * desc.dv
    _check(lib().gleam_linattn_fwd(C.byref(desc), _seq(q, want["q"], "q"), _seq(k, want["k"], "k"), _seq(v, want["v"], "v"),
                                   _flat(log_decay, 0, H, "log_decay"), _flat(lengths, 2, desc.B, "lengths"),
                                   _flat(state_in, 0, state, "state_in"), _seq(o, want["o"], "o"), _flat(state_out, 0, state, "state_out"),
                                   _ptr(ws), _nbytes(ws), _stream(stream)), "gleam_linattn_fwd")


def gleam_linattn_bwd(desc, q, k, v, log_decay, lengths, state_in, g_o, g_state_out, g_q, g_k, g_v, g_state_in, ws, stream=None):
    H, want = desc.heads, _want(desc)
    state = desc.B * desc.P * H * desc.dk * desc.dv
    _check(lib().gleam_linattn_bwd(C.byref(desc), _seq(q, want["q"], "q"), _seq(k, want["k"], "k"), _seq(v, want["v"], "v"),
                                   _flat(log_decay, 0, H, "log_decay"), _flat(lengths, 2, desc.B, "lengths"),
                                   _flat(state_in, 0, state, "state_in"), _seq(g_o, want["o"], "g_o"),
                                   _flat(g_state_out, 0, state, "g_state_out"), _seq(g_q, want["q"], "g_q"), _seq(g_k, want["k"], "g_k"),
                                   _seq(g_v, want["v"], "g_v"), _flat(g_state_in, 0, state, "g_state_in"), _ptr(ws), _nbytes(ws),
                                   _stream(stream)), "gleam_linattn_bwd")


def gleam_profile_begin():
    _check(lib().gleam_profile_begin(), "gleam_profile_begin")


def gleam_profile_end(capacity: int = 65536):
    """Returns a list of (name, flops, bytes, ms, mfma_flops), one per kernel launch since gleam_profile_begin."""
    arr = (gleam_kernel_record * capacity)()
    n = C.c_int(0)
    _check(lib().gleam_profile_end(arr, capacity, C.byref(n)), "gleam_profile_end")
    return [(arr[i].name.decode(), arr[i].flops, arr[i].bytes, arr[i].ms, arr[i].mfma_flops)
            for i in range(min(n.value, capacity))]

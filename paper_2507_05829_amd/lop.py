"""ctypes binding of liblop.so (see include/lop.h). Argument marshalling only: every
step of the path runs inside the library's HIP kernels. There is no fallback: if the
library is not built, importing this module raises.

Module-level functions carry the C names (lop_plan, lop_run_band, lop_run_chain, ...);
``Plan`` is a small convenience wrapper over the same calls. Device and pinned-host
buffers are torch tensors used purely as memory; their ``data_ptr()`` is what crosses the
boundary. ``quantize_blocks``, ``rowwise_f8``, ``head_norm_rope`` and ``attention`` are the calls of
the same names on torch tensors, whose types, shapes and strides they pass on.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import POINTER, Structure, byref, c_char_p, c_double, c_float, c_int, c_longlong, c_size_t, c_uint, c_ulonglong, c_void_p
from operator import index
from typing import List, Optional, Sequence, Tuple

import numpy as np
# torch ships its own HIP runtime; it has to be in the process before liblop.so is
# loaded so that both resolve to the same runtime (device pointers and streams are
# shared between them).
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblop.so")

LOP_OK = 0
LOP_ERR_INVALID_ARG, LOP_ERR_UNSUPPORTED, LOP_ERR_SHAPE, LOP_ERR_BAND_RANGE = -1, -2, -3, -4
LOP_ERR_OOM, LOP_ERR_HIP, LOP_ERR_NOT_READY, LOP_ERR_TOO_LARGE = -5, -6, -7, -8
LOP_STATIC_SCRATCH_BYTES = 64 << 20
LOP_CONV2D, LOP_DWCONV2D, LOP_MAXPOOL2D, LOP_ELTWISE = 0, 1, 2, 3
LOP_ACT_NONE, LOP_ACT_RELU, LOP_ACT_RELU6 = 0, 1, 2
LOP_F32, LOP_BF16 = 0, 1
LOP_INPUT, LOP_NO_RESIDUAL = -1, -2
LOP_MAX_BANDS = 64
LOP_FLAG_NO_D2H, LOP_FLAG_PLAN_ONLY, LOP_FLAG_GRAPH, LOP_FLAG_DMA_COPY = 1, 2, 4, 8
LOP_FLAG_REUSE = 16
LOP_FLAG_INDEPENDENT = 0
LOP_FLAG_NO_FUSE = 32
LOP_FLAG_POISON_SCRATCH = 64
LOP_FLAG_BATCH_BANDS = 128
LOP_LINK_INDEPENDENT, LOP_LINK_QUEUED = 0, 1
LOP_F8_BLOCK, LOP_ATTENTION_CUT, LOP_ATTENTION_CUT_F32 = 128, 512, 64


def LOP_FLAG_LANES(n: int) -> int:
    return (n & 0xFF) << 8


EXPORTS = [
    "lop_plan", "lop_plan_out_desc", "lop_plan_layer_desc", "lop_plan_n_bands",
    "lop_plan_n_layers", "lop_plan_band_out_rows", "lop_plan_band_in_rows",
    "lop_plan_band_layer_rows", "lop_plan_stats", "lop_plan_layer_work", "lop_run_band",
    "lop_run_chain", "lop_synchronize", "lop_time_layer", "lop_plan_destroy", "lop_strerror",
    "lop_last_hip_error", "lop_plan_layer_kernel", "lop_profile_chain", "lop_copy_chain",
    "lop_plan_band_compute_rows", "lop_plan_rowwise", "lop_loss_eval", "lop_loss_solve",
    "lop_run_two_party", "lop_measure_ceilings", "lop_run_chain_static", "lop_debug_guard_check",
    "lop_quantize_blocks", "lop_rowwise_f8", "lop_rowwise_f8_kernel", "lop_head_norm_rope", "lop_attention_workspace", "lop_attention",
]


class lop_layer_t(Structure):
    _fields_ = [("op", c_int), ("c_in", c_int), ("c_out", c_int),
                ("kh", c_int), ("kw", c_int), ("sh", c_int), ("sw", c_int),
                ("ph", c_int), ("pw", c_int), ("dh", c_int), ("dw", c_int),
                ("act", c_int), ("input_from", c_int), ("residual_from", c_int),
                ("weight", c_void_p), ("bias", c_void_p)]


class lop_rowwise_t(Structure):
    _fields_ = [("k", c_int), ("n", c_int), ("act", c_int), ("input_from", c_int),
                ("residual_from", c_int), ("weight", c_void_p), ("bias", c_void_p)]


class lop_loss_layer_t(Structure):
    _fields_ = [("n_ops", c_int), ("input_from", c_int), ("residual_from", c_int),
                ("k", c_int), ("s", c_int), ("p", c_int), ("d", c_int),
                ("cm_fixed", c_double), ("cm_row", c_double), ("cr_fixed", c_double),
                ("cr_row", c_double), ("row_bytes", c_double)]


class lop_loss_alloc_t(Structure):
    _fields_ = [("m_lo", c_int), ("m_hi", c_int), ("r_lo", c_int), ("r_hi", c_int)]


class lop_two_party_stats_t(Structure):
    _fields_ = [("total_ms", c_float), ("bytes_to_m", c_double), ("bytes_to_r", c_double),
                ("transfers", c_int)]


class lop_ceilings_t(Structure):
    _fields_ = [("hbm_copy_gbs", c_double), ("mfma_bf16_tflops", c_double), ("mfma_f32_tflops", c_double),
                ("launch_floor_us", c_double), ("graph_node_floor_us", c_double)]


class lop_quantize_t(Structure):
    _fields_ = [("m", c_int), ("k", c_int), ("dtype", c_int), ("block_rows", c_int),
                ("x", c_void_p), ("x_stride", c_longlong), ("q", c_void_p), ("q_stride", c_longlong),
                ("scale", c_void_p), ("scale_row", c_longlong), ("scale_col", c_longlong)]


class lop_rowwise_f8_t(Structure):
    _fields_ = [("m", c_int), ("n", c_int), ("k", c_int), ("dtype", c_int), ("act", c_int),
                ("x", c_void_p), ("x_stride", c_longlong),
                ("x_scale", c_void_p), ("x_scale_row", c_longlong), ("x_scale_col", c_longlong),
                ("w", c_void_p), ("w_stride", c_longlong),
                ("w_scale", c_void_p), ("w_scale_row", c_longlong), ("w_scale_col", c_longlong),
                ("bias", c_void_p), ("residual", c_void_p), ("residual_stride", c_longlong),
                ("y", c_void_p), ("y_stride", c_longlong)]


class lop_head_norm_rope_t(Structure):
    _fields_ = [("tokens", c_int), ("heads_q", c_int), ("heads_k", c_int), ("head_dim", c_int),
                ("rot_dim", c_int), ("interleaved", c_int), ("dtype", c_int),
                ("eps", c_float), ("amplitude", c_float),
                ("q", c_void_p), ("q_token", c_longlong), ("q_head", c_longlong),
                ("k", c_void_p), ("k_token", c_longlong), ("k_head", c_longlong),
                ("q_out", c_void_p), ("q_out_token", c_longlong), ("q_out_head", c_longlong),
                ("k_out", c_void_p), ("k_out_token", c_longlong), ("k_out_head", c_longlong),
                ("q_weight", c_void_p), ("k_weight", c_void_p), ("positions", c_void_p), ("freq", c_void_p)]


class lop_attention_t(Structure):
    _fields_ = [("dtype", c_int), ("heads_q", c_int), ("heads_k", c_int), ("head_dim", c_int),
                ("seqs", c_int), ("rows_q", c_int), ("rows_k", c_int), ("max_keys", c_int),
                ("causal", c_int), ("scale", c_float),
                ("q", c_void_p), ("q_token", c_longlong), ("q_head", c_longlong),
                ("k", c_void_p), ("k_token", c_longlong), ("k_head", c_longlong),
                ("v", c_void_p), ("v_token", c_longlong), ("v_head", c_longlong),
                ("out", c_void_p), ("out_token", c_longlong), ("out_head", c_longlong),
                ("q_offsets", c_void_p), ("k_begin", c_void_p), ("k_end", c_void_p), ("lse", c_void_p),
                ("workspace", c_void_p), ("workspace_bytes", c_ulonglong)]


class lop_tensor_desc_t(Structure):
    _fields_ = [("n", c_int), ("c", c_int), ("h", c_int), ("w", c_int), ("dtype", c_int)]


class lop_rows_t(Structure):
    _fields_ = [("lo", c_int), ("hi", c_int)]


class lop_timing_t(Structure):
    _fields_ = [("n_bands", c_int), ("wall_ms", c_float), ("compute_ms", c_float),
                ("copy_ms", c_float), ("band_compute_ms", c_float * LOP_MAX_BANDS),
                ("band_copy_ms", c_float * LOP_MAX_BANDS),
                ("band_ready_ms", c_float * LOP_MAX_BANDS)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2507_05829_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    P = c_void_p
    sig = {
        "lop_plan": (c_int, [POINTER(lop_layer_t), c_int, POINTER(lop_tensor_desc_t), c_int, c_uint,
                             POINTER(P)]),
        "lop_plan_rowwise": (c_int, [POINTER(lop_rowwise_t), c_int, c_int, c_int, c_int, c_int, c_uint,
                                     POINTER(P)]),
        "lop_loss_eval": (c_int, [POINTER(lop_loss_layer_t), c_int, c_int, c_double, c_double, c_double,
                                  POINTER(lop_loss_alloc_t), POINTER(c_double), POINTER(c_double),
                                  POINTER(c_double), POINTER(c_int), c_int]),
        "lop_loss_solve": (c_int, [POINTER(lop_loss_layer_t), c_int, c_int, c_double, c_double, c_double,
                                   c_int, c_int, ctypes.c_ulonglong, POINTER(lop_loss_alloc_t),
                                   POINTER(c_double), POINTER(c_int), c_int]),
        "lop_plan_out_desc": (c_int, [P, POINTER(lop_tensor_desc_t)]),
        "lop_plan_layer_desc": (c_int, [P, c_int, POINTER(lop_tensor_desc_t)]),
        "lop_plan_n_bands": (c_int, [P]),
        "lop_plan_n_layers": (c_int, [P]),
        "lop_plan_band_out_rows": (c_int, [P, c_int, POINTER(lop_rows_t)]),
        "lop_plan_band_in_rows": (c_int, [P, c_int, POINTER(lop_rows_t)]),
        "lop_plan_band_layer_rows": (c_int, [P, c_int, c_int, POINTER(lop_rows_t)]),
        "lop_plan_band_compute_rows": (c_int, [P, c_int, c_int, POINTER(lop_rows_t)]),
        "lop_plan_stats": (c_int, [P, POINTER(c_double), POINTER(c_double), POINTER(c_size_t)]),
        "lop_plan_layer_work": (c_int, [P, c_int, c_int, POINTER(c_double), POINTER(c_double)]),
        "lop_run_band": (c_int, [P, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
        "lop_run_chain": (c_int, [P, c_void_p, c_void_p, c_void_p, c_void_p, POINTER(lop_timing_t)]),
        "lop_run_chain_static": (c_int, [P, c_void_p, c_void_p, c_void_p]),
        "lop_synchronize": (c_int, [P]),
        "lop_time_layer": (c_int, [P, c_int, c_int, c_void_p, c_void_p, c_int, POINTER(c_float)]),
        "lop_plan_destroy": (None, [P]),
        "lop_plan_layer_kernel": (c_int, [P, c_int, c_int, ctypes.c_char_p, c_size_t, POINTER(c_int)]),
        "lop_profile_chain": (c_int, [P, c_void_p, c_void_p, c_int, POINTER(c_float), POINTER(c_float)]),
        "lop_copy_chain": (c_int, [P, c_void_p, c_void_p]),
        "lop_run_two_party": (c_int, [P, c_void_p, c_void_p, POINTER(lop_loss_alloc_t), c_int,
                                      POINTER(lop_loss_layer_t), c_double, c_double,
                                      POINTER(lop_two_party_stats_t)]),
        "lop_measure_ceilings": (c_int, [POINTER(lop_ceilings_t)]),
        "lop_quantize_blocks": (c_int, [c_void_p, c_longlong, c_void_p]),
        "lop_rowwise_f8": (c_int, [c_void_p, c_longlong, c_void_p]),
        "lop_rowwise_f8_kernel": (c_int, [c_void_p, c_longlong, c_char_p, c_size_t]),
        "lop_head_norm_rope": (c_int, [c_void_p, c_longlong, c_void_p]),
        "lop_attention_workspace": (c_int, [c_void_p, c_longlong, POINTER(c_ulonglong)]),
        "lop_attention": (c_int, [c_void_p, c_longlong, c_void_p]),
        "lop_debug_guard_check": (c_int, []),
        "lop_strerror": (c_char_p, [c_int]),
        "lop_last_hip_error": (c_int, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


class LopError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = _lib.lop_strerror(code).decode()
        if code == LOP_ERR_HIP:
            msg += f" (hipError_t {_lib.lop_last_hip_error()})"
        super().__init__(f"{where}: {msg} [{code}]")


def _check(code: int, where: str) -> None:
    if code != LOP_OK:
        raise LopError(code, where)


def _ptr(t) -> c_void_p:
    """Raw address of a torch tensor / numpy array / int / None."""
    if t is None:
        return c_void_p(0)
    if isinstance(t, int):
        return c_void_p(t)
    if hasattr(t, "data_ptr"):
        return c_void_p(t.data_ptr())
    return c_void_p(t.ctypes.data)


def _stream(s) -> c_void_p:
    if s is None:
        return c_void_p(0)
    if isinstance(s, int):
        return c_void_p(s)
    return c_void_p(s.cuda_stream)


# ------------------------------------------------------------------ C-named functions

def lop_plan(layers: Sequence[lop_layer_t], in_desc: lop_tensor_desc_t, n_bands: int,
             flags: int = 0) -> c_void_p:
    arr = (lop_layer_t * len(layers))(*layers) if len(layers) else None
    out = c_void_p(0)
    _check(_lib.lop_plan(arr, len(layers), byref(in_desc), n_bands, flags, byref(out)), "lop_plan")
    return out


def lop_plan_rowwise(layers: Sequence[lop_rowwise_t], m: int, k: int, dtype: int, n_bands: int,
                     flags: int = 0) -> c_void_p:
    arr = (lop_rowwise_t * len(layers))(*layers) if len(layers) else None
    out = c_void_p(0)
    _check(_lib.lop_plan_rowwise(arr, len(layers), m, k, dtype, n_bands, flags, byref(out)),
           "lop_plan_rowwise")
    return out


def _loss_layers(layers):
    """lop_loss_layer_t array from objects with the fields of the struct (duck-typed)."""
    return (lop_loss_layer_t * len(layers))(*[
        lop_loss_layer_t(L.n_ops, L.input_from, L.residual_from, L.k, L.s, L.p, L.d,
                         L.cm_fixed, L.cm_row, L.cr_fixed, L.cr_row, L.row_bytes) for L in layers])


def lop_loss_eval(layers, in_rows: int, in_row_bytes: float, bandwidth: float, latency: float,
                  sched: Sequence[Tuple[Tuple[int, int], Tuple[int, int]]], link_model: int = 0):
    """sched: per vertex ((m_lo, m_hi), (r_lo, r_hi)). Returns (T, s_m, s_r, violations)."""
    n = len(layers)
    arr = (lop_loss_alloc_t * n)(*[lop_loss_alloc_t(m[0], m[1], r[0], r[1]) for m, r in sched])
    T, viol = c_double(0.0), c_int(0)
    s_m, s_r = (c_double * (n + 1))(), (c_double * n)()
    _check(_lib.lop_loss_eval(_loss_layers(layers), n, in_rows, in_row_bytes, bandwidth, latency,
                              arr, byref(T), s_m, s_r, byref(viol), link_model), "lop_loss_eval")
    return T.value, list(s_m), list(s_r), viol.value


def lop_loss_solve(layers, in_rows: int, in_row_bytes: float, bandwidth: float, latency: float,
                   population: int = 0, generations: int = 200, seed: int = 1, link_model: int = 0):
    """Returns (schedule as in lop_loss_eval, T, violations)."""
    n = len(layers)
    best = (lop_loss_alloc_t * n)()
    T, viol = c_double(0.0), c_int(0)
    _check(_lib.lop_loss_solve(_loss_layers(layers), n, in_rows, in_row_bytes, bandwidth, latency,
                               population, generations, seed, best, byref(T), byref(viol), link_model),
           "lop_loss_solve")
    return [((a.m_lo, a.m_hi), (a.r_lo, a.r_hi)) for a in best], T.value, viol.value


def lop_plan_destroy(plan) -> None:
    _lib.lop_plan_destroy(plan)


def lop_plan_out_desc(plan) -> lop_tensor_desc_t:
    d = lop_tensor_desc_t()
    _check(_lib.lop_plan_out_desc(plan, byref(d)), "lop_plan_out_desc")
    return d


def lop_plan_layer_desc(plan, layer: int) -> lop_tensor_desc_t:
    d = lop_tensor_desc_t()
    _check(_lib.lop_plan_layer_desc(plan, layer, byref(d)), "lop_plan_layer_desc")
    return d


def lop_plan_n_bands(plan) -> int:
    return _lib.lop_plan_n_bands(plan)


def lop_plan_n_layers(plan) -> int:
    return _lib.lop_plan_n_layers(plan)


def _rows(fn, name, *args) -> Tuple[int, int]:
    r = lop_rows_t()
    _check(fn(*args, byref(r)), name)
    return (r.lo, r.hi)


def lop_plan_band_out_rows(plan, band: int) -> Tuple[int, int]:
    return _rows(_lib.lop_plan_band_out_rows, "lop_plan_band_out_rows", plan, band)


def lop_plan_band_in_rows(plan, band: int) -> Tuple[int, int]:
    return _rows(_lib.lop_plan_band_in_rows, "lop_plan_band_in_rows", plan, band)


def lop_plan_band_layer_rows(plan, band: int, layer: int) -> Tuple[int, int]:
    return _rows(_lib.lop_plan_band_layer_rows, "lop_plan_band_layer_rows", plan, band, layer)


def lop_plan_band_compute_rows(plan, band: int, layer: int) -> Tuple[int, int]:
    return _rows(_lib.lop_plan_band_compute_rows, "lop_plan_band_compute_rows", plan, band, layer)


def lop_plan_stats(plan) -> Tuple[float, float, int]:
    u, e, s = c_double(), c_double(), c_size_t()
    _check(_lib.lop_plan_stats(plan, byref(u), byref(e), byref(s)), "lop_plan_stats")
    return u.value, e.value, s.value


def lop_plan_layer_work(plan, band: int, layer: int) -> Tuple[float, float]:
    f, b = c_double(), c_double()
    _check(_lib.lop_plan_layer_work(plan, band, layer, byref(f), byref(b)), "lop_plan_layer_work")
    return f.value, b.value


def lop_run_band(plan, band: int, d_in, d_out, h_out=None, compute_stream=None,
                 copy_stream=None) -> None:
    _check(_lib.lop_run_band(plan, band, _ptr(d_in), _ptr(d_out), _ptr(h_out),
                             _stream(compute_stream), _stream(copy_stream)), "lop_run_band")


def lop_run_chain(plan, d_in, d_out, h_out=None, compute_stream=None,
                  timing: bool = False) -> Optional[lop_timing_t]:
    t = lop_timing_t() if timing else None
    _check(_lib.lop_run_chain(plan, _ptr(d_in), _ptr(d_out), _ptr(h_out), _stream(compute_stream),
                              byref(t) if timing else None), "lop_run_chain")
    return t


def lop_run_chain_static(plan, d_in, d_out, stream=None) -> None:
    _check(_lib.lop_run_chain_static(plan, _ptr(d_in), _ptr(d_out), _stream(stream)), "lop_run_chain_static")


def lop_synchronize(plan) -> None:
    _check(_lib.lop_synchronize(plan), "lop_synchronize")


def lop_time_layer(plan, band: int, layer: int, d_in, d_out, iters: int = 20) -> float:
    ms = c_float()
    _check(_lib.lop_time_layer(plan, band, layer, _ptr(d_in), _ptr(d_out), iters, byref(ms)),
           "lop_time_layer")
    return ms.value


def lop_plan_layer_kernel(plan, band: int, layer: int) -> Tuple[str, int]:
    """(kernel instance name, number of K slices) of a (band, layer) launch."""
    buf = ctypes.create_string_buffer(128)
    k = c_int(0)
    _check(_lib.lop_plan_layer_kernel(plan, band, layer, buf, 128, byref(k)), "lop_plan_layer_kernel")
    return buf.value.decode(), k.value


def lop_profile_chain(plan, d_in, d_out, iters: int = 5) -> Tuple[np.ndarray, np.ndarray]:
    """Mean ms of every (band, layer) main kernel and of its split-K finish kernel."""
    nb, nl = lop_plan_n_bands(plan), lop_plan_n_layers(plan)
    ms = np.zeros((nb, nl), np.float32)
    fin = np.zeros((nb, nl), np.float32)
    _check(_lib.lop_profile_chain(plan, _ptr(d_in), _ptr(d_out), iters,
                                  ms.ctypes.data_as(POINTER(c_float)),
                                  fin.ctypes.data_as(POINTER(c_float))), "lop_profile_chain")
    return ms, fin


def lop_copy_chain(plan, d_out, h_out) -> None:
    _check(_lib.lop_copy_chain(plan, _ptr(d_out), _ptr(h_out)), "lop_copy_chain")


def lop_run_two_party(plan, d_in, d_out, sched, bandwidth: float, latency: float = 0.0, costs=None):
    """sched: per layer ((m_lo, m_hi), (r_lo, r_hi)); costs: objects with the lop_loss_layer_t
    fields or None. Returns the filled lop_two_party_stats_t."""
    n = len(sched)
    arr = (lop_loss_alloc_t * n)(*[lop_loss_alloc_t(m[0], m[1], r[0], r[1]) for m, r in sched])
    st = lop_two_party_stats_t()
    _check(_lib.lop_run_two_party(plan, _ptr(d_in), _ptr(d_out), arr, n,
                                  _loss_layers(costs) if costs is not None else None,
                                  bandwidth, latency, byref(st)), "lop_run_two_party")
    return st


def lop_measure_ceilings() -> lop_ceilings_t:
    c = lop_ceilings_t()
    _check(_lib.lop_measure_ceilings(byref(c)), "lop_measure_ceilings")
    return c


def _rows_word(lo: int, hi: int) -> int:
    """A lop_rows_t that is passed by value, as the register it travels in (two 32-bit integers, the first in the low half). Numbers that
    they do not hold are no band's: -1, as every negative number."""
    lo, hi = index(lo), index(hi)
    return -1 if (lo | hi) >> 31 else lo | hi << 32


def lop_quantize_blocks(op: lop_quantize_t, rows: Tuple[int, int], stream=None) -> None:
    _check(_lib.lop_quantize_blocks(byref(op), _rows_word(*rows), _stream(stream)), "lop_quantize_blocks")


def lop_rowwise_f8(op: lop_rowwise_f8_t, rows: Tuple[int, int], stream=None) -> None:
    _check(_lib.lop_rowwise_f8(byref(op), _rows_word(*rows), _stream(stream)), "lop_rowwise_f8")


def lop_rowwise_f8_kernel(op: lop_rowwise_f8_t, rows: Tuple[int, int]) -> str:
    """Name of the kernel instance that lop_rowwise_f8 runs."""
    buf = ctypes.create_string_buffer(128)
    _check(_lib.lop_rowwise_f8_kernel(byref(op), _rows_word(*rows), buf, 128), "lop_rowwise_f8_kernel")
    return buf.value.decode()


def lop_head_norm_rope(op: lop_head_norm_rope_t, rows: Tuple[int, int], stream=None) -> None:
    _check(_lib.lop_head_norm_rope(byref(op), _rows_word(*rows), _stream(stream)), "lop_head_norm_rope")


def lop_attention_workspace(op: lop_attention_t, rows: Tuple[int, int]) -> int:
    n = c_ulonglong(0)
    _check(_lib.lop_attention_workspace(byref(op), _rows_word(*rows), byref(n)), "lop_attention_workspace")
    return n.value


def lop_attention(op: lop_attention_t, rows: Tuple[int, int], stream=None) -> None:
    _check(_lib.lop_attention(byref(op), _rows_word(*rows), _stream(stream)), "lop_attention")


def lop_debug_guard_check() -> int:
    return _lib.lop_debug_guard_check()


def lop_strerror(code: int) -> str:
    return _lib.lop_strerror(code).decode()


# ------------------------------------------------------------------ chain marshalling

_OPS = {"conv": LOP_CONV2D, "dwconv": LOP_DWCONV2D, "maxpool": LOP_MAXPOOL2D, "eltwise": LOP_ELTWISE}
_ACTS = {"none": LOP_ACT_NONE, "relu": LOP_ACT_RELU, "relu6": LOP_ACT_RELU6}
_DTYPES = {"f32": LOP_F32, "bf16": LOP_BF16}


def _storage(a: np.ndarray, dtype: str) -> np.ndarray:
    """float32 values -> the storage type's bytes (bf16: the upper 16 bits, which is exact
    because the values are already bfloat16-representable)."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    if dtype == "f32":
        return a
    u = a.view(np.uint32)
    if np.any(u & 0xFFFF):
        raise ValueError("bf16 plan: values must be bfloat16-representable")
    return (u >> 16).astype(np.uint16)


def layers_from_chain(chain, tensors=None):
    """lop_layer_t list from a chain description (duck-typed: .layers with op, c_in, c_out,
    k, s, p, d, act, input_from, residual_from) and optional host tensors. Returns the list
    and the numpy arrays that must stay alive until lop_plan returns."""
    keep, out = [], []
    for i, L in enumerate(chain.layers):
        d = lop_layer_t(_OPS[L.op], L.c_in, L.c_out, L.k[0], L.k[1], L.s[0], L.s[1],
                        L.p[0], L.p[1], L.d[0], L.d[1], _ACTS[L.act], L.input_from,
                        L.residual_from, None, None)
        if tensors is not None:
            if tensors.weights[i] is not None:
                w = _storage(tensors.weights[i], chain.dtype)
                keep.append(w)
                d.weight = w.ctypes.data
            if tensors.biases[i] is not None:
                b = np.ascontiguousarray(tensors.biases[i], dtype=np.float32)
                keep.append(b)
                d.bias = b.ctypes.data
        out.append(d)
    return out, keep


class Plan:
    """Owns a lop_plan_t handle."""

    def __init__(self, chain, tensors=None, n_bands: Optional[int] = None, flags: int = 0):
        layers, keep = layers_from_chain(chain, tensors)
        n, c, h, w = chain.in_shape
        desc = lop_tensor_desc_t(n, c, h, w, _DTYPES[chain.dtype])
        if tensors is None:
            flags |= LOP_FLAG_PLAN_ONLY
        self.handle = lop_plan(layers, desc, chain.n_bands if n_bands is None else n_bands, flags)
        del keep
        self.n_bands = lop_plan_n_bands(self.handle)
        self.n_layers = lop_plan_n_layers(self.handle)
        self.dtype = chain.dtype

    @classmethod
    def rowwise(cls, chain, tensors=None, n_bands: Optional[int] = None, flags: int = 0) -> "Plan":
        """Plan for a chain of row-wise operators (duck-typed: .m, .k, .dtype, .n_bands and
        .layers with k, n, act, input_from, residual_from) through lop_plan_rowwise."""
        keep, layers = [], []
        for i, L in enumerate(chain.layers):
            d = lop_rowwise_t(L.k, L.n, _ACTS[L.act], L.input_from, L.residual_from, None, None)
            if tensors is not None:
                w = _storage(tensors.weights[i], chain.dtype)
                keep.append(w)
                d.weight = w.ctypes.data
                if tensors.biases[i] is not None:
                    b = np.ascontiguousarray(tensors.biases[i], dtype=np.float32)
                    keep.append(b)
                    d.bias = b.ctypes.data
            layers.append(d)
        if tensors is None:
            flags |= LOP_FLAG_PLAN_ONLY
        self = cls.__new__(cls)
        self.handle = lop_plan_rowwise(layers, chain.m, chain.k, _DTYPES[chain.dtype],
                                       chain.n_bands if n_bands is None else n_bands, flags)
        del keep
        self.n_bands = lop_plan_n_bands(self.handle)
        self.n_layers = lop_plan_n_layers(self.handle)
        self.dtype = chain.dtype
        return self

    def destroy(self) -> None:
        if getattr(self, "handle", None):
            _lib.lop_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:      # interpreter shutdown: the library may already be gone
            pass

    def out_shape(self) -> Tuple[int, int, int, int]:
        d = lop_plan_out_desc(self.handle)
        return (d.n, d.c, d.h, d.w)

    def layer_shape(self, layer: int) -> Tuple[int, int, int, int]:
        d = lop_plan_layer_desc(self.handle, layer)
        return (d.n, d.c, d.h, d.w)

    def band_out_rows(self, b): return lop_plan_band_out_rows(self.handle, b)
    def band_in_rows(self, b): return lop_plan_band_in_rows(self.handle, b)
    def band_layer_rows(self, b, l): return lop_plan_band_layer_rows(self.handle, b, l)
    def band_compute_rows(self, b, l): return lop_plan_band_compute_rows(self.handle, b, l)
    def stats(self): return lop_plan_stats(self.handle)
    def layer_work(self, b, l): return lop_plan_layer_work(self.handle, b, l)

    def run_band(self, band, d_in, d_out, h_out=None, compute_stream=None, copy_stream=None):
        lop_run_band(self.handle, band, d_in, d_out, h_out, compute_stream, copy_stream)

    def run_chain(self, d_in, d_out, h_out=None, compute_stream=None, timing=False):
        return lop_run_chain(self.handle, d_in, d_out, h_out, compute_stream, timing)

    def run_chain_static(self, d_in, d_out, stream=None):
        lop_run_chain_static(self.handle, d_in, d_out, stream)

    def synchronize(self): lop_synchronize(self.handle)

    def layer_kernel(self, b, l): return lop_plan_layer_kernel(self.handle, b, l)
    def profile_chain(self, d_in, d_out, iters=5): return lop_profile_chain(self.handle, d_in, d_out, iters)
    def copy_chain(self, d_out, h_out): lop_copy_chain(self.handle, d_out, h_out)

    def run_two_party(self, d_in, d_out, sched, bandwidth, latency=0.0, costs=None):
        return lop_run_two_party(self.handle, d_in, d_out, sched, bandwidth, latency, costs)

    def time_layer(self, band, layer, d_in, d_out, iters=20):
        return lop_time_layer(self.handle, band, layer, d_in, d_out, iters)


# ------------------------------------------------------------------ operators on torch tensors
#
# lop_quantize_blocks, lop_rowwise_f8, lop_head_norm_rope and lop_attention on tensors: the descriptor is read off
# them. They run on torch's current stream of the current device, where every tensor has to be; outputs that are not
# passed are allocated there. `rows`: the band of output rows that is computed (lo, hi), everything if None. Forward
# only: a tensor that wants a gradient is refused while gradients are recorded, and one with a tangent always. Shapes and types that do not fit
# raise ValueError, what the library refuses LopError.

# (the library's host code also runs beside a stand-in for torch that has no tensors)
_TYPES = {getattr(torch, n): c for n, c in (("float32", LOP_F32), ("bfloat16", LOP_BF16)) if hasattr(torch, n)}
_F8 = getattr(torch, "float8_e4m3fn", None)


def _bad(name: str, what: str):
    raise ValueError(f"{name}: {what}")


def _refuse(device: int, grad: int, *named) -> None:
    """Says what is wrong with the first of (name, tensor, type, shape, rows) that does not fit: `shape` None for any, or with None
    for any extent; `rows`: the values of a row lie next to one another (2: all of them do)."""
    for name, t, dtype, shape, rows in named:
        if t is None:
            continue
        if t.dtype is not dtype:
            _bad(name, f"{dtype} is wanted, not {t.dtype}")
        if shape is not None and (len(shape) != t.dim() or any(a is not None and a != b for a, b in zip(shape, t.shape))):
            _bad(name, f"{tuple(shape)} is wanted, not {tuple(t.shape)}")
        if t.get_device() != device:
            _bad(name, f"on {t.device}, not on the current device ({device})")
        if grad & 1 and t.requires_grad:
            _bad(name, "forward only, but the tensor wants a gradient")
        if grad & 2 and _forward_ad.unpack_dual(t).tangent is not None:
            _bad(name, "no derivatives, but the tensor has a tangent")
        if rows == 2 and not t.is_contiguous():
            _bad(name, "dense memory is wanted")
        if rows and t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel() > 0:
            _bad(name, "the values of a row have to lie next to one another")


def _dtype(name: str, t: torch.Tensor) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        _bad(name, f"float32 or bfloat16 is wanted, not {t.dtype}")
    return code


def _dims(name: str, t, n: int):
    if t.dim() != n:
        _bad(name, f"{n} dimensions are wanted, not {t.dim()}")
    return t.shape


_current_device, _current_stream, _grad_enabled, _forward_ad = (
    (torch.cuda.current_device, torch._C._cuda_getCurrentRawStream, torch.is_grad_enabled, torch.autograd.forward_ad) if _TYPES else (None,) * 4)


def _here():
    """The current device, its current stream, and 1 where gradients are recorded + 2 where tensors may have tangents (a level of forward-mode
    derivatives is open: then _refuse looks at every tensor)."""
    device = _current_device()
    return device, _current_stream(device), _grad_enabled() if _forward_ad._current_level < 0 else _grad_enabled() + 2


def _no_number(e: struct.error):
    raise ValueError(f"a size, stride or factor that the library does not hold: {e}") from e


# Each function first asks in one expression whether everything fits, and goes through the tensors one by one only where
# something does not: a call of one token is bound by the host. (The descriptors are packed for the same reason:
# filling the fields of a ctypes structure takes four times as long.)
_QUANTIZE = struct.Struct("@4iPqPqP2q")
_ROWWISE_F8 = struct.Struct("@5iPqP2qPqP2q2PqPq")
_HEAD_NORM_ROPE = struct.Struct("@7i2fP2qP2qP2qP2q4P")
_ATTENTION = struct.Struct("@9ifP2qP2qP2qP2q5PQ")


def quantize_blocks(x, block_rows: int = 1, q=None, scale=None, rows=None):
    """x (m, k) in e4m3 with a scale for each block of `block_rows` x 128 values (see lop_quantize_blocks). Returns
    (q, scale): q float8_e4m3fn (m, k), scale float32 (ceil(m / block_rows), ceil(k / 128)), allocated with the scales
    of a column of blocks next to one another."""
    device, stream, grad = _here()
    code, shape = _TYPES.get(x.dtype) or _dtype("x", x), x.shape
    m, k = shape if len(shape) == 2 else _dims("x", x, 2)
    if block_rows != 1 and block_rows != LOP_F8_BLOCK:
        _bad("block_rows", f"1 or {LOP_F8_BLOCK}")
    blocks = (-(-m // block_rows), -(-k // LOP_F8_BLOCK))
    if q is None:
        q = torch.empty((m, k), dtype=_F8, device=x.device)
    if scale is None:
        scale = torch.empty(blocks[::-1], dtype=torch.float32, device=x.device).t()
    xs, qs, ss = x.stride(), q.stride(), scale.stride()
    if (q.dtype is not _F8 or scale.dtype is not torch.float32 or q.shape != shape or scale.shape != blocks
            or x.get_device() != device or q.get_device() != device or scale.get_device() != device
            or (grad and (grad > 1 or x.requires_grad or q.requires_grad or scale.requires_grad)) or xs[1] != 1 or qs[1] != 1):
        _refuse(device, grad, ("x", x, x.dtype, None, 1), ("q", q, _F8, shape, 1), ("scale", scale, torch.float32, blocks, 0))
    try:
        op = _QUANTIZE.pack(m, k, code, block_rows, x.data_ptr(), xs[0], q.data_ptr(), qs[0], scale.data_ptr(), ss[0], ss[1])
    except struct.error as e:
        _no_number(e)
    e = _lib.lop_quantize_blocks(op, m << 32 if rows is None else _rows_word(*rows), stream)
    if e:
        _check(e, "lop_quantize_blocks")
    return q, scale


def rowwise_f8(x, x_scale, w, w_scale, bias=None, act: str = "none", residual=None, y=None, dtype=None, rows=None):
    """act(x W^T + bias + residual) of operands quantized by quantize_blocks: x (m, k) with blocks of one row, w (n, k)
    with blocks of 128 rows (see lop_rowwise_f8). y (m, n) is allocated in `dtype` (None: bfloat16) if it is not passed."""
    device, stream, grad = _here()
    x_shape, w_shape = x.shape, w.shape
    m, k = x_shape if len(x_shape) == 2 else _dims("x", x, 2)
    n, kw = w_shape if len(w_shape) == 2 else _dims("w", w, 2)
    kb = -(-k // LOP_F8_BLOCK)
    if act not in _ACTS:
        _bad("act", f"one of {sorted(_ACTS)}")
    if y is None:
        y = torch.empty((m, n), dtype=dtype or torch.bfloat16, device=x.device)
    dtype, f32 = y.dtype, torch.float32
    code = _TYPES.get(dtype) or _dtype("y", y)
    xs, ws, ys, xss, wss = x.stride(), w.stride(), y.stride(), x_scale.stride(), w_scale.stride()
    if (x.dtype is not _F8 or w.dtype is not _F8 or x_scale.dtype is not f32 or w_scale.dtype is not f32 or kw != k
            or x_scale.shape != (m, kb) or w_scale.shape != (-(-n // LOP_F8_BLOCK), kb) or y.shape != (m, n)
            or x.get_device() != device or w.get_device() != device or x_scale.get_device() != device
            or w_scale.get_device() != device or y.get_device() != device
            or (grad and (grad > 1 or x.requires_grad or w.requires_grad or x_scale.requires_grad or w_scale.requires_grad or y.requires_grad))
            or xs[1] != 1 or ws[1] != 1 or ys[1] != 1):
        _refuse(device, grad, ("x", x, _F8, None, 1), ("w", w, _F8, (n, k), 1), ("x_scale", x_scale, f32, (m, kb), 0),
                ("w_scale", w_scale, f32, (-(-n // LOP_F8_BLOCK), kb), 0), ("y", y, dtype, (m, n), 1))
    bias_at = residual_at = residual_stride = 0
    if bias is not None:
        _refuse(device, grad, ("bias", bias, f32, (n,), 1))
        bias_at = bias.data_ptr()
    if residual is not None:
        _refuse(device, grad, ("residual", residual, dtype, (m, n), 1))
        residual_at, residual_stride = residual.data_ptr(), residual.stride(0)
    try:
        op = _ROWWISE_F8.pack(m, n, k, code, _ACTS[act], x.data_ptr(), xs[0], x_scale.data_ptr(), xss[0], xss[1], w.data_ptr(), ws[0],
                              w_scale.data_ptr(), wss[0], wss[1], bias_at, residual_at, residual_stride, y.data_ptr(), ys[0])
    except struct.error as e:
        _no_number(e)
    e = _lib.lop_rowwise_f8(op, m << 32 if rows is None else _rows_word(*rows), stream)
    if e:
        _check(e, "lop_rowwise_f8")
    return y


def head_norm_rope(q, k, positions, freq, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                   amplitude: float = 1.0, q_out=None, k_out=None, rows=None):
    """q (tokens, heads_q, d) and k (tokens, heads_k, d) or None, each head normalized (where its weight (d,) is given) and its first
    2 * len(freq) values rotated by positions * freq (see lop_head_norm_rope). positions int32 (tokens,), freq float32,
    both None for no rotation. Returns (q_out, k_out), which may be q and k."""
    device, stream, grad = _here()
    dtype, f32, shape = q.dtype, torch.float32, q.shape
    code = _TYPES.get(dtype) or _dtype("q", q)
    tokens, hq, d = shape if len(shape) == 3 else _dims("q", q, 3)
    if q_out is None:
        q_out = torch.empty(shape, dtype=dtype, device=q.device)
    qs, qos = q.stride(), q_out.stride()
    if (q_out.dtype is not dtype or q_out.shape != shape or q.get_device() != device or q_out.get_device() != device
            or (grad and (grad > 1 or q.requires_grad or q_out.requires_grad)) or qs[2] != 1 or qos[2] != 1):
        _refuse(device, grad, ("q", q, dtype, None, 1), ("q_out", q_out, dtype, shape, 1))
    hk = k_at = k_out_at = 0
    ks = kos = (0, 0)
    if k is not None:
        k_shape = _dims("k", k, 3)
        hk = k_shape[1]
        if k_out is None:
            k_out = torch.empty(k_shape, dtype=dtype, device=q.device)
        ks, kos = k.stride(), k_out.stride()
        if (k.dtype is not dtype or k_out.dtype is not dtype or k_shape[0] != tokens or k_shape[2] != d or k_out.shape != k_shape
                or k.get_device() != device or k_out.get_device() != device or (grad and (grad > 1 or k.requires_grad or k_out.requires_grad))
                or ks[2] != 1 or kos[2] != 1):
            _refuse(device, grad, ("k", k, dtype, (tokens, hk, d), 1), ("k_out", k_out, dtype, k_shape, 1))
        k_at, k_out_at = k.data_ptr(), k_out.data_ptr()
    turns = positions_at = freq_at = q_weight_at = k_weight_at = 0
    if freq is not None and positions is not None:
        turns = freq.numel()
        if (positions.dtype is not torch.int32 or freq.dtype is not f32 or freq.dim() != 1 or positions.shape != (tokens,)
                or positions.get_device() != device or freq.get_device() != device or grad > 1 or freq.requires_grad
                or positions.stride(0) != 1 or freq.stride(0) != 1):
            _refuse(device, grad, ("positions", positions, torch.int32, (tokens,), 1), ("freq", freq, f32, (None,), 1))
        positions_at, freq_at = positions.data_ptr(), freq.data_ptr()
    elif freq is not None or positions is not None:
        _bad("positions", "they and freq go together")
    if q_weight is not None:
        if (q_weight.dtype is not f32 or q_weight.shape != (d,) or q_weight.get_device() != device or grad > 1 or q_weight.requires_grad
                or q_weight.stride(0) != 1):
            _refuse(device, grad, ("q_weight", q_weight, f32, (d,), 1))
        q_weight_at = q_weight.data_ptr()
    if k_weight is not None:
        if (k_weight.dtype is not f32 or k_weight.shape != (d,) or k_weight.get_device() != device or grad > 1 or k_weight.requires_grad
                or k_weight.stride(0) != 1):
            _refuse(device, grad, ("k_weight", k_weight, f32, (d,), 1))
        k_weight_at = k_weight.data_ptr()
    try:
        op = _HEAD_NORM_ROPE.pack(tokens, hq, hk, d, 2 * turns, interleaved, code, eps, amplitude, q.data_ptr(), qs[0], qs[1],
                                  k_at, ks[0], ks[1], q_out.data_ptr(), qos[0], qos[1], k_out_at, kos[0], kos[1],
                                  q_weight_at, k_weight_at, positions_at, freq_at)
    except struct.error as e:
        _no_number(e)
    e = _lib.lop_head_norm_rope(op, tokens << 32 if rows is None else _rows_word(*rows), stream)
    if e:
        _check(e, "lop_head_norm_rope")
    return q_out, k_out


def attention(q, k, v, q_offsets, k_begin, k_end, scale: float, causal: bool = True, max_keys: Optional[int] = None, out=None, lse=None,
              workspace=None, rows=None):
    """softmax(scale q k^T) v of packed sequences (see lop_attention): q (rows_q, heads_q, d), k and v (rows_k, heads_k, d); sequence
    i's queries are rows q_offsets[i] .. q_offsets[i + 1], its keys rows k_begin[i] .. k_end[i] (int32 tensors). max_keys: keys of the longest
    sequence as far as known (None: all of k), lse: float32 (heads_q, rows_q) or None, workspace: uint8 of
    lop_attention_workspace bytes (None: allocated). Returns out."""
    device, stream, grad = _here()
    dtype, i32, shape, k_shape = q.dtype, torch.int32, q.shape, k.shape
    code = _TYPES.get(dtype) or _dtype("q", q)
    rows_q, hq, d = shape if len(shape) == 3 else _dims("q", q, 3)
    rows_k, hk, _ = k_shape if len(k_shape) == 3 else _dims("k", k, 3)
    seqs = k_begin.shape[0] if k_begin.dim() == 1 else _dims("k_begin", k_begin, 1)[0]
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    qs, ks, vs, os_ = q.stride(), k.stride(), v.stride(), out.stride()
    if (k.dtype is not dtype or v.dtype is not dtype or out.dtype is not dtype or q_offsets.dtype is not i32 or k_begin.dtype is not i32
            or k_end.dtype is not i32 or k_shape[2] != d or v.shape != k_shape or out.shape != shape or q_offsets.shape != (seqs + 1,)
            or k_end.shape != (seqs,) or q.get_device() != device or k.get_device() != device or v.get_device() != device
            or out.get_device() != device or q_offsets.get_device() != device or k_begin.get_device() != device
            or k_end.get_device() != device or (grad and (grad > 1 or q.requires_grad or k.requires_grad or v.requires_grad or out.requires_grad))
            or qs[2] != 1 or ks[2] != 1 or vs[2] != 1 or os_[2] != 1 or q_offsets.stride(0) != 1 or k_begin.stride(0) != 1
            or k_end.stride(0) != 1):
        _refuse(device, grad, ("q", q, dtype, None, 1), ("k", k, dtype, (rows_k, hk, d), 1), ("v", v, dtype, k_shape, 1),
                ("out", out, dtype, shape, 1), ("q_offsets", q_offsets, i32, (seqs + 1,), 1), ("k_begin", k_begin, i32, (seqs,), 1),
                ("k_end", k_end, i32, (seqs,), 1))
    lse_at = 0
    if lse is not None:
        _refuse(device, grad, ("lse", lse, torch.float32, (hq, rows_q), 2))
        lse_at = lse.data_ptr()
    if max_keys is None:
        max_keys = rows_k
    band = rows_q << 32 if rows is None else _rows_word(*rows)
    fields = (code, hq, hk, d, seqs, rows_q, rows_k, max_keys, causal, scale, q.data_ptr(), qs[0], qs[1], k.data_ptr(), ks[0], ks[1],
              v.data_ptr(), vs[0], vs[1], out.data_ptr(), os_[0], os_[1], q_offsets.data_ptr(), k_begin.data_ptr(), k_end.data_ptr(), lse_at)
    try:
        op = _ATTENTION.pack(*fields, 0, 0)
    except struct.error as e:
        _no_number(e)
    if workspace is None and max_keys >= (LOP_ATTENTION_CUT_F32 if code == LOP_F32 else LOP_ATTENTION_CUT):
        n = c_ulonglong(0)
        _check(_lib.lop_attention_workspace(op, band, byref(n)), "lop_attention_workspace")
        if n.value:
            workspace = torch.empty(n.value, dtype=torch.uint8, device=q.device)
    if workspace is not None:
        _refuse(device, grad, ("workspace", workspace, torch.uint8, (None,), 2))
        op = _ATTENTION.pack(*fields, workspace.data_ptr(), workspace.numel())
    e = _lib.lop_attention(op, band, stream)
    if e:
        _check(e, "lop_attention")
    return out

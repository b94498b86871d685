"""Python binding of libstlite.so (ctypes; argument marshalling only).

Every function here has the name of the C entry point it calls (declared in
``include/stlite.h``) and forwards torch CUDA tensors as raw device pointers
on the current torch stream.  No computation happens in Python: if the
library is not built this module raises at import time.

A function's ``stream`` is the torch stream to run on in place of the current
one.  The entry points take it as the library does: ordering it behind the
streams that fill the tensors, and keeping their memory until it is done, is
the caller's.  The helpers that allocate (``compress_layer``,
``decode_attention``, ``rotate_qk`` and the like) do both; reading their
results on another stream still waits for ``stream``.

    from paper_2603_00188_gb300 import stlite
    k_out, v_out, idx = stlite.compress_layer(q, k, v, frames, beta=0.2)
"""
from __future__ import annotations

import ctypes
import os
import struct
from array import array

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libstlite.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError("libstlite.so is not built (run paper_2603_00188_gb300.build.build()): %s" % _LIB_PATH)
_lib = ctypes.CDLL(_LIB_PATH)

STLITE_OK, STLITE_EINVAL, STLITE_EUNSUPPORTED, STLITE_EWORKSPACE, STLITE_ECUDA, STLITE_ETIMEOUT = range(6)
STLITE_BF16, STLITE_F32 = 0, 1
MAX_FRAMES = 256
EXPORTED = ("stlite_budget", "stlite_workspace_size", "stlite_score", "stlite_gate_frames",
            "stlite_spatial_saliency", "stlite_select_topk", "stlite_compact",
            "stlite_compress_layer", "stlite_device_status", "stlite_timing_enable", "stlite_timing_read",
            "stlite_status_string", "stlite_score_noalloc", "stlite_compress_layers", "stlite_compress_varlen",
            "stlite_workspace_size_varlen", "stlite_decode_attention", "stlite_decode_workspace_size",
            "stlite_compress_layers_budgets", "stlite_hierarchical_budgets", "stlite_spatial_saliency_size",
            "stlite_compress_varlen_layers", "stlite_prompt_score", "stlite_prompt_workspace_size",
            "stlite_decode_attention_layers", "stlite_decode_layers_workspace_size",
            "stlite_selftest_wait_timeout", "stlite_rope_init", "stlite_rotate_qk", "stlite_paged_append",
            "stlite_paged_attention", "stlite_paged_workspace_size", "stlite_compact_paged",
            "stlite_compress_layers_paged", "stlite_paged_append_q4", "stlite_paged_attention_q4",
            "stlite_paged_q4_workspace_size", "stlite_compact_paged_q4", "stlite_compress_layers_paged_q4",
            "stlite_paged_fetch_q4", "stlite_pages_step")


class Shape(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("window", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Frames(ctypes.Structure):
    _fields_ = [("n_frames", ctypes.c_int32), ("offset", ctypes.POINTER(ctypes.c_int32)),
                ("grid_h", ctypes.POINTER(ctypes.c_int32)), ("grid_w", ctypes.POINTER(ctypes.c_int32))]


class Params(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_double), ("k_override", ctypes.c_int32), ("alpha", ctypes.c_float),
                ("tsg_enable", ctypes.c_int32), ("css_enable", ctypes.c_int32), ("tsg_metric", ctypes.c_int32),
                ("tsg_fixed", ctypes.c_int32), ("tsg_fixed_tau", ctypes.c_float), ("base_scorer", ctypes.c_int32),
                ("abase_norm", ctypes.c_int32), ("css_size", ctypes.c_int32)]


STLITE_TSG_COSINE, STLITE_TSG_DOT, STLITE_TSG_NEG_L2 = 0, 1, 2
STLITE_BASE_WINDOW, STLITE_BASE_UNIFORM = 0, 1
STLITE_ABASE_RAW, STLITE_ABASE_MAX = 0, 1
STLITE_PROMPT_FULL, STLITE_PROMPT_MEAN = 0, 1


class LayerIO(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p), ("idx_out", ctypes.c_void_p)]


class DecodeIO(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p)]


class Pages(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_rows", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("table", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("cu_new", ctypes.c_void_p)]


class Rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_double * 64), ("section", ctypes.c_int32 * 3), ("interleaved", ctypes.c_int32)]


class Tokens(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float), ("pos", ctypes.c_void_p)]


class Q4PoolsC(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("k_factor", ctypes.c_void_p), ("v_factor", ctypes.c_void_p)]


class Q4Layer(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("idx", ctypes.c_void_p),
                ("pools", Q4PoolsC)]


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


_P = ctypes.c_void_p  # also takes a plain address, which costs no object
_S = ctypes.c_int32
_sig = {
    "stlite_budget": (ctypes.c_int32, [ctypes.c_int32, ctypes.c_double, ctypes.c_int32]),
    "stlite_workspace_size": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                   ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_score": (_S, [ctypes.POINTER(Shape), _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "stlite_gate_frames": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), _P, ctypes.c_int32, _P, _P, _P,
                                _P, ctypes.c_size_t, _P]),
    "stlite_spatial_saliency": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), _P, _P, _P,
                                     ctypes.c_size_t, _P]),
    "stlite_select_topk": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params), _P, _P,
                                _P, ctypes.c_int32, _P, _P, _P, ctypes.c_size_t, _P]),
    "stlite_compact": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, _P, _P, _P, _P, _P, _P]),
    "stlite_compress_layer": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params), _P,
                                   _P, _P, _P, _P, _P, ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_device_status": (_S, [_P, _P, ctypes.POINTER(ctypes.c_int32)]),
    "stlite_timing_enable": (_S, [ctypes.c_int32]),
    "stlite_timing_read": (_S, [ctypes.POINTER(KernelTime), ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]),
    "stlite_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "stlite_score_noalloc": (_S, [ctypes.POINTER(Shape), _P, _P, _P, _P]),
    "stlite_compress_layers": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                    ctypes.c_int32, _P, ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_compress_varlen": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                    ctypes.POINTER(Frames), ctypes.POINTER(Params), _P, _P, _P, _P, _P, _P,
                                    ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_workspace_size_varlen": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                          ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                          ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_decode_attention": (_S, [ctypes.POINTER(Shape), _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "stlite_decode_workspace_size": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_compress_layers_budgets": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                            ctypes.c_int32, _P, ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t,
                                            _P]),
    "stlite_spatial_saliency_size": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), _P, ctypes.c_int32, _P, _P,
                                          ctypes.c_size_t, _P]),
    "stlite_compress_varlen_layers": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                           ctypes.POINTER(Frames), ctypes.POINTER(Params), ctypes.c_int32, _P,
                                           ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_hierarchical_budgets": (_S, [ctypes.c_int32, ctypes.POINTER(ctypes.c_double), ctypes.c_int64,
                                         ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]),
    "stlite_prompt_score": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, ctypes.c_int32, _P, _P, _P, _P,
                                 ctypes.c_size_t, _P]),
    "stlite_prompt_workspace_size": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_selftest_wait_timeout": (_S, [_P, ctypes.c_int64, _P]),
    "stlite_decode_attention_layers": (_S, [ctypes.POINTER(Shape), ctypes.c_int32, _P, _P, ctypes.c_size_t, _P]),
    "stlite_decode_layers_workspace_size": (_S, [ctypes.POINTER(Shape), ctypes.c_int32,
                                                 ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_rope_init": (_S, [ctypes.c_double, ctypes.POINTER(Rope)]),
    # shape, tokens and pages as packed bytes or addresses: no object for each call
    "stlite_rotate_qk": (_S, [_P, ctypes.POINTER(Rope), _P, _P, _P, _P]),
    "stlite_paged_append": (_S, [_P, ctypes.POINTER(Rope), _P, _P, _P, _P, _P, _P]),
    "stlite_paged_attention": (_S, [_P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "stlite_paged_workspace_size": (_S, [_P, _P, ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_compact_paged": (_S, [_P, ctypes.c_int32, _P, ctypes.c_int32, ctypes.c_int32, _P, _P]),
    "stlite_compress_layers_paged": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                          _P, ctypes.c_int32, ctypes.c_int32, _P,
                                          ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_paged_append_q4": (_S, [_P, ctypes.POINTER(Rope), _P, _P, _P, _P, _P]),
    "stlite_paged_attention_q4": (_S, [_P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "stlite_paged_q4_workspace_size": (_S, [_P, _P, ctypes.POINTER(ctypes.c_size_t)]),
    "stlite_compact_paged_q4": (_S, [_P, ctypes.c_int32, _P, ctypes.c_int32, ctypes.c_int32, _P, _P]),
    "stlite_compress_layers_paged_q4": (_S, [ctypes.POINTER(Shape), ctypes.POINTER(Frames), ctypes.POINTER(Params),
                                             _P, ctypes.c_int32, ctypes.c_int32, _P,
                                             ctypes.POINTER(ctypes.c_int32), _P, ctypes.c_size_t, _P]),
    "stlite_paged_fetch_q4": (_S, [_P, _P, ctypes.c_int32, _P, _P]),
    "stlite_pages_step": (_S, [_P, _P, _P, _P, _P, ctypes.c_int32, _P, _P]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


class StliteError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, _lib.stlite_status_string(status).decode(), status))


def _check(status: int, where: str):
    if status != STLITE_OK:
        raise StliteError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _lend(stream, *tensors):
    """What a helper that allocates does before its call on a `stream` that is
    not the current one: `stream` waits for what the current one holds so far
    (the tensors' contents, a workspace's zeros, an earlier user of an
    output's memory), and the device tensors' memory is not given out again
    before `stream` has used it."""
    if stream is None or stream == torch.cuda.current_stream():
        return
    stream.wait_stream(torch.cuda.current_stream())
    for t in tensors:
        if t is not None and t.is_cuda:
            t.record_stream(stream)


_DTYPE = {torch.bfloat16: STLITE_BF16, torch.float32: STLITE_F32}


def make_shape(q, k) -> Shape:
    w, hq, d = q.shape
    n, hkv, d2 = k.shape
    if d != d2:
        raise ValueError("q and k head_dim differ")
    return Shape(n, hq, hkv, d, w, _DTYPE[k.dtype])


def _layer_table(layers):
    """The stlite_layer_io array of (q, k, v, k_out, v_out, idx_out) tuples."""
    return array("Q", [p for q, k, v, ko, vo, ix in layers for p in (
        q.data_ptr(), k.data_ptr(), v.data_ptr(), ko.data_ptr(), vo.data_ptr(), ix.data_ptr())])


def _decode_table(layers):
    """The stlite_decode_io array of (q, k, v, out) tuples."""
    return array("Q", [p for q, k, v, o in layers for p in (
        q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr())])


def _address(table) -> int:
    return table.buffer_info()[0]


class FrameSpec:
    """Host frame descriptor (offset, grid_h, grid_w), kept alive with its ctypes view."""

    def __init__(self, offset, grid_h, grid_w):
        self.offset = np.ascontiguousarray(offset, dtype=np.int32)
        self.grid_h = np.ascontiguousarray(grid_h, dtype=np.int32)
        self.grid_w = np.ascontiguousarray(grid_w, dtype=np.int32)
        ip = ctypes.POINTER(ctypes.c_int32)
        self.c = Frames(len(self.offset), self.offset.ctypes.data_as(ip), self.grid_h.ctypes.data_as(ip),
                        self.grid_w.ctypes.data_as(ip))


def _frames(frames) -> FrameSpec:
    if isinstance(frames, FrameSpec):
        return frames
    return FrameSpec(*frames)


def make_params(beta=0.2, k_override=0, alpha=1.0, tsg_enable=1, css_enable=1, tsg_metric=STLITE_TSG_COSINE,
                fixed_tau=None, base_scorer=STLITE_BASE_WINDOW, abase_norm=STLITE_ABASE_RAW, css_size=3) -> Params:
    """Parameters of the pass; the keywords after css_enable select the
    paper's ablation variants (TSG similarity metric, a fixed gate threshold,
    the uniform base prior, A_base divided by its maximum, the CSS
    neighbourhood size) and default to the method as published."""
    return Params(float(beta), int(k_override), float(alpha), int(tsg_enable), int(css_enable), int(tsg_metric),
                  0 if fixed_tau is None else 1, 0.0 if fixed_tau is None else float(fixed_tau), int(base_scorer),
                  int(abase_norm), int(css_size))


# ----------------------------------------------------------------- entries

def stlite_budget(n_tokens: int, beta: float, k_override: int = 0) -> int:
    return int(_lib.stlite_budget(int(n_tokens), float(beta), int(k_override)))


def stlite_workspace_size(shape: Shape, frames, params: Params | None = None) -> int:
    fs = _frames(frames)
    out = ctypes.c_size_t()
    _check(_lib.stlite_workspace_size(ctypes.byref(shape), ctypes.byref(fs.c),
                                      ctypes.byref(params) if params is not None else None,
                                      ctypes.byref(out)), "stlite_workspace_size")
    return int(out.value)


def workspace(shape: Shape, frames, params: Params | None = None, device="cuda"):
    """Zero-filled workspace tensor of the size the library asks for."""
    return torch.zeros(stlite_workspace_size(shape, frames, params), dtype=torch.uint8, device=device)


def stlite_score(q, k, a_base, ws, stream=None):
    sh = make_shape(q, k)
    _check(_lib.stlite_score(ctypes.byref(sh), _ptr(q), _ptr(k), _ptr(a_base), _ptr(ws), ws.numel(),
                             _stream(stream)), "stlite_score")


def stlite_gate_frames(q, k, frames, budget, rho, tau, gate, ws, stream=None):
    sh = make_shape(q, k)
    fs = _frames(frames)
    _check(_lib.stlite_gate_frames(ctypes.byref(sh), ctypes.byref(fs.c), _ptr(k), int(budget), _ptr(rho),
                                   _ptr(tau), _ptr(gate), _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_gate_frames")


def stlite_spatial_saliency(q, k, frames, phi, ws, stream=None):
    sh = make_shape(q, k)
    fs = _frames(frames)
    _check(_lib.stlite_spatial_saliency(ctypes.byref(sh), ctypes.byref(fs.c), _ptr(k), _ptr(phi), _ptr(ws),
                                        ws.numel(), _stream(stream)), "stlite_spatial_saliency")


def stlite_spatial_saliency_size(q, k, frames, size, phi, ws, stream=None):
    sh = make_shape(q, k)
    fs = _frames(frames)
    _check(_lib.stlite_spatial_saliency_size(ctypes.byref(sh), ctypes.byref(fs.c), _ptr(k), int(size), _ptr(phi),
                                             _ptr(ws), ws.numel(), _stream(stream)), "stlite_spatial_saliency_size")


def stlite_select_topk(q, k, frames, params, a_base, phi, gate, budget, idx, score_out, ws, stream=None):
    sh = make_shape(q, k)
    fs = _frames(frames)
    _check(_lib.stlite_select_topk(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params), _ptr(a_base),
                                   _ptr(phi), _ptr(gate), int(budget), _ptr(idx), _ptr(score_out), _ptr(ws),
                                   ws.numel(), _stream(stream)), "stlite_select_topk")


def stlite_compact(q, k, v, budget, idx, k_out, v_out, stream=None):
    sh = make_shape(q, k)
    _check(_lib.stlite_compact(ctypes.byref(sh), int(budget), _ptr(idx), _ptr(k), _ptr(v), _ptr(k_out),
                               _ptr(v_out), _stream(stream)), "stlite_compact")


def stlite_compress_layer(q, k, v, frames, params, k_out, v_out, idx_out, ws, stream=None) -> int:
    sh = make_shape(q, k)
    fs = _frames(frames)
    b = ctypes.c_int32(0)
    _check(_lib.stlite_compress_layer(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params), _ptr(q),
                                      _ptr(k), _ptr(v), _ptr(k_out), _ptr(v_out), _ptr(idx_out),
                                      ctypes.byref(b), _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_compress_layer")
    return int(b.value)


def stlite_compress_layers(layers, frames, params, ws, stream=None) -> int:
    """layers: list of (q, k, v, k_out, v_out, idx_out) device tensors, one
    tuple per layer (same shapes); ws: n_layers * stlite_workspace_size bytes."""
    q0, k0 = layers[0][0], layers[0][1]
    sh = make_shape(q0, k0)
    fs = _frames(frames)
    arr = _layer_table(layers)
    b = ctypes.c_int32(0)
    _check(_lib.stlite_compress_layers(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params), len(layers),
                                       _address(arr), ctypes.byref(b), _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_compress_layers")
    return int(b.value)


def stlite_compress_layers_budgets(layers, frames, params, budgets, ws, stream=None):
    """As stlite_compress_layers with layer l keeping budgets[l] tokens per
    KV head (k_out / v_out of layer l: [budgets[l]][Hkv][d], idx_out:
    [Hkv][budgets[l]])."""
    q0, k0 = layers[0][0], layers[0][1]
    sh = make_shape(q0, k0)
    fs = _frames(frames)
    arr = _layer_table(layers)
    bud = (ctypes.c_int32 * len(layers))(*[int(b) for b in budgets])
    _check(_lib.stlite_compress_layers_budgets(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params),
                                               len(layers), _address(arr), bud, _ptr(ws), ws.numel(),
                                               _stream(stream)),
           "stlite_compress_layers_budgets")


def stlite_hierarchical_budgets(layer_mass, total_budget: int, n_tokens: int) -> list:
    """B^(l) = S^(l) / sum S * B_total as integers adding up to B_total
    (floor plus largest remainder, clamped to [1, n_tokens])."""
    n = len(layer_mass)
    mass = (ctypes.c_double * n)(*[float(x) for x in layer_mass])
    out = (ctypes.c_int32 * n)()
    _check(_lib.stlite_hierarchical_budgets(n, mass, int(total_budget), int(n_tokens), out),
           "stlite_hierarchical_budgets")
    return list(out)


def _varlen_args(cu_seqlens, frames_list):
    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    specs = [_frames(f) for f in frames_list]
    arr = (Frames * len(specs))(*[f.c for f in specs])
    return cu, specs, arr


def stlite_workspace_size_varlen(shape: Shape, cu_seqlens, frames_list, params: Params | None = None) -> int:
    cu, specs, arr = _varlen_args(cu_seqlens, frames_list)
    out = ctypes.c_size_t()
    _check(_lib.stlite_workspace_size_varlen(ctypes.byref(shape), len(specs),
                                             cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), arr,
                                             ctypes.byref(params) if params is not None else None,
                                             ctypes.byref(out)), "stlite_workspace_size_varlen")
    return int(out.value)


def stlite_compress_varlen(q, k, v, cu_seqlens, frames_list, params, k_out, v_out, idx_out, ws, stream=None):
    """Packed batch of sequences (one layer): q [n_seqs][w][Hq][d], k/v packed
    [N][Hkv][d], cu_seqlens (n_seqs + 1 offsets), one frame descriptor per
    sequence (offsets relative to the sequence).  Returns the budget prefix
    sums (n_seqs + 1)."""
    n_seqs = len(frames_list)
    sh = make_shape(q[0] if q.dim() == 4 else q, k)
    cu, specs, arr = _varlen_args(cu_seqlens, frames_list)
    cb = np.zeros(n_seqs + 1, dtype=np.int32)
    ip = ctypes.POINTER(ctypes.c_int32)
    _check(_lib.stlite_compress_varlen(ctypes.byref(sh), n_seqs, cu.ctypes.data_as(ip), arr, ctypes.byref(params),
                                       _ptr(q), _ptr(k), _ptr(v), _ptr(k_out), _ptr(v_out), _ptr(idx_out),
                                       cb.ctypes.data_as(ip), _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_compress_varlen")
    return cb


def stlite_compress_varlen_layers(layers, cu_seqlens, frames_list, params, ws, stream=None):
    """stlite_compress_varlen over several layers of one packed batch: layers
    is a list of (q, k, v, k_out, v_out, idx_out) per layer, each in the
    packed layouts of stlite_compress_varlen; ws: n_layers times
    stlite_workspace_size_varlen bytes.  Returns the budget prefix sums."""
    n_seqs = len(frames_list)
    q0, k0 = layers[0][0], layers[0][1]
    sh = make_shape(q0[0] if q0.dim() == 4 else q0, k0)
    cu, specs, arr = _varlen_args(cu_seqlens, frames_list)
    lio = _layer_table(layers)
    cb = np.zeros(n_seqs + 1, dtype=np.int32)
    ip = ctypes.POINTER(ctypes.c_int32)
    _check(_lib.stlite_compress_varlen_layers(ctypes.byref(sh), n_seqs, cu.ctypes.data_as(ip), arr,
                                              ctypes.byref(params), len(layers), _address(lio),
                                              cb.ctypes.data_as(ip), _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_compress_varlen_layers")
    return cb


def stlite_decode_workspace_size(shape: Shape) -> int:
    out = ctypes.c_size_t()
    _check(_lib.stlite_decode_workspace_size(ctypes.byref(shape), ctypes.byref(out)), "stlite_decode_workspace_size")
    return int(out.value)


def stlite_decode_attention(q, k, v, out, ws, stream=None):
    """Attention of the query rows q [w][Hq][d] over the cache k, v [n][Hkv][d]
    (full or compacted) into out [w][Hq][d] float32."""
    sh = make_shape(q, k)
    _check(_lib.stlite_decode_attention(ctypes.byref(sh), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(ws),
                                        ws.numel(), _stream(stream)), "stlite_decode_attention")


def decode_attention(q, k, v, stream=None):
    """Allocates the output and the workspace and runs stlite_decode_attention."""
    sh = make_shape(q, k)
    ws = torch.zeros(stlite_decode_workspace_size(sh), dtype=torch.uint8, device=k.device)
    out = torch.empty(q.shape, dtype=torch.float32, device=k.device)
    _lend(stream, q, k, v, out, ws)
    stlite_decode_attention(q, k, v, out, ws, stream)
    return out


def prompt_shape(q_prompt, k) -> Shape:
    """Shape of a prompt-wide score call: the window field is unused (1)."""
    n_q, hq, d = q_prompt.shape
    n, hkv, d2 = k.shape
    if d != d2:
        raise ValueError("q and k head_dim differ")
    return Shape(n, hq, hkv, d, 1, _DTYPE[k.dtype])


def stlite_prompt_workspace_size(shape: Shape, n_prompt: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib.stlite_prompt_workspace_size(ctypes.byref(shape), int(n_prompt), ctypes.byref(out)),
           "stlite_prompt_workspace_size")
    return int(out.value)


def stlite_prompt_score(q_prompt, k, base, a_base, ws, stream=None):
    """Prompt-wide base scores (STLITE_PROMPT_FULL / STLITE_PROMPT_MEAN) of
    the n_prompt = q_prompt.shape[0] rows of the last positions."""
    sh = prompt_shape(q_prompt, k)
    _check(_lib.stlite_prompt_score(ctypes.byref(sh), int(q_prompt.shape[0]), int(base), _ptr(q_prompt), _ptr(k),
                                    _ptr(a_base), _ptr(ws), ws.numel(), _stream(stream)), "stlite_prompt_score")


def prompt_score(q_prompt, k, base=STLITE_PROMPT_MEAN, stream=None):
    """Allocates the output and a workspace and runs stlite_prompt_score."""
    sh = prompt_shape(q_prompt, k)
    ws = torch.zeros(stlite_prompt_workspace_size(sh, q_prompt.shape[0]), dtype=torch.uint8, device=k.device)
    a = torch.empty((sh.n_kv_heads, sh.n_tokens), dtype=torch.float32, device=k.device)
    _lend(stream, q_prompt, k, a, ws)
    stlite_prompt_score(q_prompt, k, base, a, ws, stream)
    return a, ws


def stlite_decode_layers_workspace_size(shape: Shape, n_layers: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib.stlite_decode_layers_workspace_size(ctypes.byref(shape), int(n_layers), ctypes.byref(out)),
           "stlite_decode_layers_workspace_size")
    return int(out.value)


def stlite_decode_attention_layers(layers, ws, stream=None):
    """layers: list of (q, k, v, out) device tensors, one tuple per layer
    (same shapes)."""
    sh = make_shape(layers[0][0], layers[0][1])
    arr = _decode_table(layers)
    _check(_lib.stlite_decode_attention_layers(ctypes.byref(sh), len(layers), _address(arr), _ptr(ws), ws.numel(),
                                               _stream(stream)), "stlite_decode_attention_layers")


def decode_attention_layers(qs, ks, vs, stream=None):
    """Allocates the outputs and the workspace and runs
    stlite_decode_attention_layers over the layers' (q, k, v)."""
    sh = make_shape(qs[0], ks[0])
    ws = torch.zeros(stlite_decode_layers_workspace_size(sh, len(qs)), dtype=torch.uint8, device=ks[0].device)
    outs = [torch.empty(q.shape, dtype=torch.float32, device=ks[0].device) for q in qs]
    _lend(stream, *qs, *ks, *vs, *outs, ws)
    stlite_decode_attention_layers(list(zip(qs, ks, vs, outs)), ws, stream)
    return outs, ws


# ------------------------------------------------------------ paged caches

def make_rope(base=10000.0, section=(64, 0, 0), interleaved=False, inv_freq=None) -> Rope:
    """Rotary frequencies base^(-2 i / 128), or inv_freq (64 values, for
    scaled ones); section: pairs turned by each of the three position axes."""
    rope = Rope()
    _check(_lib.stlite_rope_init(float(base), ctypes.byref(rope)), "stlite_rope_init")
    if inv_freq is not None:
        rope.inv_freq[:] = [float(x) for x in inv_freq]
    rope.section[:] = [int(x) for x in section]
    rope.interleaved = int(interleaved)
    return rope


class PageTable:
    """stlite_pages of int32 device tensors (kept alive with it): table
    [S][max_pages], length [S], cu_new [S + 1] or None.  max_new: the most
    new tokens of a sequence (of every sequence where cu_new is None)."""

    def __init__(self, n_pages, page_rows, table, length=None, cu_new=None, max_new=1):
        for t, n in ((table, 2), (length, 1), (cu_new, 1)):
            if t is not None and (t.dtype != torch.int32 or t.dim() != n or not t.is_contiguous()
                                  or t.device != table.device):
                raise ValueError("table, length and cu_new are contiguous int32 tensors of one device")
        n_seqs = table.shape[0]
        if (length is not None and length.shape[0] != n_seqs) or (cu_new is not None and cu_new.shape[0] != n_seqs + 1):
            raise ValueError("length is [S] and cu_new [S + 1] for a table [S][max_pages]")
        self.table, self.length, self.cu_new, self.max_new = table, length, cu_new, int(max_new)
        self.c = Pages(n_seqs, int(n_pages), int(page_rows), table.shape[1], _ptr(table), _ptr(length), _ptr(cu_new))
        self._address, self._device = ctypes.addressof(self.c), table.get_device()
        self._pool = (int(n_pages), int(page_rows))


def make_pages(n_pages, page_rows, table, length=None, cu_new=None, max_new=1) -> PageTable:
    return PageTable(n_pages, page_rows, table, length, cu_new, max_new)


_SHAPE = struct.Struct("=6i")            # stlite_shape
_TOKENS = struct.Struct("=3Q3q2Qf4xQ")   # stlite_tokens
_CURRENT = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # of a device


def _pool_error(pages, hkv):
    return ValueError("a page pool is a contiguous tensor %s of the cache's type" % ((*pages._pool, hkv, 128),))


def _output_error(shape):
    return ValueError("an output is a contiguous %s of q's type" % (tuple(shape),))


_ELSEWHERE = "the tensors are not on the current CUDA device"


def _tokens(q, k, v, pos, rope, q_norm, k_norm, eps, qs, ks, dtype) -> bytes:
    """stlite_tokens of q, k, v [T][H][128] (qs, ks: the shapes of q and k),
    each token's heads packed."""
    n, hq, d = qs
    nk, hkv, dk = ks
    sq0, sq1, sq2 = q.stride()
    sk0, sk1, sk2 = k.stride()
    if not (d == 128 == dk and nk == n and sq2 == 1 == sk2 and (sq1 == 128 or hq == 1) and (sk1 == 128 or hkv == 1)
            and k.dtype == dtype):
        raise ValueError("q and k are [T][H][128] of one type, each token's heads packed")
    pv = sv0 = 0
    if v is not None:
        sv0, sv1, sv2 = v.stride()
        pv, sv0 = v.data_ptr(), sv0 or 1
        if not (sv2 == 1 and (sv1 == 128 or hkv == 1) and v.shape == ks and v.dtype == dtype):
            raise ValueError("v is as k")
    pq = pk = 0
    if q_norm is not None or k_norm is not None:
        for w in (q_norm, k_norm):
            if w is not None and (w.shape != (128,) or w.dtype != dtype or not w.is_contiguous()):
                raise ValueError("a norm's weights are [128] of q's type")
            if w is not None and w.get_device() != q.get_device():
                raise ValueError(_ELSEWHERE)
        pq, pk = _ptr(q_norm) or 0, _ptr(k_norm) or 0
    one = rope.section[0] == 64
    if (pos.dtype != torch.int32 or pos.numel() != (n if one else 3 * n) or not pos.is_contiguous()
            or not (one or pos.dim() == 1 or pos.shape[0] == 3)):
        raise ValueError("pos is a contiguous int32 [T], or [3][T] for three axes")
    if n == 1:  # no next token: whatever its distance would be
        return _TOKENS.pack(q.data_ptr(), k.data_ptr(), pv, 0, 0, 0, pq, pk, eps, pos.data_ptr())
    # 0 stands for packed, so a broadcast token's goes as 1, which the library refuses
    return _TOKENS.pack(q.data_ptr(), k.data_ptr(), pv, sq0 or 1, sk0 or 1, sv0, pq, pk, eps, pos.data_ptr())


def stlite_rotate_qk(q, k, pos, rope, q_out, k_out, q_norm=None, k_norm=None, eps=1e-6, stream=None):
    """Norm (where weights are given) and rotation of every head of q
    [T][Hq][128] and k [T][Hkv][128] (each may be a slice of one projection's
    output) into q_out and k_out; pos: int32 [T], or [3][T] for three axes.
    T = 0 does nothing."""
    qs, ks, dtype, dev = q.shape, k.shape, q.dtype, q.get_device()
    x = _tokens(q, k, None, pos, rope, q_norm, k_norm, eps, qs, ks, dtype)
    if q_out.shape != qs or q_out.dtype != dtype or not q_out.is_contiguous():
        raise _output_error(qs)
    if k_out.shape != ks or k_out.dtype != dtype or not k_out.is_contiguous():
        raise _output_error(ks)
    if dev < 0 or not (torch._C._cuda_getDevice() == dev == k.get_device() == pos.get_device() == q_out.get_device()
                       == k_out.get_device()):
        raise ValueError(_ELSEWHERE)
    if qs[0] == 0:
        return
    st = _lib.stlite_rotate_qk(_SHAPE.pack(qs[0], qs[1], ks[1], 128, 1, _DTYPE[dtype]), rope, x, q_out.data_ptr(),
                               k_out.data_ptr(), _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_rotate_qk")


def rotate_qk(q, k, pos, rope, q_norm=None, k_norm=None, eps=1e-6, stream=None):
    """Allocates the outputs and runs stlite_rotate_qk."""
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    _lend(stream, q, k, pos, q_norm, k_norm, q_out, k_out)
    stlite_rotate_qk(q, k, pos, rope, q_out, k_out, q_norm, k_norm, eps, stream)
    return q_out, k_out


def stlite_paged_append(q, k, v, pos, rope, pages, q_out, k_pages, v_pages, q_norm=None, k_norm=None, eps=1e-6,
                        stream=None):
    """The new tokens' rotated keys and their values into the pages, the
    rotated queries into q_out (see stlite_rotate_qk for q, k, v and pos)."""
    qs, ks, dtype, dev = q.shape, k.shape, q.dtype, q.get_device()
    x = _tokens(q, k, v, pos, rope, q_norm, k_norm, eps, qs, ks, dtype)
    if q_out.shape != qs or q_out.dtype != dtype or not q_out.is_contiguous():
        raise _output_error(qs)
    hkv = ks[1]
    want = (*pages._pool, hkv, 128)
    if (k_pages.shape != want or v_pages.shape != want or k_pages.dtype != dtype or v_pages.dtype != dtype
            or not (k_pages.is_contiguous() and v_pages.is_contiguous())):
        raise _pool_error(pages, hkv)
    if dev < 0 or not (torch._C._cuda_getDevice() == dev == k.get_device() == v.get_device() == pos.get_device()
                       == q_out.get_device() == k_pages.get_device() == v_pages.get_device() == pages._device):
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_paged_append(
        _SHAPE.pack(qs[0], qs[1], hkv, 128, pages.max_new if pages.cu_new is None else 1, _DTYPE[dtype]), rope, x,
        pages._address, q_out.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
        _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_paged_append")


def _paged_shape(q, k_pages, pages) -> Shape:
    if q.dim() != 3 or q.shape[2] != 128 or not q.is_contiguous():
        raise ValueError("q is a contiguous [T][Hq][128]")
    return Shape(q.shape[0], q.shape[1], k_pages.shape[2], 128, pages.max_new, _DTYPE[q.dtype])


def stlite_paged_workspace_size(shape: Shape, pages: PageTable) -> int:
    out = ctypes.c_size_t()
    _check(_lib.stlite_paged_workspace_size(ctypes.byref(shape), ctypes.byref(pages.c), ctypes.byref(out)),
           "stlite_paged_workspace_size")
    return int(out.value)


def paged_workspace(q, k_pages, pages):
    """Zero-filled workspace tensor of stlite_paged_attention."""
    return torch.zeros(stlite_paged_workspace_size(_paged_shape(q, k_pages, pages), pages), dtype=torch.uint8,
                       device=q.device)


def stlite_paged_attention(q, k_pages, v_pages, pages, out, ws, stream=None):
    """Attention of the new tokens q [T][Hq][128] over their sequences'
    pages into out (q's shape and type)."""
    (n, hq, d), dtype, dev = q.shape, q.dtype, q.get_device()
    if d != 128 or not q.is_contiguous():
        raise ValueError("q is a contiguous [T][Hq][128]")
    if out.shape != q.shape or out.dtype != dtype or not out.is_contiguous():
        raise _output_error(q.shape)
    p, r, hkv, d = pool = k_pages.shape
    if ((p, r) != pages._pool or d != 128 or k_pages.dtype != dtype or v_pages.dtype != dtype
            or v_pages.shape != pool or not (k_pages.is_contiguous() and v_pages.is_contiguous())):
        raise _pool_error(pages, "Hkv")
    if dev < 0 or not (torch._C._cuda_getDevice() == dev == k_pages.get_device() == v_pages.get_device()
                       == out.get_device() == ws.get_device() == pages._device):
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_paged_attention(
        _SHAPE.pack(n, hq, hkv, 128, pages.max_new, _DTYPE[dtype]), pages._address, q.data_ptr(), k_pages.data_ptr(),
        v_pages.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.nbytes,
        _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_paged_attention")


def paged_attention(q, k_pages, v_pages, pages, stream=None):
    """Allocates the output and the workspace and runs stlite_paged_attention."""
    out, ws = torch.empty_like(q), paged_workspace(q, k_pages, pages)
    _lend(stream, q, k_pages, v_pages, pages.table, pages.length, pages.cu_new, out, ws)
    stlite_paged_attention(q, k_pages, v_pages, pages, out, ws, stream)
    return out


def stlite_compact_paged(layers, budget, pages, seq, stream=None):
    """The kept rows of every layer into sequence seq's pages; layers: list
    of (k, v, k_pages, v_pages, idx)."""
    k0 = layers[0][0]
    shape, dtype, dev, flat = k0.shape, k0.dtype, k0.get_device(), []
    n, hkv, d = shape
    want, index = (*pages._pool, hkv, d), (hkv, budget)
    for k, v, kp, vp, ix in layers:
        if not (k.shape == shape == v.shape and kp.shape == want == vp.shape and ix.shape == index
                and k.dtype == dtype == v.dtype and kp.dtype == dtype == vp.dtype and ix.dtype == torch.int32
                and k.is_contiguous() and v.is_contiguous() and kp.is_contiguous() and vp.is_contiguous()
                and ix.is_contiguous()):
            raise ValueError("every layer's k and v are [N][Hkv][128], pools %s of their type and idx int32 "
                             "[Hkv][budget], contiguous" % (want,))
        if not k.get_device() == kp.get_device() == vp.get_device() == ix.get_device() == dev or (
                v.get_device() != dev and not v.is_pinned()):
            raise ValueError(_ELSEWHERE)
        a = k.data_ptr()
        flat += (a, a, v.data_ptr(), kp.data_ptr(), vp.data_ptr(), ix.data_ptr())
    if dev < 0 or not torch._C._cuda_getDevice() == dev == pages._device:
        raise ValueError(_ELSEWHERE)
    arr = array("Q", flat)
    st = _lib.stlite_compact_paged(_SHAPE.pack(n, hkv, hkv, d, 1, _DTYPE[dtype]), budget, pages._address, seq,
                                   len(layers), _address(arr), _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_compact_paged")


def stlite_compress_layers_paged(layers, frames, params, pages, seq, ws, stream=None) -> int:
    """stlite_compress_layers with the kept rows in sequence seq's pages;
    layers: list of (q, k, v, k_pages, v_pages, idx_out)."""
    q0, k0 = layers[0][:2]
    sh = make_shape(q0, k0)
    qs, shape, dtype, dev = q0.shape, k0.shape, k0.dtype, k0.get_device()
    want = (*pages._pool, sh.n_kv_heads, 128)
    kept = sh.n_kv_heads * stlite_budget(sh.n_tokens, params.beta, params.k_override)
    for q, k, v, kp, vp, ix in layers:
        if not (kp.shape == want == vp.shape and kp.dtype == dtype == vp.dtype and kp.is_contiguous()
                and vp.is_contiguous()):
            raise _pool_error(pages, sh.n_kv_heads)
        if not (q.shape == qs and k.shape == shape == v.shape and q.dtype == dtype == k.dtype and v.dtype == dtype
                and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("every layer's q is [w][Hq][128] and its k and v [N][Hkv][128], of one type, contiguous")
        if ix.dtype != torch.int32 or ix.numel() < kept or not ix.is_contiguous():
            raise ValueError("every layer's idx_out is contiguous int32 with room for [Hkv][B]")
        if not q.get_device() == k.get_device() == kp.get_device() == vp.get_device() == ix.get_device() == dev or (
                v.get_device() != dev and not v.is_pinned()):
            raise ValueError(_ELSEWHERE)
    if dev < 0 or not torch._C._cuda_getDevice() == dev == pages._device == ws.get_device():
        raise ValueError(_ELSEWHERE)
    fs = _frames(frames)
    arr = _layer_table(layers)
    b = ctypes.c_int32(0)
    _check(_lib.stlite_compress_layers_paged(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params),
                                             pages._address, int(seq), len(layers), _address(arr), ctypes.byref(b),
                                             _ptr(ws), ws.numel(), _stream(stream)), "stlite_compress_layers_paged")
    return int(b.value)


# ---------------------------------------------------------- pages in 4 bits

class Q4Pools:
    """stlite_q4_pools of one layer's device tensors (kept alive with it): codes
    k, v uint8 [n_pages][Hkv][page_rows][64], scales k_scale, v_scale
    (torch.float8_e4m3fn or uint8) [n_pages][Hkv][page_rows][8], factors float32
    [Hkv] or None."""

    def __init__(self, k, v, k_scale, v_scale, k_factor=None, v_factor=None):
        if k.dim() != 4 or k.shape[3] != 64:
            raise ValueError("codes are [n_pages][Hkv][page_rows][64]")
        p, hkv, r, _ = k.shape
        for t, shape, types in ((k, k.shape, (torch.uint8,)), (v, k.shape, (torch.uint8,)),
                                (k_scale, (p, hkv, r, 8), (torch.float8_e4m3fn, torch.uint8)),
                                (v_scale, (p, hkv, r, 8), (torch.float8_e4m3fn, torch.uint8)),
                                (k_factor, (hkv,), (torch.float32,)), (v_factor, (hkv,), (torch.float32,))):
            if t is not None and (t.shape != shape or t.dtype not in types or not t.is_contiguous()
                                  or t.device != k.device):
                raise ValueError("codes are uint8 [n_pages][Hkv][page_rows][64], scales e4m3 [n_pages][Hkv][page_rows]"
                                 "[8] and factors float32 [Hkv], contiguous, of one device")
        self.k, self.v, self.k_scale, self.v_scale, self.k_factor, self.v_factor = k, v, k_scale, v_scale, k_factor, v_factor
        self.c = Q4PoolsC(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(k_factor), _ptr(v_factor))
        self.hkv, self._pool, self._device = hkv, (p, r), k.get_device()
        self._kind = (p, r, hkv)
        self._address, self._bytes = ctypes.addressof(self.c), bytes(self.c)


def make_q4_pools(n_pages, page_rows, hkv, k_factor=None, v_factor=None, device="cuda") -> Q4Pools:
    """Allocates zero-filled pools of one layer."""
    shape = (int(n_pages), int(hkv), int(page_rows))
    k, v = (torch.zeros(shape + (64,), dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros(shape + (8,), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2))
    return Q4Pools(k, v, ks, vs, k_factor, v_factor)


_ROWS = struct.Struct("=4Q")  # the rows of stlite_q4_layer, before its pools


def _q4_error():
    return ValueError("every layer's pools are Q4Pools of the pages' numbers and of k's heads")


def stlite_paged_append_q4(q, k, v, pos, rope, pages, q_out, pools, q_norm=None, k_norm=None, eps=1e-6, stream=None):
    """stlite_paged_append into a layer's 4-bit pages (Q4Pools)."""
    qs, ks, dtype, dev = q.shape, k.shape, q.dtype, q.get_device()
    x = _tokens(q, k, v, pos, rope, q_norm, k_norm, eps, qs, ks, dtype)
    if q_out.shape != qs or q_out.dtype != dtype or not q_out.is_contiguous():
        raise _output_error(qs)
    hkv = ks[1]
    if pools._kind != (*pages._pool, hkv):
        raise _q4_error()
    if dev < 0 or not (torch._C._cuda_getDevice() == dev == k.get_device() == v.get_device() == pos.get_device()
                       == q_out.get_device() == pools._device == pages._device):
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_paged_append_q4(
        _SHAPE.pack(qs[0], qs[1], hkv, 128, pages.max_new if pages.cu_new is None else 1, _DTYPE[dtype]), rope, x,
        pages._address, q_out.data_ptr(), pools._address, _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_paged_append_q4")


def stlite_paged_q4_workspace_size(shape: Shape, pages: PageTable) -> int:
    out = ctypes.c_size_t()
    _check(_lib.stlite_paged_q4_workspace_size(ctypes.byref(shape), ctypes.byref(pages.c), ctypes.byref(out)),
           "stlite_paged_q4_workspace_size")
    return int(out.value)


def paged_q4_workspace(q, pools, pages):
    """Zero-filled workspace tensor of stlite_paged_attention_q4."""
    if q.dim() != 3 or q.shape[2] != 128 or not q.is_contiguous():
        raise ValueError("q is a contiguous [T][Hq][128]")
    shape = Shape(q.shape[0], q.shape[1], pools.hkv, 128, pages.max_new, _DTYPE[q.dtype])
    return torch.zeros(stlite_paged_q4_workspace_size(shape, pages), dtype=torch.uint8, device=q.device)


def stlite_paged_attention_q4(q, pools, pages, out, ws, stream=None):
    """stlite_paged_attention over a layer's 4-bit pages (Q4Pools)."""
    (n, hq, d), dtype, dev = q.shape, q.dtype, q.get_device()
    if d != 128 or not q.is_contiguous():
        raise ValueError("q is a contiguous [T][Hq][128]")
    if out.shape != q.shape or out.dtype != dtype or not out.is_contiguous():
        raise _output_error(q.shape)
    if pools._pool != pages._pool:
        raise _q4_error()
    if dev < 0 or not (torch._C._cuda_getDevice() == dev == out.get_device() == ws.get_device() == pools._device
                       == pages._device):
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_paged_attention_q4(
        _SHAPE.pack(n, hq, pools.hkv, 128, pages.max_new, _DTYPE[dtype]), pages._address, q.data_ptr(), pools._address,
        out.data_ptr(), ws.data_ptr(), ws.nbytes, _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_paged_attention_q4")


def paged_attention_q4(q, pools, pages, stream=None):
    """Allocates the output and the workspace and runs stlite_paged_attention_q4."""
    out, ws = torch.empty_like(q), paged_q4_workspace(q, pools, pages)
    _lend(stream, q, pools.k, pools.v, pools.k_scale, pools.v_scale, pools.k_factor, pools.v_factor, pages.table,
          pages.length, pages.cu_new, out, ws)
    stlite_paged_attention_q4(q, pools, pages, out, ws, stream)
    return out


def stlite_compact_paged_q4(layers, budget, pages, seq, stream=None):
    """The kept rows of every layer into sequence seq's 4-bit pages; layers:
    list of (k, v, pools, idx)."""
    k0 = layers[0][0]
    shape, dtype, dev, parts = k0.shape, k0.dtype, k0.get_device(), []
    n, hkv, d = shape
    kind, index = (*pages._pool, hkv), (hkv, budget)
    for k, v, pools, ix in layers:
        if pools._kind != kind:
            raise _q4_error()
        if not ((k is k0 or (k.shape == shape and k.dtype == dtype)) and v.shape == shape and v.dtype == dtype
                and ix.shape == index and ix.dtype == torch.int32 and k.is_contiguous() and v.is_contiguous()
                and ix.is_contiguous()):
            raise ValueError("every layer's k and v are [N][Hkv][128] of one type and idx int32 [Hkv][budget], "
                             "contiguous")
        if not k.get_device() == pools._device == ix.get_device() == dev or (v.get_device() != dev
                                                                             and not v.is_pinned()):
            raise ValueError(_ELSEWHERE)
        parts += (_ROWS.pack(0, k.data_ptr(), v.data_ptr(), ix.data_ptr()), pools._bytes)
    if dev < 0 or not torch._C._cuda_getDevice() == dev == pages._device:
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_compact_paged_q4(_SHAPE.pack(n, hkv, hkv, d, 1, _DTYPE[dtype]), budget, pages._address, seq,
                                      len(layers), b"".join(parts),
                                      _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_compact_paged_q4")


def stlite_compress_layers_paged_q4(layers, frames, params, pages, seq, ws, stream=None) -> int:
    """stlite_compress_layers with the kept rows in sequence seq's 4-bit
    pages; layers: list of (q, k, v, pools, idx_out)."""
    q0, k0 = layers[0][:2]
    sh = make_shape(q0, k0)
    qs, shape, dtype, dev, parts = q0.shape, k0.shape, k0.dtype, k0.get_device(), []
    kept = sh.n_kv_heads * stlite_budget(sh.n_tokens, params.beta, params.k_override)
    kind = (*pages._pool, sh.n_kv_heads)
    for q, k, v, pools, ix in layers:
        if pools._kind != kind:
            raise _q4_error()
        if not (q.shape == qs and k.shape == shape == v.shape and q.dtype == dtype == k.dtype and v.dtype == dtype
                and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("every layer's q is [w][Hq][128] and its k and v [N][Hkv][128], of one type, contiguous")
        if ix.dtype != torch.int32 or ix.numel() < kept or not ix.is_contiguous():
            raise ValueError("every layer's idx_out is contiguous int32 with room for [Hkv][B]")
        if not q.get_device() == k.get_device() == pools._device == ix.get_device() == dev or (
                v.get_device() != dev and not v.is_pinned()):
            raise ValueError(_ELSEWHERE)
        parts += (_ROWS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), ix.data_ptr()), pools._bytes)
    if dev < 0 or not torch._C._cuda_getDevice() == dev == pages._device == ws.get_device():
        raise ValueError(_ELSEWHERE)
    fs = _frames(frames)
    b = ctypes.c_int32(0)
    _check(_lib.stlite_compress_layers_paged_q4(ctypes.byref(sh), ctypes.byref(fs.c), ctypes.byref(params),
                                                pages._address, int(seq), len(layers), b"".join(parts), ctypes.byref(b),
                                                _ptr(ws), ws.numel(), _stream(stream)),
           "stlite_compress_layers_paged_q4")
    return int(b.value)


def stlite_paged_fetch_q4(layers, pages, stream=None):
    """Rows out of every layer's 4-bit pages, as values: the last cu_new[s + 1]
    - cu_new[s] (or max_new) rows of each sequence; layers: list of (pools, k_out,
    v_out), outputs [T][Hkv][128]."""
    k0 = layers[0][1]
    shape, dtype, dev, parts = k0.shape, k0.dtype, k0.get_device(), []
    n, hkv, d = shape
    kind = (*pages._pool, hkv)
    for pools, k, v in layers:
        if pools._kind != kind:
            raise _q4_error()
        if not ((k is k0 or (k.shape == shape and k.dtype == dtype)) and v.shape == shape and v.dtype == dtype
                and d == 128 and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("every layer's outputs are contiguous [T][Hkv][128] of one type")
        if not k.get_device() == v.get_device() == pools._device == dev:
            raise ValueError(_ELSEWHERE)
        parts += (_ROWS.pack(0, k.data_ptr(), v.data_ptr(), 0), pools._bytes)
    if dev < 0 or not torch._C._cuda_getDevice() == dev == pages._device:
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_paged_fetch_q4(
        _SHAPE.pack(n, hkv, hkv, 128, pages.max_new if pages.cu_new is None else 1, _DTYPE[dtype]), pages._address,
        len(layers), b"".join(parts), _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_paged_fetch_q4")


def paged_fetch_q4(pools, pages, n, dtype=torch.bfloat16, stream=None):
    """Allocates the outputs and runs stlite_paged_fetch_q4 on one layer for
    the n packed tokens of pages; rows that it leaves out are zeros."""
    k, v = (torch.zeros((n, pools.hkv, 128), dtype=dtype, device=pools.k.device) for _ in range(2))
    _lend(stream, pools.k, pools.v, pools.k_scale, pools.v_scale, pools.k_factor, pools.v_factor, pages.table,
          pages.length, pages.cu_new, k, v)
    stlite_paged_fetch_q4([(pools, k, v)], pages, stream)
    return k, v


# ------------------------------------------------------- a step's page tables

def stlite_pages_step(pages, keep, fresh, free_pages, n_free, slot, stream=None):
    """Gives pages to the sessions that grow and takes them from those that
    shrink or end: updates pages.table, length and cu_new, free_pages [n_pages]
    and n_free [1].  keep [S] (or None: all): rows that stay; fresh [S]: new
    tokens asked for; slot: int32 [n_tokens], the place of every new token, or
    the number of places.  All int32."""
    dev, S, i32 = pages._device, pages.c.n_seqs, torch.int32
    if pages.length is None or pages.cu_new is None:
        raise ValueError("a step's pages have length and cu_new")
    places = slot if isinstance(slot, int) else slot.shape[0] if slot.dim() == 1 else -1
    if (fresh.dtype != i32 or fresh.shape != (S,) or not fresh.is_contiguous() or free_pages.dtype != i32
            or free_pages.shape != pages._pool[:1] or not free_pages.is_contiguous() or n_free.dtype != i32
            or n_free.numel() != 1 or (keep is not None and (keep.dtype != i32 or keep.shape != (S,)
                                                             or not keep.is_contiguous()))
            or places < 0 or (slot is not places and (slot.dtype != i32 or not slot.is_contiguous()))):
        raise ValueError("keep and fresh are [S], free_pages [n_pages], n_free [1] and slot [n_tokens], contiguous int32")
    if dev < 0 or not torch._C._cuda_getDevice() == dev == fresh.get_device() == free_pages.get_device() == (
            n_free.get_device()) or (keep is not None and keep.get_device() != dev) or (
            slot is not places and slot.get_device() != dev):
        raise ValueError(_ELSEWHERE)
    st = _lib.stlite_pages_step(pages._address, None if keep is None else keep.data_ptr(), fresh.data_ptr(),
                                free_pages.data_ptr(), n_free.data_ptr(), places,
                                None if slot is places or places == 0 else slot.data_ptr(),
                                _CURRENT(dev) if stream is None else stream.cuda_stream)
    if st != STLITE_OK:
        raise StliteError(st, "stlite_pages_step")


def stlite_selftest_wait_timeout(ws, limit_ns: int, stream=None):
    """Runs the failure-path diagnostic: a bounded wait that runs out after
    limit_ns and records STLITE_ETIMEOUT in ws's error word."""
    _check(_lib.stlite_selftest_wait_timeout(_ptr(ws), int(limit_ns), _stream(stream)),
           "stlite_selftest_wait_timeout")


def stlite_device_status(ws, stream=None) -> int:
    """Reads and clears a workspace's device error word; ws=None reads the
    error word of stlite_score_noalloc's fixed scratch on the current device."""
    st = ctypes.c_int32(0)
    _check(_lib.stlite_device_status(_ptr(ws), _stream(stream), ctypes.byref(st)), "stlite_device_status")
    return int(st.value)


def stlite_score_noalloc(q, k, a_base, stream=None):
    """Window score without a workspace (for callers that cannot allocate
    device memory); see include/stlite.h."""
    sh = make_shape(q, k)
    _check(_lib.stlite_score_noalloc(ctypes.byref(sh), _ptr(q), _ptr(k), _ptr(a_base), _stream(stream)),
           "stlite_score_noalloc")


def stlite_timing_enable(on: bool = True):
    _check(_lib.stlite_timing_enable(1 if on else 0), "stlite_timing_enable")


def stlite_timing_read() -> dict:
    """{kernel name: (launches, total device ms)} since the last read."""
    cap = 64
    buf = (KernelTime * cap)()
    cnt = ctypes.c_int32(0)
    _check(_lib.stlite_timing_read(buf, cap, ctypes.byref(cnt)), "stlite_timing_read")
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(min(cnt.value, cap))}


# ------------------------------------------------------- convenience layer

def compress_layer(q, k, v, frames, beta=0.2, k_override=0, alpha=1.0, tsg_enable=1, css_enable=1,
                   ws=None, stream=None, tsg_metric=STLITE_TSG_COSINE, fixed_tau=None, base_scorer=STLITE_BASE_WINDOW,
                   abase_norm=STLITE_ABASE_RAW, css_size=3):
    """Allocates outputs (and a workspace if none is given) and runs
    stlite_compress_layer.  Returns (k_out, v_out, idx)."""
    fs = _frames(frames)
    params = make_params(beta, k_override, alpha, tsg_enable, css_enable, tsg_metric, fixed_tau, base_scorer,
                         abase_norm, css_size)
    sh = make_shape(q, k)
    b = stlite_budget(sh.n_tokens, beta, k_override)
    if b < 1:
        raise StliteError(STLITE_EINVAL, "stlite_budget")
    if ws is None:
        ws = workspace(sh, fs, params, device=k.device)
    k_out = torch.empty((b, sh.n_kv_heads, sh.head_dim), dtype=k.dtype, device=k.device)
    v_out = torch.empty_like(k_out)
    idx = torch.empty((sh.n_kv_heads, b), dtype=torch.int32, device=k.device)
    _lend(stream, q, k, v, ws, k_out, v_out, idx)
    stlite_compress_layer(q, k, v, fs, params, k_out, v_out, idx, ws, stream)
    return k_out, v_out, idx

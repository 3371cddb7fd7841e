"""Thin ctypes binding of libomnimem.so (the C ABI in include/omnimem.h).

Argument marshalling only: every stage of the compression step runs in the
library's HIP kernels.  torch tensors serve as device buffers and streams.
There is no fallback: if the library is missing or fails to load, every
call raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import typing

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libomnimem.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_INFEASIBLE, ERR_CAPACITY, ERR_HIP = range(6)
BF16, F32 = 0, 1
SIM_MAX, SIM_ADJ = 0, 1
SRC_VALUES, SRC_KEYS, SRC_HIDDEN = 0, 1, 2
TOPK_AUTO, TOPK_REGISTERS, TOPK_ONE_WORKGROUP, TOPK_SPLIT = 0, 1, 2, 3

EXPORTED = [
    "omnimem_config_default", "omnimem_create", "omnimem_destroy", "omnimem_last_error",
    "omnimem_score", "omnimem_redundancy", "omnimem_allocate", "omnimem_select_compact",
    "omnimem_calibrate", "omnimem_calibration_reset", "omnimem_calibration_budgets",
    "omnimem_allocate_fixed", "omnimem_profile", "omnimem_profile_report", "omnimem_inplace_status",
    "omnimem_append", "omnimem_allocate_noalloc", "omnimem_set_topk_path",
    "omnimem_attn_create", "omnimem_attn_destroy", "omnimem_attn_last_error", "omnimem_rotate", "omnimem_pack",
    "omnimem_unpack", "omnimem_memory_bytes", "omnimem_attend",
]


class OmnimemError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"omnimem status {status}: {message}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("lambda_", ctypes.c_float),
        ("ratio_r", ctypes.c_float), ("temperature", ctypes.c_float), ("b_min_frac", ctypes.c_float),
        ("b_max_frac", ctypes.c_float), ("causal", ctypes.c_int32), ("sim", ctypes.c_int32),
        ("sim_source", ctypes.c_int32), ("shared_selection", ctypes.c_int32), ("max_tokens", ctypes.c_int64),
        ("max_chunk", ctypes.c_int64), ("hidden_dim", ctypes.c_int32), ("inplace_stage_rows", ctypes.c_int32),
    ]


class Layer(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("q_head_stride", ctypes.c_int64), ("q_row_stride", ctypes.c_int64),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("kv_head_stride", ctypes.c_int64),
        ("kv_row_stride", ctypes.c_int64), ("modality", ctypes.c_void_p), ("n_cache", ctypes.c_int64),
        ("n_chunk", ctypes.c_int64), ("sm_scale", ctypes.c_float), ("lse", ctypes.c_void_p),
        ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p), ("out_head_stride", ctypes.c_int64),
        ("out_row_stride", ctypes.c_int64), ("hidden", ctypes.c_void_p), ("hidden_row_stride", ctypes.c_int64),
        ("hidden_out", ctypes.c_void_p), ("hidden_out_row_stride", ctypes.c_int64), ("out_rows", ctypes.c_int64),
        ("modality_out", ctypes.c_void_p),
    ]


class Chunk(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("head_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64), ("modality", ctypes.c_void_p), ("n_rows", ctypes.c_int64),
    ]


class AttnConfig(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class Rope(ctypes.Structure):
    _fields_ = [
        ("rotary_dim", ctypes.c_int32), ("neighbours", ctypes.c_int32), ("n_axes", ctypes.c_int32),
        ("inv_freq", ctypes.POINTER(ctypes.c_double)), ("axis", ctypes.POINTER(ctypes.c_uint8)),
        ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
    ]


class Projection(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("q_head_stride", ctypes.c_int64), ("q_row_stride", ctypes.c_int64),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("kv_head_stride", ctypes.c_int64),
        ("kv_row_stride", ctypes.c_int64), ("pos", ctypes.c_void_p), ("pos_stride", ctypes.c_int64),
        ("modality", ctypes.c_void_p), ("n_rows", ctypes.c_int64), ("q_out", ctypes.c_void_p),
        ("q_out_head_stride", ctypes.c_int64), ("q_out_row_stride", ctypes.c_int64), ("k_out", ctypes.c_void_p),
        ("v_out", ctypes.c_void_p), ("out_head_stride", ctypes.c_int64), ("out_row_stride", ctypes.c_int64),
        ("modality_out", ctypes.c_void_p),
    ]


class Held(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("kv_head_stride", ctypes.c_int64),
        ("kv_row_stride", ctypes.c_int64), ("data", ctypes.c_void_p), ("data_head_stride", ctypes.c_int64),
        ("n_rows", ctypes.c_int64),
    ]


class Query(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("q_head_stride", ctypes.c_int64), ("q_row_stride", ctypes.c_int64),
        ("n_queries", ctypes.c_int64), ("memory", ctypes.c_void_p), ("memory_head_stride", ctypes.c_int64),
        ("memory_rows", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("kv_head_stride", ctypes.c_int64), ("kv_row_stride", ctypes.c_int64), ("n_tail", ctypes.c_int64),
        ("sm_scale", ctypes.c_float), ("out", ctypes.c_void_p), ("out_head_stride", ctypes.c_int64),
        ("out_row_stride", ctypes.c_int64), ("lse", ctypes.c_void_p), ("lse_head_stride", ctypes.c_int64),
    ]


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


_lib = None


def load_library(path=LIB_PATH):
    """Load libomnimem.so; raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2606_07577_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.omnimem_config_default.argtypes = [ctypes.POINTER(Config)]
    lib.omnimem_config_default.restype = None
    lib.omnimem_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
    lib.omnimem_create.restype = i32
    lib.omnimem_destroy.argtypes = [vp]
    lib.omnimem_destroy.restype = i32
    lib.omnimem_last_error.argtypes = [vp]
    lib.omnimem_last_error.restype = ctypes.c_char_p
    lib.omnimem_score.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, vp]
    lib.omnimem_score.restype = i32
    lib.omnimem_redundancy.argtypes = [vp, ctypes.POINTER(Layer), vp, vp]
    lib.omnimem_redundancy.restype = i32
    lib.omnimem_allocate.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, i64, vp, vp, vp]
    lib.omnimem_allocate.restype = i32
    lib.omnimem_select_compact.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, vp, vp, vp]
    lib.omnimem_select_compact.restype = i32
    lib.omnimem_calibrate.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, vp, vp]
    lib.omnimem_calibrate.restype = i32
    lib.omnimem_calibration_reset.argtypes = [vp]
    lib.omnimem_calibration_reset.restype = i32
    lib.omnimem_calibration_budgets.argtypes = [vp, i64, vp, vp]
    lib.omnimem_calibration_budgets.restype = i32
    lib.omnimem_allocate_fixed.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, vp, vp, vp, vp]
    lib.omnimem_allocate_fixed.restype = i32
    lib.omnimem_allocate_noalloc.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(Layer), vp, vp, i64, vp, vp, vp]
    lib.omnimem_allocate_noalloc.restype = i32
    lib.omnimem_inplace_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
    lib.omnimem_inplace_status.restype = i32
    lib.omnimem_append.argtypes = [vp, ctypes.POINTER(Layer), ctypes.POINTER(Chunk), vp]
    lib.omnimem_append.restype = i32
    lib.omnimem_set_topk_path.argtypes = [vp, i32]
    lib.omnimem_set_topk_path.restype = i32
    lib.omnimem_profile.argtypes = [vp, ctypes.c_int32]
    lib.omnimem_profile.restype = i32
    lib.omnimem_profile_report.argtypes = [vp, ctypes.POINTER(KernelTime), ctypes.c_int32,
                                           ctypes.POINTER(ctypes.c_int32)]
    lib.omnimem_profile_report.restype = i32
    lib.omnimem_attn_create.argtypes = [ctypes.POINTER(AttnConfig), ctypes.POINTER(vp)]
    lib.omnimem_attn_create.restype = i32
    lib.omnimem_attn_destroy.argtypes = [vp]
    lib.omnimem_attn_destroy.restype = i32
    lib.omnimem_attn_last_error.argtypes = [vp]
    lib.omnimem_attn_last_error.restype = ctypes.c_char_p
    lib.omnimem_rotate.argtypes = [vp, ctypes.POINTER(Rope), ctypes.POINTER(Projection), ctypes.c_int32, vp]
    lib.omnimem_rotate.restype = i32
    lib.omnimem_pack.argtypes = [vp, ctypes.POINTER(Held), ctypes.c_int32, vp]
    lib.omnimem_pack.restype = i32
    lib.omnimem_unpack.argtypes = [vp, ctypes.POINTER(Held), ctypes.c_int32, vp]
    lib.omnimem_unpack.restype = i32
    lib.omnimem_memory_bytes.argtypes = [ctypes.c_int32, i64]
    lib.omnimem_memory_bytes.restype = ctypes.c_int64
    lib.omnimem_attend.argtypes = [vp, ctypes.POINTER(Query), ctypes.c_int32, ctypes.c_int32, vp]
    lib.omnimem_attend.restype = i32
    _lib = lib
    return lib


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("device tensors (torch, cuda) are required")
    return t.data_ptr()


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def make_layer(q, k, v, modality, n_cache, sm_scale=0.0, lse=None, k_out=None, v_out=None, hidden=None,
               hidden_out=None, out_rows=0, modality_out=None, n=None):
    """Descriptor of one layer's working set from device tensors.

    q [H_q, C, d]; k, v [H_kv, >=N, d] (the working set is their first N
    rows, N = k.shape[1] unless given); modality uint8 [>=N]; optional lse
    [H_q, C] fp32; optional k_out, v_out [H_kv, out_rows, d] (same strides;
    k_out is k and v_out is v for compaction in place); optional hidden
    [N, d_model] and hidden_out [>=M, d_model]; optional modality_out uint8.
    """
    if k.stride() != v.stride():
        raise ValueError("k and v must share strides")
    if k_out is not None and (v_out is None or k_out.stride() != v_out.stride()):
        raise ValueError("k_out and v_out must both be given with equal strides")
    if modality.dtype != torch.uint8:
        raise TypeError("modality must be uint8")
    n = k.shape[1] if n is None else int(n)
    lay = Layer()
    lay.q = _ptr(q)
    lay.q_head_stride, lay.q_row_stride = (q.stride(0), q.stride(1)) if q is not None else (0, 0)
    lay.k, lay.v = _ptr(k), _ptr(v)
    lay.kv_head_stride, lay.kv_row_stride = k.stride(0), k.stride(1)
    lay.modality = _ptr(modality)
    lay.n_cache = int(n_cache)
    lay.n_chunk = int(n - n_cache)
    lay.sm_scale = float(sm_scale)
    lay.lse = _ptr(lse)
    if k_out is not None:
        lay.k_out, lay.v_out = _ptr(k_out), _ptr(v_out)
        lay.out_head_stride, lay.out_row_stride = k_out.stride(0), k_out.stride(1)
        lay.out_rows = int(out_rows)
    if modality_out is not None:
        if modality_out.dtype != torch.uint8:
            raise TypeError("modality_out must be uint8")
        lay.modality_out = _ptr(modality_out)
    if hidden is not None:
        lay.hidden, lay.hidden_row_stride = _ptr(hidden), hidden.stride(0)
    if hidden_out is not None:
        lay.hidden_out, lay.hidden_out_row_stride = _ptr(hidden_out), hidden_out.stride(0)
    return lay


class Context:
    """An omnimem_ctx: workspace for the given capacities on the current device."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, max_tokens, max_chunk,
                 dtype=BF16, **options):
        lib = load_library()
        cfg = Config()
        lib.omnimem_config_default(ctypes.byref(cfg))
        cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        cfg.dtype, cfg.max_tokens, cfg.max_chunk = dtype, max_tokens, max_chunk
        for key, val in options.items():
            setattr(cfg, "lambda_" if key == "lam" else key, val)
        self.cfg = cfg
        self._lib = lib
        handle = ctypes.c_void_p()
        st = lib.omnimem_create(ctypes.byref(cfg), ctypes.byref(handle))
        if st != OK:
            raise OmnimemError(st, lib.omnimem_last_error(None).decode())
        self.handle = handle

    @staticmethod
    def default_config():
        """The library's default omnimem_config (sizes 0)."""
        cfg = Config()
        load_library().omnimem_config_default(ctypes.byref(cfg))
        return cfg

    def _check(self, st):
        if st != OK:
            raise OmnimemError(st, self._lib.omnimem_last_error(self.handle).decode())

    def _layers(self, layers):
        if len(layers) != self.cfg.n_layers:
            raise ValueError(f"expected {self.cfg.n_layers} layer descriptors")
        if isinstance(layers, ctypes.Array) and layers._type_ is Layer:
            return layers
        return (Layer * len(layers))(*layers)

    def close(self):
        if self.handle:
            self._lib.omnimem_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # The four stages of the C ABI, same names.
    def omnimem_score(self, layers, a, lse_out=None, stream=None):
        self._check(self._lib.omnimem_score(self.handle, self._layers(layers), _ptr(a), _ptr(lse_out),
                                            _stream(stream)))

    def omnimem_redundancy(self, layers, s, stream=None):
        self._check(self._lib.omnimem_redundancy(self.handle, self._layers(layers), _ptr(s), _stream(stream)))

    def omnimem_allocate(self, layers, a, s, total_budget, budgets, stats=None, stream=None):
        self._check(self._lib.omnimem_allocate(self.handle, self._layers(layers), _ptr(a), _ptr(s),
                                               int(total_budget), _ptr(budgets), _ptr(stats), _stream(stream)))

    def omnimem_select_compact(self, layers, a, s, budgets, idx=None, stream=None):
        self._check(self._lib.omnimem_select_compact(self.handle, self._layers(layers), _ptr(a), _ptr(s),
                                                     _ptr(budgets), _ptr(idx), _stream(stream)))

    # Offline budgets (calibration), same names as the C ABI.
    def omnimem_calibrate(self, layers, a, s, stats=None, stream=None):
        self._check(self._lib.omnimem_calibrate(self.handle, self._layers(layers), _ptr(a), _ptr(s), _ptr(stats),
                                                _stream(stream)))

    def omnimem_calibration_reset(self):
        self._check(self._lib.omnimem_calibration_reset(self.handle))

    def omnimem_calibration_budgets(self, total_budget, layer_budgets, stream=None):
        self._check(self._lib.omnimem_calibration_budgets(self.handle, int(total_budget), _ptr(layer_budgets),
                                                          _stream(stream)))

    def omnimem_allocate_fixed(self, layers, a, s, layer_budgets, budgets, stats=None, stream=None):
        self._check(self._lib.omnimem_allocate_fixed(self.handle, self._layers(layers), _ptr(a), _ptr(s),
                                                     _ptr(layer_budgets), _ptr(budgets), _ptr(stats),
                                                     _stream(stream)))


    def omnimem_inplace_status(self):
        """Largest staging need of the in-place compactions since the last
        query (0: none); raises OmnimemError when one moved nothing for lack
        of staging rows or an ordering wait gave up.  Synchronous."""
        need = ctypes.c_int64()
        self._check(self._lib.omnimem_inplace_status(self.handle, ctypes.byref(need)))
        return need.value

    def omnimem_append(self, layers, chunks, stream=None):
        if len(chunks) != self.cfg.n_layers:
            raise ValueError(f"expected {self.cfg.n_layers} chunk descriptors")
        arr = chunks if isinstance(chunks, ctypes.Array) else (Chunk * len(chunks))(*chunks)
        self._check(self._lib.omnimem_append(self.handle, self._layers(layers), arr, _stream(stream)))

    def omnimem_set_topk_path(self, path):
        """Ranking path of later select_compact calls (TOPK_AUTO,
        TOPK_REGISTERS, TOPK_ONE_WORKGROUP or TOPK_SPLIT)."""
        self._check(self._lib.omnimem_set_topk_path(self.handle, int(path)))

    def omnimem_profile(self, on):
        self._check(self._lib.omnimem_profile(self.handle, int(bool(on))))

    def omnimem_profile_report(self):
        """{kernel name: (launches, total milliseconds)} of the recorded launches."""
        buf = (KernelTime * 32)()
        n = ctypes.c_int32()
        self._check(self._lib.omnimem_profile_report(self.handle, buf, 32, ctypes.byref(n)))
        return {buf[i].name.decode(): (buf[i].launches, buf[i].total_ms) for i in range(n.value)}


def allocate_noalloc(cfg, layers, a, s, total_budget, budgets, stats=None, stream=None):
    """omnimem_allocate_noalloc: the allocation stage with no context and no
    device allocation (cfg is a Config; layers a list of Layer)."""
    lib = load_library()
    arr = layers if isinstance(layers, ctypes.Array) else (Layer * len(layers))(*layers)
    st = lib.omnimem_allocate_noalloc(ctypes.byref(cfg), arr, _ptr(a), _ptr(s), int(total_budget), _ptr(budgets),
                                      _ptr(stats), _stream(stream))
    if st != OK:
        raise OmnimemError(st, lib.omnimem_last_error(None).decode())


def make_chunk(k, v, modality):
    """Descriptor of one layer's new chunk rows: k, v [H_kv, C, d] (equal
    strides), modality uint8 [C] (device tensors)."""
    if k.stride() != v.stride():
        raise ValueError("chunk k and v must share strides")
    if modality.dtype != torch.uint8:
        raise TypeError("modality must be uint8")
    ch = Chunk()
    ch.k, ch.v = _ptr(k), _ptr(v)
    ch.head_stride, ch.row_stride = k.stride(0), k.stride(1)
    ch.modality = _ptr(modality)
    ch.n_rows = k.shape[1]
    return ch


MEMORY_ROWS = 32   # rows of a memory block


class _Layout(typing.NamedTuple):
    """What a descriptor's tensors say of the handle and the rope that they fit (None: nothing)."""
    n_q_heads: object = None
    n_kv_heads: object = None
    head_dim: object = None
    dtype: object = None
    device: object = None
    axes: object = None


def array_of(descriptors):
    """A ctypes array of descriptors of one type: built once, passed to any number of calls."""
    arr = (type(descriptors[0]) * len(descriptors))(*descriptors)
    arr._layouts = {d._layout for d in descriptors if hasattr(d, "_layout")}
    return arr


def columns_of(array):
    """A numpy structured view of a ctypes array of descriptors: array[i].f is columns["f"][i]."""
    kind = array._type_
    dtype = np.dtype({"names": [name for name, _ in kind._fields_],
                      "formats": ["u8" if t is ctypes.c_void_p else np.dtype(t) for _, t in kind._fields_],
                      "offsets": [getattr(kind, name).offset for name, _ in kind._fields_], "itemsize": ctypes.sizeof(kind)})
    return np.frombuffer(array, dtype=dtype)


def memory_shape(n_kv_heads, head_dim, rows):
    """Shape of the uint8 tensor that holds `rows` rows of every KV head in 4 bits."""
    return n_kv_heads, -(-int(rows) // MEMORY_ROWS), 34 * head_dim


def _rows(what, *tensors):
    """Tensors [heads, rows, d] of one type with their channels next to each other (k and v of one shape and strides)."""
    first = tensors[0]
    for t in tensors:
        if t.dim() != 3 or t.stride(2) != 1 or t.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"{what} must be [heads, rows, d], bf16 or fp32, its channels contiguous")
        if t.shape != first.shape or t.stride() != first.stride() or t.dtype != first.dtype:
            raise ValueError(f"{what} must share shape, strides and type")


def _one_device(*tensors):
    if len({t.device for t in tensors if t is not None}) != 1:
        raise ValueError("a descriptor's tensors must lie on one device")


def _memory(data, rows, k_like=None):
    if data.dtype != torch.uint8 or data.dim() != 3 or data.stride(2) != 1 or data.stride(1) != data.shape[2]:
        raise ValueError("a memory is a uint8 tensor [H_kv, blocks, 34 d], its blocks contiguous")
    if not 0 <= rows <= data.shape[1] * MEMORY_ROWS:
        raise ValueError(f"{rows} rows do not fit {data.shape[1]} blocks of {MEMORY_ROWS}")
    if k_like is not None and (data.shape[0] != k_like.shape[0] or data.shape[2] != 34 * k_like.shape[2]):
        raise ValueError("the memory's heads or width differ from the rows'")


def make_rope(head_dim, inv_freq, axis=None, n_axes=None, rotary_dim=None, neighbours=False, q_weight=None,
              k_weight=None, eps=1e-6):
    """Descriptor of a model's rotary positions: inv_freq (radians per position, one per pair of channels), axis (the
    position axis of each; default all 0), the leading rotary_dim channels of a head (default: two per frequency) paired
    j with j + rotary_dim/2, or 2j with 2j + 1 (neighbours), and optional norm weights [d] (device) for queries and keys."""
    freq = [float(f) for f in inv_freq]
    rot = 2 * len(freq) if rotary_dim is None else int(rotary_dim)
    if rot != 2 * len(freq) or rot > head_dim:
        raise ValueError(f"rotary_dim {rot} of {head_dim} channels takes {rot // 2} frequencies, got {len(freq)}")
    axis = [0] * len(freq) if axis is None else [int(a) for a in axis]
    if len(axis) != len(freq) or any(not 0 <= a < 4 for a in axis):
        raise ValueError("one axis in 0 .. 3 per frequency")
    weights = [w for w in (q_weight, k_weight) if w is not None]
    if any(w.shape != (head_dim,) or w.stride(0) != 1 for w in weights):
        raise ValueError(f"norm weights must be contiguous [{head_dim}]")
    r = Rope()
    r.rotary_dim, r.neighbours = rot, int(bool(neighbours))
    r.n_axes = int(n_axes) if n_axes is not None else max(axis, default=0) + 1
    r._freq, r._axis = (ctypes.c_double * max(1, len(freq)))(*freq), (ctypes.c_uint8 * max(1, len(freq)))(*axis)
    r.inv_freq, r.axis = r._freq, r._axis
    r.q_weight, r.k_weight, r.eps = _ptr(q_weight), _ptr(k_weight), float(eps)
    r._weights = weights    # (kept alive with the descriptor)
    r._layouts = {_Layout(head_dim=head_dim)} | {_Layout(dtype=w.dtype, device=w.device.index) for w in weights}
    return r


def make_projection(q, k, v, pos, q_out, k_out, v_out, modality=None, modality_out=None):
    """Descriptor of a sequence's projected rows q [H_q, n, d], k, v [H_kv, n, d] at positions pos int32 [axes, n], and
    of where they go: q_out [H_q, n, d]; k_out, v_out [H_kv, >= n, d] from the first row behind the cache."""
    n = k.shape[1]
    k_out, v_out = k_out[:, :n], v_out[:, :n]
    for what, group in (("q", (q,)), ("k and v", (k, v)), ("q_out", (q_out,)), ("k_out and v_out", (k_out, v_out))):
        _rows(what, *group)
    if q_out.shape != q.shape or k_out.shape != k.shape or q.shape[1:] != k.shape[1:]:
        raise ValueError("outputs must have their inputs' heads, rows and width")
    if len({t.dtype for t in (q, k, q_out, k_out)}) != 1:
        raise TypeError("rows must have one type")
    if pos.dtype != torch.int32 or pos.dim() != 2 or pos.shape[1] != n or pos.stride(1) != 1:
        raise ValueError("pos must be int32 [axes, n], its positions contiguous")
    for m in (modality, modality_out):
        if m is not None and (m.dtype != torch.uint8 or m.dim() != 1 or m.shape[0] < n or m.stride(0) != 1):
            raise TypeError("modality must be contiguous uint8 [>= n]")
    _one_device(q, k, v, pos, q_out, k_out, v_out, modality, modality_out)
    p = Projection()
    p.q, p.q_head_stride, p.q_row_stride = _ptr(q), q.stride(0), q.stride(1)
    p.k, p.v, p.kv_head_stride, p.kv_row_stride = _ptr(k), _ptr(v), k.stride(0), k.stride(1)
    p.pos, p.pos_stride, p.n_rows = _ptr(pos), pos.stride(0), n
    p.q_out, p.q_out_head_stride, p.q_out_row_stride = _ptr(q_out), q_out.stride(0), q_out.stride(1)
    p.k_out, p.v_out, p.out_head_stride, p.out_row_stride = _ptr(k_out), _ptr(v_out), k_out.stride(0), k_out.stride(1)
    p.modality, p.modality_out = _ptr(modality), _ptr(modality_out)
    p._layout = _Layout(q.shape[0], k.shape[0], q.shape[2], q.dtype, q.device.index, pos.shape[0])
    return p


def make_held(k, v, data):
    """Descriptor of rows k, v [H_kv, n, d] and the memory that holds them: uint8 of memory_shape (or with more blocks)."""
    _rows("k and v", k, v)
    _memory(data, k.shape[1], k)
    _one_device(k, v, data)
    h = Held()
    h.k, h.v, h.kv_head_stride, h.kv_row_stride = _ptr(k), _ptr(v), k.stride(0), k.stride(1)
    h.data, h.data_head_stride, h.n_rows = _ptr(data), data.stride(0), k.shape[1]
    h._layout = _Layout(None, k.shape[0], k.shape[2], k.dtype, k.device.index)
    return h


def make_query(q, out, k=None, v=None, memory=None, memory_rows=0, sm_scale=0.0, lse=None):
    """Descriptor of a sequence's queries q [H_q, n, d], their results out [H_q, n, d] (lse fp32 [H_q, n]) and the rows
    they attend to: memory_rows rows of an optional memory, then the tail rows k, v [H_kv, n_tail, d]."""
    _rows("q", q)
    _rows("out", out)
    if out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must have q's shape and type")
    if (k is None) != (v is None):
        raise ValueError("k and v must both be given")
    if k is not None:
        _rows("k and v", k, v)
        if k.dtype != q.dtype or k.shape[2] != q.shape[2]:
            raise ValueError("k and v must have q's type and width")
    if memory is not None:
        _memory(memory, int(memory_rows), k)
        if memory.shape[2] != 34 * q.shape[2]:
            raise ValueError("the memory's width differs from the queries'")
    elif memory_rows:
        raise ValueError("memory_rows without a memory")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or lse.stride(1) != 1):
        raise ValueError("lse must be fp32 [H_q, n], its queries contiguous")
    _one_device(q, out, k, v, memory, lse)
    x = Query()
    x.q, x.q_head_stride, x.q_row_stride, x.n_queries = _ptr(q), q.stride(0), q.stride(1), q.shape[1]
    x.out, x.out_head_stride, x.out_row_stride = _ptr(out), out.stride(0), out.stride(1)
    x.sm_scale = float(sm_scale)
    if k is not None:
        x.k, x.v, x.kv_head_stride, x.kv_row_stride, x.n_tail = _ptr(k), _ptr(v), k.stride(0), k.stride(1), k.shape[1]
    if memory is not None:
        x.memory, x.memory_head_stride, x.memory_rows = _ptr(memory), memory.stride(0), int(memory_rows)
    if lse is not None:
        x.lse, x.lse_head_stride = _ptr(lse), lse.stride(0)
    kv = k if k is not None else memory
    x._layout = _Layout(q.shape[0], kv.shape[0] if kv is not None else None, q.shape[2], q.dtype, q.device.index)
    return x


class Attention:
    """An omnimem_attn: the operators around the compression step for one head layout, on the current device.  Calls
    take lists of descriptors or arrays from array_of, one entry per sequence, of tensors on that device."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim, dtype=BF16):
        lib = load_library()
        self.handle = None
        self.cfg = AttnConfig(n_q_heads, n_kv_heads, head_dim, dtype)
        self._lib = lib
        handle = ctypes.c_void_p()
        st = lib.omnimem_attn_create(ctypes.byref(self.cfg), ctypes.byref(handle))
        if st != OK:
            raise OmnimemError(st, lib.omnimem_attn_last_error(None).decode())
        self.handle = handle
        self.device = torch.cuda.current_device()
        self._layout = _Layout(n_q_heads, n_kv_heads, head_dim, torch.bfloat16 if dtype == BF16 else torch.float32, self.device)
        self._fits = set()      # layouts that were compared

    def _check_layouts(self, layouts):
        for layout in layouts - self._fits:
            for name, want, got in zip(_Layout._fields, self._layout, layout):
                if want is not None and got is not None and want != got:
                    raise ValueError(f"the handle's {name} is {want}, a descriptor's {got}")
            self._fits.add(layout)

    def _call(self, function, descriptors, kind, *more, before=(), stream=None):
        if not (isinstance(descriptors, ctypes.Array) and descriptors._type_ is kind):
            descriptors = array_of(descriptors) if len(descriptors) else None
        n = len(descriptors) if descriptors is not None else 0
        self._check_layouts(getattr(descriptors, "_layouts", frozenset()))
        # (the raw handle costs a tenth of a microsecond, a Stream object a whole one: a fifth of a small call)
        s = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(self.device)
        st = function(self.handle, *before, descriptors, n, *more, s)
        if st != OK:
            raise OmnimemError(st, self._lib.omnimem_attn_last_error(self.handle).decode())

    # Same names as the C ABI.
    def omnimem_rotate(self, rope, projections, stream=None):
        self._check_layouts(getattr(rope, "_layouts", frozenset()))
        for layout in getattr(projections, "_layouts", None) or {p._layout for p in projections if hasattr(p, "_layout")}:
            if layout.axes < rope.n_axes:
                raise ValueError(f"the rope has {rope.n_axes} axes, a projection positions for {layout.axes}")
        self._call(self._lib.omnimem_rotate, projections, Projection, before=(ctypes.byref(rope),), stream=stream)

    def omnimem_pack(self, held, stream=None):
        self._call(self._lib.omnimem_pack, held, Held, stream=stream)

    def omnimem_unpack(self, held, stream=None):
        self._call(self._lib.omnimem_unpack, held, Held, stream=stream)

    def omnimem_attend(self, queries, causal=True, stream=None):
        self._call(self._lib.omnimem_attend, queries, Query, int(bool(causal)), stream=stream)

    def close(self):
        if self.handle:
            self._lib.omnimem_attn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def default_scale(head_dim):
    return 1.0 / math.sqrt(head_dim)

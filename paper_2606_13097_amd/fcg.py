"""Thin Python binding of libfcg.so (C ABI in include/fcg.h).

Argument marshalling only: every step of the grafting path runs in the HIP
kernels of libfcg.so.  Functions carry the C names.  Device tensors are torch
tensors on the GPU (only their ``data_ptr`` is passed); host index arrays are
anything ``numpy.asarray(..., int32)`` accepts.  A failing call raises
``FcgError`` with the status and the library's message.

If libfcg.so is missing this module raises at import: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
# PyTorch ships its own libamdhip64 (soname libamdhip64.so.7).  Loading torch
# first makes the dynamic linker bind libfcg.so to that same runtime, so
# torch's streams and allocations and libfcg's kernels share one HIP runtime.
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfcg.so")

FCG_F32, FCG_BF16 = 0, 1
FCG_LAYOUT_ONLY = 1
FCG_ALIAS_V = 2
STATUS = ["FCG_OK", "FCG_EINVAL", "FCG_ERANGE", "FCG_EOVERLAP", "FCG_EHOLE", "FCG_ENOMEM", "FCG_ESTATE",
          "FCG_EHIP"]
FCG_OK, FCG_EINVAL, FCG_ERANGE, FCG_EOVERLAP, FCG_EHOLE, FCG_ENOMEM, FCG_ESTATE, FCG_EHIP = range(8)

# every symbol include/fcg.h declares
EXPORTS = [
    "fcg_lib_create", "fcg_lib_add_segment", "fcg_lib_segment_info", "fcg_lib_device_ptrs", "fcg_lib_destroy",
    "fcg_lib_host_reserve", "fcg_lib_offload", "fcg_lib_reload", "fcg_lib_segment_state", "fcg_lib_update_residency",
    "fcg_cache_create", "fcg_cache_reset", "fcg_cache_truncate", "fcg_cache_export_layout", "fcg_cache_export_v_alias",
    "fcg_cache_device_ptrs",
    "fcg_cache_destroy", "fcg_graft", "fcg_patch_prefill", "fcg_decode", "fcg_decode_noalloc", "fcg_status_string",
    "fcg_last_error",
    "fcg_cache_timing", "fcg_cache_timing_read",
    "fcg_locality_create", "fcg_locality_record", "fcg_locality_set_ppl", "fcg_locality_scores",
    "fcg_locality_residency", "fcg_locality_destroy",
    "fcg_rope_create", "fcg_rope_frequencies", "fcg_rope_destroy", "fcg_rope_apply", "fcg_graft_rope", "fcg_append",
    "fcg_prefix_attend",
    "fcg_norm_rope_apply", "fcg_norm_rope_workspace", "fcg_norm_rope_backward", "fcg_append_norm",
    "fcg_attend_weights", "fcg_evict",
    "fcg_token_logprobs_workspace", "fcg_token_logprobs", "fcg_token_logprobs_backward", "fcg_locality_measure_ppl",
]
FCG_ROPE_HALF, FCG_ROPE_PAIRS = 0, 1
FCG_ROPE_PLAIN, FCG_ROPE_LINEAR, FCG_ROPE_NTK, FCG_ROPE_PARTS, FCG_ROPE_GIVEN = range(5)
FCG_ROPE_BACKWARD = 1
FCG_REPLACE = 1
FCG_ADD = 1
FCG_TIME_GRAFT, FCG_TIME_PREFILL_ATTN, FCG_TIME_PREFILL, FCG_TIME_DECODE, FCG_TIME_DECODE_ATTN = range(5)


class FcgError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS[status] if 0 <= status < len(STATUS) else status}: {msg}")
        self.status = status


class ModelDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("rope_theta", C.c_double), ("dtype", C.c_int32),
                ("rope_style", C.c_int32)]


class RopeDesc(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("theta", C.c_double),
                ("factor", C.c_double), ("orig_tokens", C.c_double), ("low_turns", C.c_double),
                ("high_turns", C.c_double), ("attn_factor", C.c_double), ("freqs", C.c_void_p)]


class TensorView(C.Structure):
    """``fcg_tensor``: address and strides (elements) of layer, token and head."""
    _fields_ = [("data", C.c_void_p), ("layer", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class NormDesc(C.Structure):
    """``fcg_norm``: weights of a row norm and their strides."""
    _fields_ = [("weight", C.c_void_p), ("layer", C.c_int64), ("head", C.c_int64), ("eps", C.c_double),
                ("offset", C.c_double)]


class NormSide(C.Structure):
    """``fcg_norm_side``: queries or keys of a norm's gradient."""
    _fields_ = [("heads", C.c_int32), ("norm", C.POINTER(NormDesc)), ("x", TensorView), ("grad", TensorView),
                ("dx", TensorView), ("dweight", C.c_void_p)]


def model_desc(n_layers, n_q_heads, n_kv_heads, head_dim, rope_theta, dtype) -> ModelDesc:
    dt = {"f32": FCG_F32, "bf16": FCG_BF16}.get(dtype, dtype)
    return ModelDesc(n_layers, n_q_heads, n_kv_heads, head_dim, float(rope_theta), int(dt), 0)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_13097_amd.build`")
    lib = C.CDLL(LIB_PATH)
    P, I32, I64, U32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
    PI32, PI64 = C.POINTER(C.c_int32), C.POINTER(C.c_int64)
    sig = {
        "fcg_lib_create": [C.POINTER(ModelDesc), I64, I32, U32, C.POINTER(P)],
        "fcg_lib_add_segment": [P, I32, I32, P, P, P, PI32],
        "fcg_lib_segment_info": [P, I32, PI64, PI32, PI32],
        "fcg_lib_device_ptrs": [P, I32, C.POINTER(P), C.POINTER(P)],
        "fcg_lib_destroy": [P],
        "fcg_lib_host_reserve": [P, I64],
        "fcg_lib_offload": [P, I32, P],
        "fcg_lib_reload": [P, I32, P],
        "fcg_lib_segment_state": [P, I32, PI32, PI32],
        "fcg_lib_update_residency": [P, P, I64, C.c_double, P, PI32, PI32],
        "fcg_cache_create": [C.POINTER(ModelDesc), I32, I32, I32, I32, U32, C.POINTER(P)],
        "fcg_cache_reset": [P, I32],
        "fcg_cache_truncate": [P, I32, I32, P],
        "fcg_cache_export_v_alias": [P, I32, P],
        "fcg_cache_export_layout": [P, I32, I32, P, PI32, P],
        "fcg_cache_device_ptrs": [P, I32, C.POINTER(P), C.POINTER(P)],
        "fcg_cache_destroy": [P],
        # int32 arrays go as plain addresses (ndarray.ctypes.data): no pointer objects per call
        "fcg_graft": [P, P, I32, P, P, P, P],
        "fcg_patch_prefill": [P, I32, I32, P, P, P, P, P, P, P],
        "fcg_decode": [P, I32, I32, P, P, P, P, P, P, P],
        "fcg_decode_noalloc": [P, I32, I32, P, P, P, P, P, P, P],
        "fcg_cache_timing": [P, I32],
        "fcg_cache_timing_read": [P, I32, PI32, C.POINTER(C.c_double)],
        "fcg_locality_create": [I32, I32, C.c_double, C.c_double, C.c_double, C.POINTER(P)],
        "fcg_locality_record": [P, I32, P],
        "fcg_locality_set_ppl": [P, I32, C.c_double],
        "fcg_locality_scores": [P, P],
        "fcg_locality_residency": [P, I64, P, P],
        "fcg_locality_destroy": [P],
    }
    PT = C.POINTER(TensorView)
    sig.update({
        "fcg_rope_create": [C.POINTER(RopeDesc), C.POINTER(P)],
        "fcg_rope_frequencies": [P, P],
        "fcg_rope_destroy": [P],
        "fcg_rope_apply": [P, I32, I32, I32, I32, P, I32, PT, PT, I32, PT, PT, U32, P],
        "fcg_graft_rope": [P, P, P, I32, P, P, P, P],
        "fcg_append": [P, I32, I32, I32, P, P, P, PT, PT, PT, PT, U32, P],
        "fcg_prefix_attend": [P, I32, I32, I32, I32, P, P, PT, PT, P, P],
    })
    PN, PS = C.POINTER(NormDesc), C.POINTER(NormSide)
    sig.update({
        "fcg_norm_rope_apply": [P, I32, I32, I32, I32, P, I32, PN, PT, PT, I32, PN, PT, PT, P],
        "fcg_norm_rope_workspace": [I32, I32, I32, I32, I32, PI64],
        "fcg_norm_rope_backward": [P, I32, I32, I32, I32, P, PS, PS, P, I64, P],
        "fcg_attend_weights": [P, I32, I32, I32, I32, P, P, PT, P, P, U32, P],
        "fcg_evict": [P, I32, P, P, P, I32, I32, P, P, P, P],
        "fcg_token_logprobs_workspace": [I32, I32, I32, PI64],
        "fcg_token_logprobs": [I32, I32, I32, P, I64, P, P, P, P, I32, P, P, P, I64, P],
        "fcg_token_logprobs_backward": [I32, I32, I32, P, I64, P, P, P, P, P, P, P, I64, P],
        "fcg_locality_measure_ppl": [P, I32, P, P, P, P],
        "fcg_append_norm": [P, I32, I32, I32, P, P, P, PN, PN, PT, PT, PT, PT, U32, P],
    })
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = C.c_int
    lib.fcg_status_string.argtypes = [C.c_int]
    lib.fcg_status_string.restype = C.c_char_p
    lib.fcg_last_error.argtypes = []
    lib.fcg_last_error.restype = C.c_char_p
    return lib


_L = _load()


def _check(status: int) -> None:
    if status != FCG_OK:
        raise FcgError(status, _L.fcg_last_error().decode())


def _i32(a) -> np.ndarray:
    if type(a) is np.ndarray and a.dtype == np.int32 and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


_first_byte = C.c_char.from_buffer


def _p(a: np.ndarray):
    """Address of an array's data (``.ctypes.data`` costs about two microseconds, this a third of one, but it takes
    writable arrays only)."""
    if not a.size:
        return None
    return C.addressof(_first_byte(a)) if a.flags.writeable else a.ctypes.data


_SMALL = 64  # int32 arrays up to this length go as ctypes arrays


def _i32_small(a):
    """An int32 array argument as (ctypes array or None, length).  Building a small
    ctypes array costs well under a microsecond; an ndarray's ``.ctypes.data``
    costs about two, and a decode call passes two such arrays."""
    vals = a.tolist() if isinstance(a, np.ndarray) else [int(x) for x in a]
    n = len(vals)
    return ((C.c_int32 * n)(*vals) if n else None), n


def _dptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _current_stream() -> Optional[int]:
    """Raw handle of torch's current stream on the current device (None without a GPU)."""
    import torch
    if not torch.cuda.is_available():
        return None
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # no Stream object per call
    if raw is not None:
        return raw(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class Library:
    """Handle of a segment library (``fcg_lib``)."""

    h = None

    def __init__(self, desc: ModelDesc, capacity_tokens: int, max_segments: int, flags: int = 0):
        h = C.c_void_p()
        _check(_L.fcg_lib_create(C.byref(desc), int(capacity_tokens), int(max_segments), int(flags), C.byref(h)))
        self.h, self.desc = h, desc
        self._lib = _L   # kept for close(), which may run while the interpreter tears down globals
        self.capacity = int(capacity_tokens)

    def close(self):
        if self.h:
            self._lib.fcg_lib_destroy(self.h)
            self.h = None

    __del__ = close


class Cache:
    """Handle of a composite cache (``fcg_cache``)."""

    h = None

    def __init__(self, desc: ModelDesc, n_seqs: int, max_tokens: int, page_size: int = 0, n_pages: int = 0,
                 flags: int = 0):
        h = C.c_void_p()
        _check(_L.fcg_cache_create(C.byref(desc), int(n_seqs), int(max_tokens), int(page_size), int(n_pages),
                                   int(flags), C.byref(h)))
        self.h, self.desc = h, desc
        self._lib = _L   # kept for close(), which may run while the interpreter tears down globals
        self.n_seqs, self.max_tokens, self.page_size, self.n_pages = n_seqs, max_tokens, page_size, n_pages
        # the device its memory is on (None: layout only)
        self.device = None if flags & FCG_LAYOUT_ONLY else torch.cuda.current_device()
        self.n_lp = -(-max_tokens // page_size) if page_size else 0

    def close(self):
        if self.h:
            self._lib.fcg_cache_destroy(self.h)
            self.h = None

    __del__ = close


def fcg_lib_create(desc: ModelDesc, capacity_tokens: int, max_segments: int, flags: int = 0) -> Library:
    return Library(desc, capacity_tokens, max_segments, flags)


def fcg_lib_add_segment(lib: Library, length: int, src_pos0: int, k=None, v=None, stream=None) -> int:
    sid = C.c_int32()
    _check(_L.fcg_lib_add_segment(lib.h, int(length), int(src_pos0), _dptr(k), _dptr(v),
                                  _stream(stream) if k is not None else None, C.byref(sid)))
    return sid.value


def fcg_lib_segment_info(lib: Library, seg_id: int):
    off, n, src = C.c_int64(), C.c_int32(), C.c_int32()
    _check(_L.fcg_lib_segment_info(lib.h, int(seg_id), C.byref(off), C.byref(n), C.byref(src)))
    return off.value, n.value, src.value


def fcg_lib_device_ptrs(lib: Library, layer: int):
    k, v = C.c_void_p(), C.c_void_p()
    _check(_L.fcg_lib_device_ptrs(lib.h, int(layer), C.byref(k), C.byref(v)))
    return k.value, v.value


def fcg_lib_destroy(lib: Library) -> None:
    lib.close()


def fcg_lib_host_reserve(lib: Library, host_tokens: int) -> None:
    _check(_L.fcg_lib_host_reserve(lib.h, int(host_tokens)))


def fcg_lib_offload(lib: Library, seg: int, stream=None) -> None:
    _check(_L.fcg_lib_offload(lib.h, int(seg), _stream(stream)))


def fcg_lib_reload(lib: Library, seg: int, stream=None) -> None:
    _check(_L.fcg_lib_reload(lib.h, int(seg), _stream(stream)))


def fcg_lib_segment_state(lib: Library, seg: int):
    """-> (in device memory, has a host copy)."""
    a, b = C.c_int32(), C.c_int32()
    _check(_L.fcg_lib_segment_state(lib.h, int(seg), C.byref(a), C.byref(b)))
    return bool(a.value), bool(b.value)


def fcg_lib_update_residency(lib: Library, loc: "Locality", budget_bytes: int = -1, ppl_threshold: float = 0.0,
                             stream=None):
    """The update step: offload / reload segments by locality under a byte budget -> (offloaded, reloaded)."""
    a, b = C.c_int32(), C.c_int32()
    _check(_L.fcg_lib_update_residency(lib.h, loc.h, int(budget_bytes), float(ppl_threshold),
                                       _stream(stream), C.byref(a), C.byref(b)))
    return a.value, b.value


def fcg_cache_create(desc: ModelDesc, n_seqs: int, max_tokens: int, page_size: int = 0, n_pages: int = 0,
                     flags: int = 0) -> Cache:
    return Cache(desc, n_seqs, max_tokens, page_size, n_pages, flags)


def fcg_cache_reset(cache: Cache, seq: int) -> None:
    _check(_L.fcg_cache_reset(cache.h, int(seq)))


def fcg_cache_truncate(cache: Cache, seq: int, pos: int, stream=None) -> None:
    """Keep positions [0, pos) of ``seq`` in every layer (cache-patching reuses that prefix)."""
    _check(_L.fcg_cache_truncate(cache.h, int(seq), int(pos), _stream(stream)))


def fcg_cache_export_v_alias(cache: Cache, seq: int) -> np.ndarray:
    """-> int32 [n_lp]: library token of each logical page's first position, -1 = own values."""
    out = np.zeros(max(cache.n_lp, 1), dtype=np.int32)
    _check(_L.fcg_cache_export_v_alias(cache.h, int(seq), out.ctypes.data))
    return out[:cache.n_lp]


def fcg_cache_export_layout(cache: Cache, seq: int, layer: int):
    """-> (page_table int32 [n_lp] or None, seq_len, written uint8 [max_tokens])."""
    pt = np.zeros(max(cache.n_lp, 1), dtype=np.int32)
    n = C.c_int32()
    wr = np.zeros(cache.max_tokens, dtype=np.uint8)
    _check(_L.fcg_cache_export_layout(cache.h, int(seq), int(layer), _p(pt) if cache.page_size else None,
                                      C.byref(n), wr.ctypes.data))
    return (pt[:cache.n_lp] if cache.page_size else None), n.value, wr


def fcg_cache_device_ptrs(cache: Cache, layer: int):
    k, v = C.c_void_p(), C.c_void_p()
    _check(_L.fcg_cache_device_ptrs(cache.h, int(layer), C.byref(k), C.byref(v)))
    return k.value, v.value


def fcg_cache_destroy(cache: Cache) -> None:
    cache.close()


def fcg_graft(cache: Cache, lib: Library, seq: Sequence[int], seg: Sequence[int], dst: Sequence[int],
              stream=None) -> None:
    s, g, d = _i32(seq), _i32(seg), _i32(dst)
    if not (s.size == g.size == d.size):
        raise ValueError("seq, seg and dst differ in length")
    _check(_L.fcg_graft(cache.h, lib.h, int(s.size), _p(s), _p(g), _p(d), _stream(stream)))


def fcg_patch_prefill(cache: Cache, layer: int, seq, pos, q, k, v, out, stream=None) -> None:
    s, p = _i32(seq), _i32(pos)
    if s.size != p.size:
        raise ValueError("seq and pos differ in length")
    _check(_L.fcg_patch_prefill(cache.h, int(layer), int(s.size), _p(s), _p(p), _dptr(q), _dptr(k), _dptr(v),
                                _dptr(out), _stream(stream) if q is not None else None))


def _decode_call(fn, cache: Cache, layer: int, seqs, q, k, v, out, stream) -> np.ndarray:
    if len(seqs) > _SMALL:
        s = _i32(seqs)
        pos = np.zeros(max(s.size, 1), dtype=np.int32)
        _check(fn(cache.h, int(layer), int(s.size), _p(s), _dptr(q), _dptr(k), _dptr(v), _dptr(out), pos.ctypes.data,
                  _stream(stream) if q is not None else None))
        return pos[:s.size]
    # one step of a small batch: the per-call marshalling is a visible part of the step
    s, n = _i32_small(seqs)
    pos = (C.c_int32 * max(n, 1))()
    _check(fn(cache.h, int(layer), n, s, _dptr(q), _dptr(k), _dptr(v), _dptr(out), pos,
              _stream(stream) if q is not None else None))
    return np.frombuffer(pos, dtype=np.int32, count=n)


def fcg_decode(cache: Cache, layer: int, seqs, q, k, v, out, stream=None) -> np.ndarray:
    return _decode_call(_L.fcg_decode, cache, layer, seqs, q, k, v, out, stream)


def fcg_decode_noalloc(cache: Cache, layer: int, seqs, q, k, v, out, stream=None) -> np.ndarray:
    """fcg_decode through the entry point that allocates nothing (static device scratch)."""
    return _decode_call(_L.fcg_decode_noalloc, cache, layer, seqs, q, k, v, out, stream)


def fcg_cache_timing(cache: Cache, enable: bool) -> None:
    _check(_L.fcg_cache_timing(cache.h, int(bool(enable))))


def fcg_cache_timing_read(cache: Cache, kind: int):
    """-> (number of recorded intervals, their summed duration in ms)."""
    n, ms = C.c_int32(), C.c_double()
    _check(_L.fcg_cache_timing_read(cache.h, int(kind), C.byref(n), C.byref(ms)))
    return n.value, ms.value


class Locality:
    """Handle of a locality scorer (``fcg_locality``)."""

    h = None

    def __init__(self, n_funcs: int, window: int = 20, alpha: float = 0.4, beta: float = 0.3, gamma: float = 0.3):
        h = C.c_void_p()
        _check(_L.fcg_locality_create(int(n_funcs), int(window), float(alpha), float(beta), float(gamma),
                                      C.byref(h)))
        self.h, self.n_funcs = h, int(n_funcs)
        self._lib = _L

    def close(self):
        if self.h:
            self._lib.fcg_locality_destroy(self.h)
            self.h = None

    __del__ = close


def fcg_locality_record(loc: Locality, func_ids) -> None:
    a = np.ascontiguousarray(func_ids, dtype=np.int32)
    _check(_L.fcg_locality_record(loc.h, len(a), a.ctypes.data if len(a) else None))


def fcg_locality_set_ppl(loc: Locality, func: int, ppl: float) -> None:
    _check(_L.fcg_locality_set_ppl(loc.h, int(func), float(ppl)))


def fcg_locality_scores(loc: Locality) -> np.ndarray:
    out = np.zeros(loc.n_funcs, dtype=np.float64)
    _check(_L.fcg_locality_scores(loc.h, out.ctypes.data))
    return out


def fcg_locality_residency(loc: Locality, budget: int, cost) -> np.ndarray:
    c = np.ascontiguousarray(cost, dtype=np.int64)
    if len(c) != loc.n_funcs:
        raise ValueError("one cost per function")
    out = np.zeros(loc.n_funcs, dtype=np.uint8)
    _check(_L.fcg_locality_residency(loc.h, int(budget), c.ctypes.data, out.ctypes.data))
    return out


# ------------------------------------------- rotary forms, appending, attention over a shared prefix

class Rope:
    """Handle of a rotary form (``fcg_rope``); host memory, any device."""

    h = None

    def __init__(self, desc: RopeDesc):
        h = C.c_void_p()
        _check(_L.fcg_rope_create(C.byref(desc), C.byref(h)))
        self.h, self.rotary_dim = h, desc.rotary_dim
        self._lib = _L

    def close(self):
        if self.h:
            self._lib.fcg_rope_destroy(self.h)
            self.h = None

    __del__ = close


def fcg_rope_create(rotary_dim: int, theta: float = 10000.0, layout: int = FCG_ROPE_HALF,
                    scaling: int = FCG_ROPE_PLAIN, factor: float = 1.0, orig_tokens: float = 0.0,
                    low_turns: float = 1.0, high_turns: float = 32.0, attn_factor: float = 1.0, freqs=None) -> Rope:
    w = None
    if freqs is not None:
        w = np.ascontiguousarray(freqs, dtype=np.float64)
        if w.shape != (int(rotary_dim) // 2,):
            raise ValueError("one frequency per rotary pair")
    return Rope(RopeDesc(int(rotary_dim), int(layout), int(scaling), float(theta), float(factor), float(orig_tokens),
                         float(low_turns), float(high_turns), float(attn_factor),
                         None if w is None else w.ctypes.data))


def fcg_rope_frequencies(rope: Rope) -> np.ndarray:
    out = np.zeros(rope.rotary_dim // 2, dtype=np.float64)
    _check(_L.fcg_rope_frequencies(rope.h, out.ctypes.data))
    return out


def fcg_rope_destroy(rope: Rope) -> None:
    rope.close()


_TORCH_DT = {torch.float32: FCG_F32, torch.bfloat16: FCG_BF16}
_DT_TORCH = {v: k for k, v in _TORCH_DT.items()}


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _view(t, shape: tuple, dtype, device, what: str):
    """fcg_tensor of a tensor of shape [n_layers][n_tok][n_heads][head_dim], or without the first dimension (one layer).
    One call makes up to four of these, a visible part of a small step, so the checks are few and plain."""
    if t is None:
        return None
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what}: requires a gradient, which these calls do not record (call under torch.no_grad(), "
                         "or from the forward of an autograd function)")
    if t.dtype is not dtype or (t.get_device() != device if device is not None else not t.is_cuda):
        raise ValueError(f"{what}: a {t.dtype} tensor on {t.device}, expected {dtype} on GPU {device}")
    st, sh = t.stride(), t.shape
    if sh != shape and (sh != shape[1:] or shape[0] != 1):
        raise ValueError(f"{what}: shape {tuple(sh)}, expected {shape} (one layer: or without the first dimension)")
    if st[-1] != 1 and t.numel():
        raise ValueError(f"{what}: the elements of a row must be adjacent")
    return TensorView(t.data_ptr(), *st[:3]) if len(st) == 4 else TensorView(t.data_ptr(), 0, st[0], st[1])


def _ref(v: Optional[TensorView]):
    return None if v is None else C.byref(v)


def _stream_of(stream, device) -> Optional[int]:
    """The given stream, or torch's current stream of ``device``."""
    if stream is not None:
        return _stream(stream)
    if device is None:
        return None
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def fcg_rope_apply(rope: Rope, pos, q=None, q_out=None, k=None, k_out=None, flags: int = 0, stream=None) -> None:
    """Encode q and k ([n][heads][head_dim], or with layers in front) at ``pos`` (int32 GPU tensor [n]) into q_out, k_out.
    Records no gradient (and refuses tensors that would need it): FCG_ROPE_BACKWARD is that of an autograd function."""
    if not pos.is_cuda or pos.dtype != torch.int32 or pos.dim() != 1 or not pos.is_contiguous():
        raise ValueError("pos: a contiguous int32 GPU tensor [n_tok]")
    like = q if q is not None else k
    if like is None:
        raise ValueError("neither q nor k")
    if like.dtype not in _TORCH_DT or like.dim() not in (3, 4):
        raise ValueError("a float32 or bfloat16 tensor of three or four dimensions")
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("an input without its output, or an output without its input")
    td, dev, n, d = like.dtype, pos.get_device(), pos.numel(), like.shape[-1]
    layers = like.shape[0] if like.dim() == 4 else 1
    hq, hk = 0 if q is None else q.shape[-2], 0 if k is None else k.shape[-2]
    sq, sk = (layers, n, hq, d), (layers, n, hk, d)
    vq, vqo = _view(q, sq, td, dev, "q"), _view(q_out, sq, td, dev, "q_out")
    vk, vko = _view(k, sk, td, dev, "k"), _view(k_out, sk, td, dev, "k_out")
    args = (rope.h, _TORCH_DT[td], d, layers, n, pos.data_ptr(), hq, _ref(vq), _ref(vqo), hk, _ref(vk), _ref(vko),
            int(flags), _stream_of(stream, dev))
    if dev == torch.cuda.current_device():
        _check(_L.fcg_rope_apply(*args))
    else:
        with torch.cuda.device(dev):
            _check(_L.fcg_rope_apply(*args))


def fcg_graft_rope(cache: Cache, lib: Library, rope: Rope, seq: Sequence[int], seg: Sequence[int], dst: Sequence[int],
                   stream=None) -> None:
    s, g, d = _i32(seq), _i32(seg), _i32(dst)
    if not (s.size == g.size == d.size):
        raise ValueError("seq, seg and dst differ in length")
    _check(_L.fcg_graft_rope(cache.h, lib.h, rope.h, int(s.size), _p(s), _p(g), _p(d), _stream_of(stream, cache.device)))


def fcg_append(cache: Cache, layer: int, seq, pos, k=None, v=None, rope: Optional[Rope] = None, q=None, q_out=None,
               flags: int = 0, stream=None, n_layers: int = 1) -> None:
    """Place k, v ([n][Hkv][D]: layer ``layer``; [L][n][Hkv][D]: the L layers from it) at (seq, pos), keys encoded;
    with q, its encoding goes to q_out.  Without k and v the positions of ``n_layers`` layers are reserved."""
    s, p = _i32(seq), _i32(pos)
    if s.ndim != 1 or s.shape != p.shape:
        raise ValueError("seq and pos differ in length")
    if q is not None and q_out is None:
        raise ValueError("q without q_out")
    if k is not None:
        layers = k.shape[0] if k.dim() == 4 else 1
        if n_layers != 1 and n_layers != layers:
            raise ValueError(f"n_layers {n_layers}, but k has {layers} layers")
        n_layers = layers
    d, n = cache.desc, int(s.size)
    sq, skv = (n_layers, n, d.n_q_heads, d.head_dim), (n_layers, n, d.n_kv_heads, d.head_dim)
    td, dev = _DT_TORCH[d.dtype], cache.device
    vq, vqo = _view(q, sq, td, dev, "q"), _view(q_out, sq, td, dev, "q_out")
    vk, vv = _view(k, skv, td, dev, "k"), _view(v, skv, td, dev, "v")
    _check(_L.fcg_append(cache.h, int(layer), int(n_layers), n, _p(s), _p(p), None if rope is None else rope.h,
                         _ref(vq), _ref(vqo), _ref(vk), _ref(vv), int(flags), _stream_of(stream, dev)))


def fcg_prefix_attend(cache: Cache, layer: int, prefix_seq: int, prefix_len: int, seq, pos, q, out, lse=None,
                      stream=None) -> None:
    """Attention of tokens (seq, pos) over positions [0, prefix_len) of prefix_seq and their own from prefix_len on.
    q (encoded) and out [n][Hq][D]; lse float32 [n][Hq] or None."""
    s, p = _i32(seq), _i32(pos)
    if s.ndim != 1 or s.shape != p.shape:
        raise ValueError("seq and pos differ in length")
    d, n = cache.desc, int(s.size)
    sq, td, dev = (1, n, d.n_q_heads, d.head_dim), _DT_TORCH[d.dtype], cache.device
    vq, vo = _view(q, sq, td, dev, "q"), _view(out, sq, td, dev, "out")
    if lse is not None and (not lse.is_cuda or lse.dtype != torch.float32 or not lse.is_contiguous() or
                            lse.shape != (n, d.n_q_heads) or lse.get_device() != cache.device):
        raise ValueError("lse: a contiguous float32 GPU tensor [n_tok][Hq]")
    _check(_L.fcg_prefix_attend(cache.h, int(layer), int(prefix_seq), int(prefix_len), n, _p(s), _p(p), _ref(vq),
                                _ref(vo), _dptr(lse), _stream_of(stream, cache.device)))


# ------------------------------------------- norms of queries and keys

class Norm:
    """A norm of rows (``fcg_norm``): (offset + weight) x / sqrt(mean(x^2) + eps) over each head.  weight: [head_dim],
    [heads][head_dim] or [layers][heads][head_dim] (a dimension of 1 is shared), or None for ones.  A call takes the
    weight's storage as it is then: a parameter may be moved or replaced between calls."""

    def __init__(self, weight=None, eps: float = 1e-6, offset: float = 0.0):
        self.weight = weight
        # one structure, brought up to date by each call (a new one is a visible part of a small step)
        self._desc = NormDesc(None, 0, 0, float(eps), float(offset))
        self._ref = C.byref(self._desc)
        self._lay_out()

    def __reduce__(self):                     # (a copy has a structure of its own)
        return Norm, (self.weight, self._desc.eps, self._desc.offset)

    def _lay_out(self) -> None:
        w, d = self.weight, self._desc
        self._shape, self._strides = (None, None) if w is None else (w.shape, w.stride())
        d.weight, d.layer, d.head = None, 0, 0
        if w is not None:
            sh, st = self._shape, self._strides
            if not 1 <= len(sh) <= 3 or (st[-1] != 1 and w.numel()):
                self._strides = None          # (looked at again in the next call)
                raise ValueError("norm weight: one to three dimensions, the elements of a head adjacent")
            d.weight = w.data_ptr()
            d.layer = st[0] if len(sh) == 3 and sh[0] > 1 else 0
            d.head = st[-2] if len(sh) > 1 and sh[-2] > 1 else 0

    @property
    def desc(self) -> NormDesc:
        """The description of the present weight."""
        self._lay_out()
        return self._desc

    def dweight_shape(self, layers: int, heads: int) -> tuple:
        """Shape of the weights' gradient: [layers][heads or 1][head_dim]."""
        return (layers, heads if self.desc.head and heads > 1 else 1, self.weight.shape[-1])


def _norm_ref(norm: Optional[Norm], layers: int, heads: int, d: int, dtype, device, what: str):
    if norm is None:
        return None
    w = norm.weight
    if w is None:
        if norm._shape is not None:
            norm._lay_out()
        return norm._ref
    if w.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what}: the weights require a gradient, which these calls do not record")
    if w.dtype is not dtype or w.get_device() != device:
        raise ValueError(f"{what}: weights of {w.dtype} on {w.device}, expected {dtype} on GPU {device}")
    sh = w.shape
    if w.stride() != norm._strides or sh != norm._shape:
        norm._lay_out()
    norm._desc.weight = w.data_ptr()
    if sh[-1] != d or (len(sh) > 1 and sh[-2] not in (1, heads)) or (len(sh) > 2 and sh[0] not in (1, layers)):
        raise ValueError(f"{what}: weights of shape {tuple(sh)} for {layers} layers of {heads} heads of {d}")
    return norm._ref


def _rows_of(pos, q, k):
    """(dtype, device, layers, tokens, head_dim, query heads, key heads) of the rows at ``pos``."""
    if not pos.is_cuda or pos.dtype != torch.int32 or pos.dim() != 1 or not pos.is_contiguous():
        raise ValueError("pos: a contiguous int32 GPU tensor [n_tok]")
    like = q if q is not None else k
    if like is None:
        raise ValueError("neither q nor k")
    if like.dtype not in _TORCH_DT or like.dim() not in (3, 4):
        raise ValueError("a float32 or bfloat16 tensor of three or four dimensions")
    layers = like.shape[0] if like.dim() == 4 else 1
    return (like.dtype, pos.get_device(), layers, pos.numel(), like.shape[-1], 0 if q is None else q.shape[-2],
            0 if k is None else k.shape[-2])


def _on_device(dev: int, fn, args) -> None:
    if dev == torch.cuda.current_device():
        _check(fn(*args))
    else:
        with torch.cuda.device(dev):
            _check(fn(*args))


def _workspace(given, nbytes: int, dev: int, stream):
    """(address, bytes) of a call's workspace; without one, memory of the current stream's pool."""
    if given is None:
        if not nbytes:
            return None, 0, None
        if stream is not None and _stream(stream) != _stream_of(None, dev):
            raise ValueError("a call on a stream other than the current one needs a workspace of its own")
        given = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{dev}")
    if given.get_device() != dev or not given.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor on GPU {dev}")
    return given.data_ptr(), given.numel() * given.element_size(), given


def fcg_norm_rope_apply(rope: Rope, pos, q=None, q_norm: Optional[Norm] = None, q_out=None, k=None,
                        k_norm: Optional[Norm] = None, k_out=None, stream=None) -> None:
    """``fcg_rope_apply`` of rows that q_norm and k_norm normalise first; records no gradient either."""
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("an input without its output, or an output without its input")
    td, dev, layers, n, d, hq, hk = _rows_of(pos, q, k)
    sq, sk = (layers, n, hq, d), (layers, n, hk, d)
    vq, vqo = _view(q, sq, td, dev, "q"), _view(q_out, sq, td, dev, "q_out")
    vk, vko = _view(k, sk, td, dev, "k"), _view(k_out, sk, td, dev, "k_out")
    nq = None if q is None else _norm_ref(q_norm, layers, hq, d, td, dev, "q_norm")
    nk = None if k is None else _norm_ref(k_norm, layers, hk, d, td, dev, "k_norm")
    _on_device(dev, _L.fcg_norm_rope_apply, (rope.h, _TORCH_DT[td], d, layers, n, pos.data_ptr(), hq, nq, _ref(vq),
                                             _ref(vqo), hk, nk, _ref(vk), _ref(vko), _stream_of(stream, dev)))


def fcg_norm_rope_workspace(n_layers: int, n_tok: int, n_q_heads: int, n_k_heads: int, head_dim: int) -> int:
    """Bytes that ``fcg_norm_rope_backward`` needs for weight gradients."""
    n = C.c_int64()
    _check(_L.fcg_norm_rope_workspace(int(head_dim), int(n_layers), int(n_tok), int(n_q_heads), int(n_k_heads), C.byref(n)))
    return n.value


def _norm_side(x, norm, grad, dx, dw, shape, td, dev, what: str):
    if grad is None:
        if x is not None or dx is not None or dw is not None:
            raise ValueError(f"{what}: without the gradient of its result")
        return None
    if dx is None or (x is None and norm is not None):
        raise ValueError(f"{what}: a gradient without the input or its own output")
    ref = _norm_ref(norm, shape[0], shape[2], shape[3], td, dev, what + "_norm")
    if dw is not None:
        if norm is None or norm.weight is None:
            raise ValueError(f"{what}: a gradient of weights that are not given")
        want = norm.dweight_shape(shape[0], shape[2])
        if (dw.dtype != torch.float32 or dw.get_device() != dev or not dw.is_contiguous() or
                dw.numel() != want[0] * want[1] * want[2]):
            raise ValueError(f"{what}: weight gradient, a contiguous float32 GPU tensor {want}")
    empty = TensorView(None, 0, 0, 0)
    return NormSide(shape[2], None if ref is None else C.pointer(norm._desc), _view(x, shape, td, dev, what) or empty,
                    _view(grad, shape, td, dev, what + "_grad"), _view(dx, shape, td, dev, "d" + what), _dptr(dw))


def fcg_norm_rope_backward(rope: Rope, pos, q=None, q_norm: Optional[Norm] = None, q_grad=None, dq=None, dq_weight=None,
                           k=None, k_norm: Optional[Norm] = None, k_grad=None, dk=None, dk_weight=None, workspace=None,
                           stream=None) -> None:
    """Gradient of ``fcg_norm_rope_apply``: from that of its results (q_grad, k_grad) to that of its inputs (dq, dk) and
    of the norms' weights (float32, of ``Norm.dweight_shape``)."""
    td, dev, layers, n, d, hq, hk = _rows_of(pos, q_grad, k_grad)
    sides = (_norm_side(q, q_norm, q_grad, dq, dq_weight, (layers, n, hq, d), td, dev, "q"),
             _norm_side(k, k_norm, k_grad, dk, dk_weight, (layers, n, hk, d), td, dev, "k"))
    need = 0
    if workspace is None and (dq_weight is not None or dk_weight is not None):
        need = fcg_norm_rope_workspace(layers, n, hq, hk, d)
    ws, nbytes, keep = _workspace(workspace, need, dev, stream)
    _on_device(dev, _L.fcg_norm_rope_backward, (rope.h, _TORCH_DT[td], d, layers, n, pos.data_ptr(), _ref(sides[0]),
                                                _ref(sides[1]), ws, nbytes, _stream_of(stream, dev)))


def fcg_append_norm(cache: Cache, layer: int, seq, pos, k, v, k_norm: Optional[Norm] = None, rope: Optional[Rope] = None,
                    q=None, q_norm: Optional[Norm] = None, q_out=None, flags: int = 0, stream=None) -> None:
    """``fcg_append`` of keys and queries that k_norm and q_norm normalise first."""
    s, p = _i32(seq), _i32(pos)
    if s.ndim != 1 or s.shape != p.shape:
        raise ValueError("seq and pos differ in length")
    if k is None or v is None:
        raise ValueError("k and v")
    if (q is None) != (q_out is None) or (q is None and q_norm is not None):
        raise ValueError("q, its norm and q_out belong together")
    layers = k.shape[0] if k.dim() == 4 else 1
    d, n = cache.desc, int(s.size)
    td, dev = _DT_TORCH[d.dtype], cache.device
    sq, skv = (layers, n, d.n_q_heads, d.head_dim), (layers, n, d.n_kv_heads, d.head_dim)
    vq, vqo = _view(q, sq, td, dev, "q"), _view(q_out, sq, td, dev, "q_out")
    vk, vv = _view(k, skv, td, dev, "k"), _view(v, skv, td, dev, "v")
    nq = _norm_ref(q_norm, layers, d.n_q_heads, d.head_dim, td, dev, "q_norm")
    nk = _norm_ref(k_norm, layers, d.n_kv_heads, d.head_dim, td, dev, "k_norm")
    _check(_L.fcg_append_norm(cache.h, int(layer), layers, n, _p(s), _p(p), None if rope is None else rope.h, nq, nk,
                              _ref(vq), _ref(vqo), _ref(vk), _ref(vv), int(flags), _stream_of(stream, dev)))


# ------------------------------------ what a cache keeps of its positions

def _plain(t, shape: tuple, dtype, device, what: str, strict: bool = True):
    """Address of a contiguous GPU tensor of a shape (None: not given, where strict is False)."""
    if t is None and not strict:
        return None
    if t is None or t.dtype is not dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor {shape} on GPU {device}")
    return t.data_ptr()


def fcg_attend_weights(cache: Cache, layer: int, prefix_seq: int, prefix_len: int, seq, pos, q, lse, weights,
                       flags: int = 0, stream=None) -> None:
    """Attention weight per cached position, summed over tokens and the heads of a kv head, of the tokens of a
    ``fcg_prefix_attend`` (its arguments and its lse).  weights float32 [n_seqs][Hkv][max_tokens] of the layer."""
    s, p = _i32(seq), _i32(pos)
    if s.ndim != 1 or s.shape != p.shape:
        raise ValueError("seq and pos differ in length")
    d, n, dev = cache.desc, int(s.size), cache.device
    vq = _view(q, (1, n, d.n_q_heads, d.head_dim), _DT_TORCH[d.dtype], dev, "q")
    a = _plain(lse, (n, d.n_q_heads), torch.float32, dev, "lse")
    w = _plain(weights, (cache.n_seqs, d.n_kv_heads, cache.max_tokens), torch.float32, dev, "weights")
    _check(_L.fcg_attend_weights(cache.h, int(layer), int(prefix_seq), int(prefix_len), n, _p(s), _p(p), _ref(vq), a, w,
                                 int(flags), _stream_of(stream, dev)))


def fcg_evict(cache: Cache, src, dst, keep, weights, first: int = 0, recent: int = 0, rope: Optional[Rope] = None,
              kept=None, stream=None) -> None:
    """Squeeze sequences ``src`` to ``keep`` positions each (the ``first``, the ``recent`` and those of most weight) as
    sequences ``dst``, which may be ``src``.  weights float32 [n_layers][n_seqs][Hkv][max_tokens], rewritten with the
    rows; kept int32 [n_layers][n_items][Hkv][max(keep)] or None receives the positions kept."""
    a, b, k = _i32(src), _i32(dst), _i32(keep)
    if a.ndim != 1 or a.shape != b.shape or a.shape != k.shape:
        raise ValueError("src, dst and keep differ in length")
    d, dev, n = cache.desc, cache.device, int(a.size)
    pw = pk = None
    if dev is not None:
        pw = _plain(weights, (d.n_layers, cache.n_seqs, d.n_kv_heads, cache.max_tokens), torch.float32, dev, "weights")
        pk = _plain(kept, (d.n_layers, n, d.n_kv_heads, int(k.max(initial=0))), torch.int32, dev, "kept", strict=False)
    _check(_L.fcg_evict(cache.h, n, _p(a), _p(b), _p(k), int(first), int(recent), None if rope is None else rope.h, pw, pk,
                        _stream_of(stream, dev)))


# -------------------------------------------------- log probabilities

def _logits(t, what: str):
    """(dtype code, rows, vocab, row stride) of a tensor of logits [n][vocab]."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what}: requires a gradient, which these calls do not record")
    if t.dim() != 2 or t.dtype not in _TORCH_DT or not t.is_cuda or (t.shape[1] > 1 and t.stride(1) != 1 and t.numel()):
        raise ValueError(f"{what}: a float32 or bfloat16 GPU tensor [rows][vocab], the logits of a row adjacent")
    return _TORCH_DT[t.dtype], t.shape[0], t.shape[1], t.stride(0)


def fcg_token_logprobs_workspace(n_rows: int, vocab: int, n_top: int = 0) -> int:
    """Bytes of workspace that ``fcg_token_logprobs`` needs (0 for many rows)."""
    n = C.c_int64()
    _check(_L.fcg_token_logprobs_workspace(int(n_rows), int(vocab), int(n_top), C.byref(n)))
    return n.value


def fcg_token_logprobs(logits, targets=None, logprob=None, entropy=None, lse=None, top_id=None, top_logprob=None,
                       workspace=None, stream=None) -> None:
    """Of each row of logits [n][vocab]: the log probability of its target (int32 [n]; outside the vocabulary: none), its
    entropy, its log-sum-exp (float32 [n]) and the most likely tokens (top_id int32, top_logprob float32 [n][k], k <= 64);
    None: not wanted.  Records no gradient: fcg_token_logprobs_backward is that of an autograd function."""
    dt, n, vocab, step = _logits(logits, "logits")
    dev, f32, k = logits.get_device(), torch.float32, 0 if top_id is None else top_id.shape[-1]
    if top_id is None and top_logprob is not None:
        raise ValueError("top_logprob without top_id")
    if logprob is not None and targets is None:
        raise ValueError("log probabilities without targets")
    outs = [_plain(t, (n,), d, dev, what, strict=False) for t, d, what in
            ((targets, torch.int32, "targets"), (logprob, f32, "logprob"), (entropy, f32, "entropy"), (lse, f32, "lse"))]
    tops = [_plain(top_id, (n, k), torch.int32, dev, "top_id", strict=False),
            _plain(top_logprob, (n, k), f32, dev, "top_logprob", strict=False)]
    ws, nbytes, keep = _workspace(workspace, 0 if workspace is not None else fcg_token_logprobs_workspace(n, vocab, k), dev,
                                  stream)
    _on_device(dev, _L.fcg_token_logprobs, (dt, n, vocab, logits.data_ptr(), step, *outs, k, *tops, ws, nbytes,
                                            _stream_of(stream, dev)))


def fcg_token_logprobs_backward(logits, targets, lse, entropy, dlogits, g_logprob=None, g_entropy=None, g_lse=None,
                                stream=None) -> None:
    """Gradient of the logits from those of logprob, entropy and lse (float32 [n], None: zero), with the lse and entropy of
    the forward pass.  dlogits may be the logits in place."""
    dt, n, vocab, step = _logits(logits, "logits")
    dev, f32 = logits.get_device(), torch.float32
    if (dlogits.shape != logits.shape or dlogits.dtype != logits.dtype or dlogits.get_device() != dev or
            (dlogits.shape[1] > 1 and dlogits.stride(1) != 1 and dlogits.numel())):
        raise ValueError("dlogits: a tensor as the logits")
    ins = [_plain(t, (n,), d, dev, what, strict=False) for t, d, what in
           ((targets, torch.int32, "targets"), (lse, f32, "lse"), (entropy, f32, "entropy"), (g_logprob, f32, "g_logprob"),
            (g_entropy, f32, "g_entropy"), (g_lse, f32, "g_lse"))]
    _on_device(dev, _L.fcg_token_logprobs_backward, (dt, n, vocab, logits.data_ptr(), step, *ins, dlogits.data_ptr(),
                                                     dlogits.stride(0), _stream_of(stream, dev)))


def fcg_locality_measure_ppl(loc: Locality, funcs, lengths, logprob, stream=None) -> None:
    """Set the perplexities of ``funcs`` from the log probabilities of their tokens (float32 GPU tensor, ``lengths[i]`` of
    function i after those before it).  Waits for the stream."""
    f, n = _i32(funcs), _i32(lengths)
    if f.ndim != 1 or f.shape != n.shape:
        raise ValueError("funcs and lengths differ in length")
    if logprob.dtype != torch.float32 or not logprob.is_cuda or not logprob.is_contiguous() or \
            logprob.numel() < int(n.sum(dtype=np.int64)):
        raise ValueError("logprob: a contiguous float32 GPU tensor of every function's tokens")
    dev = logprob.get_device()
    _on_device(dev, _L.fcg_locality_measure_ppl, (loc.h, int(f.size), _p(f), _p(n), logprob.data_ptr(),
                                                  _stream_of(stream, dev)))


def fcg_status_string(status: int) -> str:
    return _L.fcg_status_string(int(status)).decode()


def fcg_last_error() -> str:
    return _L.fcg_last_error().decode()

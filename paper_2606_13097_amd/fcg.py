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
]
FCG_ROPE_HALF, FCG_ROPE_PAIRS = 0, 1
FCG_ROPE_PLAIN, FCG_ROPE_LINEAR, FCG_ROPE_NTK, FCG_ROPE_PARTS, FCG_ROPE_GIVEN = range(5)
FCG_ROPE_BACKWARD = 1
FCG_REPLACE = 1
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


def fcg_status_string(status: int) -> str:
    return _L.fcg_status_string(int(status)).decode()


def fcg_last_error() -> str:
    return _L.fcg_last_error().decode()

"""Python binding of libsq: the GB300 hot path of SideQuest's KV-cache
management (paged GQA decode attention over copy-on-write prefix pages, and
span eviction by in-place compaction).

Argument marshalling only: every step runs in the CUDA library
(_build/libsq.so, built by `build.build_all()`).  There is no CPU fallback:
if the library is missing, importing the binding's functions raises.

Functions carry the C names of include/sq.h.  Device buffers may be given as
torch CUDA tensors or raw integer addresses; streams as torch.cuda.Stream,
raw cudaStream_t integers, or None (torch's current stream).
"""
from __future__ import annotations

import array
import ctypes
import os
import threading
from typing import Iterable, List, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libsq.so")

SQ_OK = 0
SQ_ERR_INVALID_ARG = -1
SQ_ERR_BAD_HANDLE = -2
SQ_ERR_NO_PAGES = -3
SQ_ERR_CAPACITY = -4
SQ_ERR_CUDA = -5
SQ_ERR_DEVICE = -6
SQ_ERR_DEVICE_TIMEOUT = -7
SQ_ERR_UNSUPPORTED = -8
SQ_ERR_NO_MEMORY = -9
SQ_OUT_BF16 = 0
SQ_OUT_F32 = 1
SQ_DEBUG_DROP_DECODE_STAGE = 1
SQ_MAX_DRAFT = 256


class sq_config(ctypes.Structure):
    _fields_ = [
        ("num_layers", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("max_seqs", ctypes.c_int32),
        ("max_pages_per_seq", ctypes.c_int32),
        ("kv_pool", ctypes.c_void_p),
        ("decode_ctas", ctypes.c_int32),
    ]


class sq_span(ctypes.Structure):
    _fields_ = [("start", ctypes.c_int32), ("end", ctypes.c_int32)]


class sq_norm_rope(ctypes.Structure):
    _fields_ = [
        ("q_weight", ctypes.c_void_p),
        ("k_weight", ctypes.c_void_p),
        ("rope", ctypes.c_void_p),
        ("weight_dtype", ctypes.c_int32),
        ("rot_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("max_pos", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class sq_stats_t(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in (
        "live_pages", "peak_live_pages", "decode_calls", "decode_logical_bytes",
        "decode_unique_bytes", "evict_calls", "evicted_tokens", "evict_moved_rows",
        "evict_bytes", "appended_tokens", "cow_pages", "prefill_calls", "prefill_pairs",
        "decode_early_calls", "decode_early_held", "decode_plans_built")]

    def as_dict(self):
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


class SqError(RuntimeError):
    def __init__(self, code: int, call: str):
        self.code = code
        super().__init__(f"{call} failed: {strerror(code)} ({code})")


_lib = None
_lock = threading.Lock()

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_I32P = ctypes.POINTER(ctypes.c_int32)
_F32 = ctypes.c_float
_SIGS = {
    "sq_pool_bytes": (ctypes.c_size_t, [ctypes.POINTER(sq_config)]),
    "sq_cache_create": (ctypes.c_int, [ctypes.POINTER(sq_config), ctypes.POINTER(_P)]),
    "sq_cache_destroy": (ctypes.c_int, [_P]),
    "sq_seq_new": (ctypes.c_int, [_P, _I32P]),
    "sq_append_kv": (ctypes.c_int, [_P, _I32, _I32, _P, _P, _P]),
    "sq_fork_aux": (ctypes.c_int, [_P, _I32, _I32P]),
    "sq_append_kv_batch": (ctypes.c_int, [_P, _I32P, _I32, _P, _P, _P]),
    "sq_decode_attention": (ctypes.c_int, [_P, _I32P, _I32, _I32, _P, _P, _I32, ctypes.c_float, _P]),
    "sq_evict_spans": (ctypes.c_int, [_P, _I32, _P, _I32, _P]),
    "sq_evict_spans_ragged": (ctypes.c_int, [_P, _I32, _P, _I32, _P]),
    "sq_prefill_attention": (ctypes.c_int, [_P, _I32, _I32, _I32, _P, _P, _I32, _P, ctypes.c_float,
                                            _P, _I32, _P]),
    "sq_release": (ctypes.c_int, [_P, _I32, _P]),
    "sq_seq_info": (ctypes.c_int, [_P, _I32, _I32P, _I32P]),
    "sq_seq_next_pos": (ctypes.c_int, [_P, _I32, ctypes.POINTER(ctypes.c_int64)]),
    "sq_get_page_table": (ctypes.c_int, [_P, _I32, _I32P, _I32, _I32P]),
    "sq_get_page_fill": (ctypes.c_int, [_P, _I32, _I32P, _I32, _I32P]),
    "sq_page_refcount": (ctypes.c_int, [_P, _I32, _I32P]),
    "sq_free_pages": (ctypes.c_int, [_P, _I32P]),
    "sq_pool_ptr": (ctypes.c_int, [_P, ctypes.POINTER(_P)]),
    "sq_stats": (ctypes.c_int, [_P, ctypes.POINTER(sq_stats_t)]),
    "sq_sync_status": (ctypes.c_int, [_P, _P]),
    "sq_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "sq_probe_read": (ctypes.c_int, [_P, _P, ctypes.c_size_t, _P]),
    "sq_debug_set": (ctypes.c_int, [_P, _I32]),
    "sq_decode_attention_noalloc": (ctypes.c_int, [_P, _I32P, _I32, _I32, _P, _P, _I32,
                                                   ctypes.c_float, _P]),
    "sq_extend": (ctypes.c_int, [_P, _P, _I32, _P, _P]),
    "sq_qk_norm_rope_store": (ctypes.c_int, [_P, _P, _I32, _P, _I32, _P, _I64, _P, _I64, _P, _I64,
                                             _P, _P, _P, _P]),
    "sq_qk_norm_rope": (ctypes.c_int, [_P, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _P]),
    "sq_qk_norm_rope_backward": (ctypes.c_int, [_P, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _P,
                                                _I64, _P, _I64, _P, _P, _P]),
    "sq_window_attention": (ctypes.c_int, [_P, _P, _I32, _P, _I32, _P, _P, _I32, _P, _F32, _I32,
                                           _I32, _P]),
    "sq_tree_attention": (ctypes.c_int, [_P, _P, _I32, _P, _P, _I32, _P, _P, _I32, _P, _F32, _I32,
                                         _I32, _P]),
    "sq_accept_draft": (ctypes.c_int, [_P, _I32, _I32, _P, _I32, _P]),
}


def lib() -> ctypes.CDLL:
    """The loaded libsq.so.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(
                    f"libsq.so not found at {LIB_PATH}: build it with "
                    "`python -m paper_2602_22603_gb300.build` (needs nvcc)")
            L = ctypes.CDLL(LIB_PATH)
            for name, (res, args) in _SIGS.items():
                f = getattr(L, name)
                f.restype = res
                f.argtypes = args
            _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().sq_strerror(int(code)).decode()


sq_strerror = strerror


def _check(rc: int, call: str) -> None:
    if rc != SQ_OK:
        raise SqError(rc, call)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


# torch's current stream as a raw handle.  torch.cuda.current_stream() builds a
# Stream object (2.9 us of a 17 us decode call); the same handle comes from the
# functions below it, where this torch has them.
_raw_stream = None


def _current_stream() -> int:
    global _raw_stream
    if _raw_stream is None:
        import torch
        first = int(torch.cuda.current_stream().cuda_stream)  # (initialises CUDA)
        get, device = (getattr(torch._C, n, None)
                       for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if get is None or device is None:
            _raw_stream = lambda: int(torch.cuda.current_stream().cuda_stream)  # noqa: E731
        else:
            _raw_stream = lambda: get(device())  # noqa: E731
        return first
    return _raw_stream()


def _stream(s) -> Optional[int]:
    if s is None:
        return _current_stream()
    if isinstance(s, int):
        return s
    return int(s.cuda_stream)


def _spans(spans):
    """(address, what keeps it alive) of the spans as sq_span[]: two int32 each.

    An array of integers: a third of the time of one sq_span object for each
    span (96 spans: 4.5 us against 13 us)."""
    if not len(spans):
        return None, None
    values = [int(x) for a, b in spans for x in (a, b)]
    try:
        buf = array.array("i", values)
    except OverflowError:  # wrapped, as ctypes stores them
        buf = array.array("i", [ctypes.c_int32(v).value for v in values])
    return buf.buffer_info()[0], buf


def _ints(x):
    """(address, what keeps it alive) of host int32 values: a sequence of them, an
    array.array("i") or a ctypes int32 array; None stays None."""
    if x is None:
        return None, None
    if x.__class__ is not list and x.__class__ is not tuple:
        if isinstance(x, ctypes.Array):
            return ctypes.addressof(x), x
        if isinstance(x, array.array) and x.typecode == "i":
            return x.buffer_info()[0], x
    x = array.array("i", x)
    return x.buffer_info()[0], x


# torch's types, once a call has tensors to check (their names cost a
# microsecond a tensor to compare)
_BF16 = _FLOAT = _INT = None


def _types():
    global _BF16, _FLOAT, _INT
    import torch
    _BF16, _FLOAT, _INT = torch.bfloat16, torch.float32, torch.int32


def _wrong(name, want, x):
    raise ValueError(f"{name}: {want} on a cuda device expected, not {x.dtype} {list(x.shape)} of strides "
                     f"{x.stride()} on {x.device}")


def _rows(x, heads, dim, name, n=None):
    """(address, elements between tokens, tokens) of a bfloat16 [tokens, heads,
    dim] tensor whose rows are contiguous; an address alone stands for a
    contiguous one of n tokens."""
    if x.__class__ is int:
        return x, heads * dim, n
    if x.dim() == 3:
        (tokens, h, d), (apart, s1, s2) = x.shape, x.stride()
        if (h == heads and d == dim and s2 == 1 and s1 == dim and x.dtype is _BF16 and x.is_cuda
                and (n is None or tokens == n)):
            # (one token has no distance to the next)
            return x.data_ptr(), apart if tokens > 1 else heads * dim, tokens
    _wrong(name, f"bfloat16 [{'tokens' if n is None else n}, {heads}, {dim}] of contiguous rows", x)


def _flat(x, want, count, name):
    """Address of a contiguous tensor of `count` elements of a type on a device (None
    and addresses as they are)."""
    if x is None or x.__class__ is int:
        return x
    if x.dtype is want and x.numel() == count and x.is_contiguous() and x.is_cuda:
        return x.data_ptr()
    _wrong(name, f"{count} contiguous elements of {want}", x)


def norm_rope(rope=None, rot_dim=0, eps=1e-6, q_weight=None, k_weight=None,
              interleaved=False) -> sq_norm_rope:
    """The parameters of the norms and the rotation: `rope` a float32 CUDA tensor
    [max_pos, rot_dim / 2, 2] of cosines and sines (rope_table makes one),
    weights bfloat16 or float32 CUDA tensors [head_dim] of one type, or None (ones)."""
    _types()
    weights = [w for w in (q_weight, k_weight) if w is not None]
    for w in weights:
        if (w.dtype not in (_BF16, _FLOAT) or w.dtype is not weights[0].dtype or not w.is_contiguous()
                or not w.is_cuda or w.numel() != weights[0].numel()):
            _wrong("weights", "contiguous, of one size, both bfloat16 or both float32", w)
    f32 = bool(weights) and weights[0].dtype is _FLOAT
    max_pos = 0
    if rope is not None and rot_dim:
        max_pos = rope.shape[0]
        _flat(rope, _FLOAT, max_pos * rot_dim, "rope")
    p = sq_norm_rope(_ptr(q_weight), _ptr(k_weight), _ptr(rope) if max_pos else None,
                     SQ_OUT_F32 if f32 else SQ_OUT_BF16, rot_dim, int(interleaved),
                     max_pos, eps)
    p._keep = (rope, q_weight, k_weight)
    p._dim = weights[0].numel() if weights else None
    return p


def _weights_fit(params, dim):
    """Refuses parameters whose weights are not one head's (those of a structure filled
    by hand are not known)."""
    n = getattr(params, "_dim", None)
    if n is not None and n != dim:
        raise ValueError(f"weights: {dim} elements expected, not {n}")


def rope_table(max_pos, rot_dim, theta=10000.0, device="cuda"):
    """Cosines and sines of position x theta^(-2 i / rot_dim), float32 [max_pos,
    rot_dim / 2, 2] (angles in 64 bits)."""
    import torch
    inv = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    angle = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


# ---- the C calls ------------------------------------------------------------
def make_config(num_layers, num_q_heads, num_kv_heads, head_dim, page_size, num_pages,
                max_seqs=64, max_pages_per_seq=None, kv_pool=None, decode_ctas=0) -> sq_config:
    return sq_config(num_layers, num_q_heads, num_kv_heads, head_dim, page_size, num_pages,
                     max_seqs, max_pages_per_seq or num_pages, _ptr(kv_pool), decode_ctas)


def sq_pool_bytes(cfg: sq_config) -> int:
    return int(lib().sq_pool_bytes(ctypes.byref(cfg)))


def sq_cache_create(cfg: sq_config) -> int:
    out = _P()
    _check(lib().sq_cache_create(ctypes.byref(cfg), ctypes.byref(out)), "sq_cache_create")
    return out.value


def sq_cache_destroy(cache: int) -> None:
    _check(lib().sq_cache_destroy(cache), "sq_cache_destroy")


def sq_seq_new(cache: int) -> int:
    h = _I32()
    _check(lib().sq_seq_new(cache, ctypes.byref(h)), "sq_seq_new")
    return h.value


def sq_append_kv(cache: int, seq: int, n_tokens: int, k, v, stream=None) -> None:
    _check(lib().sq_append_kv(cache, seq, n_tokens, _ptr(k), _ptr(v), _stream(stream)),
           "sq_append_kv")


def sq_append_kv_batch(cache: int, seqs, k, v, stream=None) -> None:
    arr = seqs if isinstance(seqs, ctypes.Array) else (ctypes.c_int32 * len(seqs))(*seqs)
    _check(lib().sq_append_kv_batch(cache, arr, len(seqs), _ptr(k), _ptr(v), _stream(stream)),
           "sq_append_kv_batch")


def sq_fork_aux(cache: int, parent: int) -> int:
    h = _I32()
    _check(lib().sq_fork_aux(cache, parent, ctypes.byref(h)), "sq_fork_aux")
    return h.value


def sq_decode_attention(cache: int, seqs: Sequence[int], layer: int, q, out,
                        out_dtype: int = SQ_OUT_BF16, sm_scale: float = 1.0,
                        stream=None) -> None:
    arr = seqs if isinstance(seqs, ctypes.Array) else (ctypes.c_int32 * len(seqs))(*seqs)
    _check(lib().sq_decode_attention(cache, arr, len(seqs), layer, _ptr(q), _ptr(out),
                                     out_dtype, float(sm_scale), _stream(stream)),
           "sq_decode_attention")


def sq_decode_attention_noalloc(cache: int, seqs: Sequence[int], layer: int, q, out,
                                out_dtype: int = SQ_OUT_BF16, sm_scale: float = 1.0,
                                stream=None) -> None:
    """sq_decode_attention without any device allocation (fixed library
    scratch; see include/sq.h for the limits and the sharing rule)."""
    arr = (ctypes.c_int32 * len(seqs))(*seqs)
    _check(lib().sq_decode_attention_noalloc(cache, arr, len(seqs), layer, _ptr(q), _ptr(out),
                                             out_dtype, float(sm_scale), _stream(stream)),
           "sq_decode_attention_noalloc")


def sq_evict_spans(cache: int, seq: int, spans: Sequence[Tuple[int, int]], stream=None) -> None:
    arr, _keep = _spans(spans)
    _check(lib().sq_evict_spans(cache, seq, arr, len(spans), _stream(stream)), "sq_evict_spans")


def sq_evict_spans_ragged(cache: int, seq: int, spans: Sequence[Tuple[int, int]],
                          stream=None) -> None:
    arr, _keep = _spans(spans)
    _check(lib().sq_evict_spans_ragged(cache, seq, arr, len(spans), _stream(stream)),
           "sq_evict_spans_ragged")


def sq_prefill_attention(cache: int, seq: int, layer: int, n_q: int, q, out,
                         out_dtype: int = SQ_OUT_BF16, lse=None, sm_scale: float = 1.0,
                         spans: Sequence[Tuple[int, int]] = (), stream=None) -> None:
    arr, _keep = _spans(spans)
    _check(lib().sq_prefill_attention(cache, seq, layer, n_q, _ptr(q), _ptr(out), out_dtype,
                                      _ptr(lse), float(sm_scale), arr, len(spans),
                                      _stream(stream)),
           "sq_prefill_attention")


def sq_extend(cache: int, seqs, n_new=None, stream=None) -> None:
    """Lengthen sequences by n_new[i] rows (None: one each) stored later."""
    arr, _keep = _ints(seqs)
    cnt, _keep2 = _ints(n_new)
    _check(lib().sq_extend(cache, arr, len(seqs), cnt, _stream(stream)), "sq_extend")


def sq_qk_norm_rope_store(cache: int, seqs, n_new, layer: int, q, q_stride, k, k_stride, v, v_stride,
                          positions, params: sq_norm_rope, q_out, stream=None) -> None:
    arr, _keep = _ints(seqs)
    cnt, _keep2 = _ints(n_new)
    _check(lib().sq_qk_norm_rope_store(cache, arr, len(seqs), cnt, layer, _ptr(q), q_stride, _ptr(k),
                                       k_stride, _ptr(v), v_stride, _ptr(positions),
                                       ctypes.addressof(params), _ptr(q_out), _stream(stream)),
           "sq_qk_norm_rope_store")


def sq_qk_norm_rope(cache: int, n_tokens: int, q, q_stride, k, k_stride, positions,
                    params: sq_norm_rope, q_out, k_out, stream=None) -> None:
    _check(lib().sq_qk_norm_rope(cache, n_tokens, _ptr(q), q_stride, _ptr(k), k_stride,
                                 _ptr(positions), ctypes.addressof(params), _ptr(q_out), _ptr(k_out),
                                 _stream(stream)), "sq_qk_norm_rope")


def sq_qk_norm_rope_backward(cache: int, n_tokens: int, q, q_stride, k, k_stride, positions,
                             params: sq_norm_rope, dq_out, dk_out, dq, dq_stride, dk, dk_stride,
                             dq_weight=None, dk_weight=None, stream=None) -> None:
    _check(lib().sq_qk_norm_rope_backward(cache, n_tokens, _ptr(q), q_stride, _ptr(k), k_stride,
                                          _ptr(positions), ctypes.addressof(params), _ptr(dq_out),
                                          _ptr(dk_out), _ptr(dq), dq_stride, _ptr(dk), dk_stride,
                                          _ptr(dq_weight), _ptr(dk_weight), _stream(stream)),
           "sq_qk_norm_rope_backward")


def sq_window_attention(cache: int, seqs, n_q, layer: int, q, out, window: int, n_sink: int = 0,
                        out_dtype: int = SQ_OUT_BF16, lse=None, sm_scale: float = 1.0,
                        stream=None) -> None:
    arr, _keep = _ints(seqs)
    cnt, _keep2 = _ints(n_q)
    _check(lib().sq_window_attention(cache, arr, len(seqs), cnt, layer, _ptr(q), _ptr(out), out_dtype,
                                     _ptr(lse), float(sm_scale), window, n_sink, _stream(stream)),
           "sq_window_attention")


def sq_tree_attention(cache: int, seqs, n_draft, parents, layer: int, q, out, window: int = 0,
                      n_sink: int = 0, out_dtype: int = SQ_OUT_BF16, lse=None, sm_scale: float = 1.0,
                      stream=None) -> None:
    arr, _keep = _ints(seqs)
    cnt, _keep2 = _ints(n_draft)
    par, _keep3 = _ints(parents)
    _check(lib().sq_tree_attention(cache, arr, len(seqs), cnt, par, layer, _ptr(q), _ptr(out),
                                   out_dtype, _ptr(lse), float(sm_scale), window, n_sink,
                                   _stream(stream)),
           "sq_tree_attention")


def sq_accept_draft(cache: int, seq: int, n_draft: int, path, stream=None) -> None:
    arr, _keep = _ints(path)
    _check(lib().sq_accept_draft(cache, seq, n_draft, arr, len(path), _stream(stream)),
           "sq_accept_draft")


def sq_release(cache: int, seq: int, stream=None) -> None:
    _check(lib().sq_release(cache, seq, _stream(stream)), "sq_release")


def sq_seq_info(cache: int, seq: int) -> Tuple[int, int]:
    n, p = _I32(), _I32()
    _check(lib().sq_seq_info(cache, seq, ctypes.byref(n), ctypes.byref(p)), "sq_seq_info")
    return n.value, p.value


def sq_seq_next_pos(cache: int, seq: int) -> int:
    """Position of the sequence's next token (tokens ever appended; eviction
    does not lower it)."""
    x = ctypes.c_int64()
    _check(lib().sq_seq_next_pos(cache, seq, ctypes.byref(x)), "sq_seq_next_pos")
    return x.value


def sq_get_page_table(cache: int, seq: int) -> List[int]:
    _, npages = sq_seq_info(cache, seq)
    buf = (ctypes.c_int32 * max(1, npages))()
    n = _I32()
    _check(lib().sq_get_page_table(cache, seq, buf, npages, ctypes.byref(n)), "sq_get_page_table")
    return list(buf[: n.value])


def sq_get_page_fill(cache: int, seq: int) -> List[int]:
    _, npages = sq_seq_info(cache, seq)
    buf = (ctypes.c_int32 * max(1, npages))()
    n = _I32()
    _check(lib().sq_get_page_fill(cache, seq, buf, npages, ctypes.byref(n)), "sq_get_page_fill")
    return list(buf[: n.value])


def sq_page_refcount(cache: int, page: int) -> int:
    out = _I32()
    _check(lib().sq_page_refcount(cache, page, ctypes.byref(out)), "sq_page_refcount")
    return out.value


def sq_free_pages(cache: int) -> int:
    out = _I32()
    _check(lib().sq_free_pages(cache, ctypes.byref(out)), "sq_free_pages")
    return out.value


def sq_pool_ptr(cache: int) -> int:
    out = _P()
    _check(lib().sq_pool_ptr(cache, ctypes.byref(out)), "sq_pool_ptr")
    return out.value


def sq_stats(cache: int) -> dict:
    st = sq_stats_t()
    _check(lib().sq_stats(cache, ctypes.byref(st)), "sq_stats")
    return st.as_dict()


def sq_probe_read(cache: int, buf, nbytes: int, stream=None) -> None:
    _check(lib().sq_probe_read(cache, _ptr(buf), nbytes, _stream(stream)), "sq_probe_read")


def sq_debug_set(cache: int, flags: int) -> None:
    _check(lib().sq_debug_set(cache, flags), "sq_debug_set")


def sq_sync_status(cache: int, stream=None) -> int:
    """Synchronise the stream and return the device status code (no raise)."""
    return int(lib().sq_sync_status(cache, _stream(stream)))


# ---- a small object wrapper --------------------------------------------------
class Cache:
    """Owns one sq_cache.  Methods are the C calls with the cache bound."""

    def __init__(self, num_layers, num_q_heads, num_kv_heads, head_dim, page_size, num_pages,
                 max_seqs=64, max_pages_per_seq=None, kv_pool=None, decode_ctas=0):
        self.cfg = make_config(num_layers, num_q_heads, num_kv_heads, head_dim, page_size,
                               num_pages, max_seqs, max_pages_per_seq, kv_pool, decode_ctas)
        self._keep = kv_pool
        self.handle = sq_cache_create(self.cfg)
        self.L, self.Hq, self.Hkv = num_layers, num_q_heads, num_kv_heads
        self.D, self.P, self.num_pages = head_dim, page_size, num_pages

    def close(self):
        if self.handle:
            sq_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def pool_view(self):
        """The pool as a torch bf16 tensor [L, num_pages, 2, Hkv, P, D]
        (a zero-copy view of library memory)."""
        import torch

        class _Arr:
            pass

        a = _Arr()
        shape = (self.L, self.num_pages, 2, self.Hkv, self.P, self.D)
        a.__cuda_array_interface__ = {
            "shape": shape, "typestr": "<i2", "data": (sq_pool_ptr(self.handle), False),
            "version": 3, "strides": None}
        return torch.as_tensor(a, device="cuda").view(torch.bfloat16)

    seq_new = lambda self: sq_seq_new(self.handle)
    append_kv = lambda self, seq, n, k, v, stream=None: sq_append_kv(self.handle, seq, n, k, v, stream)
    fork_aux = lambda self, parent: sq_fork_aux(self.handle, parent)
    append_kv_batch = lambda self, seqs, k, v, stream=None: sq_append_kv_batch(self.handle, seqs, k, v, stream)
    decode_attention = (lambda self, seqs, layer, q, out, out_dtype=SQ_OUT_BF16, sm_scale=1.0,
                        stream=None: sq_decode_attention(self.handle, seqs, layer, q, out,
                                                         out_dtype, sm_scale, stream))
    evict_spans = lambda self, seq, spans, stream=None: sq_evict_spans(self.handle, seq, spans, stream)
    evict_spans_ragged = (lambda self, seq, spans, stream=None:
                          sq_evict_spans_ragged(self.handle, seq, spans, stream))
    prefill_attention = (lambda self, seq, layer, n_q, q, out, out_dtype=SQ_OUT_BF16, lse=None,
                         sm_scale=1.0, spans=(), stream=None:
                         sq_prefill_attention(self.handle, seq, layer, n_q, q, out, out_dtype, lse,
                                              sm_scale, spans, stream))
    extend = lambda self, seqs, n_new=None, stream=None: sq_extend(self.handle, seqs, n_new, stream)

    def _counted(self, seqs, counts, n, what):
        """The call's rows, which the tensors' tokens (n) have to be."""
        if counts is None:
            total = len(seqs)
        else:
            total = sum(counts)
            if len(counts) != len(seqs):
                raise ValueError(f"{what}: {len(counts)} counts for {len(seqs)} sequences")
        if n is not None and n != total:
            raise ValueError(f"{what}: {n} tokens given, {total} counted")
        return total

    def qk_norm_rope_store(self, seqs, n_new, layer, q, k, v, positions, params, q_out, stream=None):
        """q [tokens, Hq, D], k and v [tokens, Hkv, D] (parts of a fused projection
        do) of the sequences' newest rows: queries normed and rotated into q_out,
        keys into the cache with the values."""
        if _BF16 is None:
            _types()
        hq, hkv, d = self.Hq, self.Hkv, self.D
        _weights_fit(params, d)
        q, qs, n = _rows(q, hq, d, "q")
        n = self._counted(seqs, n_new, n, "qk_norm_rope_store")
        k, ks, _ = _rows(k, hkv, d, "k", n)
        v, vs, _ = _rows(v, hkv, d, "v", n)
        sq_qk_norm_rope_store(self.handle, seqs, n_new, layer, q, qs, k, ks, v, vs,
                              _flat(positions, _INT, n, "positions"), params,
                              _flat(q_out, _BF16, n * hq * d, "q_out"), stream)

    def qk_norm_rope(self, q, k, positions, params, q_out, k_out, stream=None):
        """Norms and rotation of q [tokens, Hq, D] and k [tokens, Hkv, D] into tensors."""
        if _BF16 is None:
            _types()
        hq, hkv, d = self.Hq, self.Hkv, self.D
        _weights_fit(params, d)
        q, qs, n = _rows(q, hq, d, "q")
        k, ks, _ = _rows(k, hkv, d, "k", n)
        sq_qk_norm_rope(self.handle, n, q, qs, k, ks, _flat(positions, _INT, n, "positions"), params,
                        _flat(q_out, _BF16, n * hq * d, "q_out"),
                        _flat(k_out, _BF16, n * hkv * d, "k_out"), stream)

    def qk_norm_rope_backward(self, q, k, positions, params, dq_out, dk_out, dq, dk, dq_weight=None,
                              dk_weight=None, stream=None):
        """Gradients of qk_norm_rope: dq and dk (rows apart as they are) and, where
        wanted, the weights' (float32)."""
        if _BF16 is None:
            _types()
        hq, hkv, d = self.Hq, self.Hkv, self.D
        _weights_fit(params, d)
        q, qs, n = _rows(q, hq, d, "q")
        k, ks, _ = _rows(k, hkv, d, "k", n)
        dq, dqs, _ = _rows(dq, hq, d, "dq", n)
        dk, dks, _ = _rows(dk, hkv, d, "dk", n)
        sq_qk_norm_rope_backward(self.handle, n, q, qs, k, ks, _flat(positions, _INT, n, "positions"),
                                 params, _flat(dq_out, _BF16, n * hq * d, "dq_out"),
                                 _flat(dk_out, _BF16, n * hkv * d, "dk_out"), dq, dqs, dk, dks,
                                 _flat(dq_weight, _FLOAT, d, "dq_weight"),
                                 _flat(dk_weight, _FLOAT, d, "dk_weight"), stream)

    def _attention(self, seqs, counts, q, out, out_dtype, lse, what):
        """Addresses of the tensors of a call on query blocks, and its queries."""
        if _BF16 is None:
            _types()
        n = self._counted(seqs, counts, None, what)
        rows = n * self.Hq
        size = rows * self.D
        return (_flat(q, _BF16, size, "q"),
                _flat(out, _FLOAT if out_dtype == SQ_OUT_F32 else _BF16, size, "out"),
                lse if lse is None else _flat(lse, _FLOAT, rows, "lse"), n)

    def window_attention(self, seqs, n_q, layer, q, out, window, n_sink=0, out_dtype=SQ_OUT_BF16,
                         lse=None, sm_scale=1.0, stream=None):
        """Attention of the newest n_q[i] tokens (None: one) of each sequence, each
        seeing its last `window` tokens and the first n_sink."""
        q, out, lse, _ = self._attention(seqs, n_q, q, out, out_dtype, lse, "window_attention")
        sq_window_attention(self.handle, seqs, n_q, layer, q, out, window, n_sink, out_dtype, lse,
                            sm_scale, stream)

    def tree_attention(self, seqs, n_draft, parents, layer, q, out, window=0, n_sink=0,
                       out_dtype=SQ_OUT_BF16, lse=None, sm_scale=1.0, stream=None):
        """Attention of trees of drafted tokens, each sequence's newest n_draft[i]
        rows; parents: every drafted token's parent in its tree, -1 the context."""
        q, out, lse, n = self._attention(seqs, n_draft, q, out, out_dtype, lse, "tree_attention")
        if len(parents) != n:
            raise ValueError(f"tree_attention: {len(parents)} parents of {n} drafted tokens")
        sq_tree_attention(self.handle, seqs, n_draft, parents, layer, q, out, window, n_sink, out_dtype,
                          lse, sm_scale, stream)

    accept_draft = (lambda self, seq, n_draft, path, stream=None:
                    sq_accept_draft(self.handle, seq, n_draft, path, stream))
    release = lambda self, seq, stream=None: sq_release(self.handle, seq, stream)
    seq_info = lambda self, seq: sq_seq_info(self.handle, seq)
    next_pos = lambda self, seq: sq_seq_next_pos(self.handle, seq)
    page_table = lambda self, seq: sq_get_page_table(self.handle, seq)
    page_fills = lambda self, seq: sq_get_page_fill(self.handle, seq)
    page_refcount = lambda self, page: sq_page_refcount(self.handle, page)
    free_pages = lambda self: sq_free_pages(self.handle)
    stats = lambda self: sq_stats(self.handle)
    sync_status = lambda self, stream=None: sq_sync_status(self.handle, stream)

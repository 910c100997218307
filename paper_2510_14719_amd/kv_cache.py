"""The operators around a paged cache of keys and values (the C ABI of ``include/kv_cache.h``): rotary positions, new tokens into the
cache, attention of new tokens over it, the upkeep of its pages.

Argument marshalling only, like :mod:`.binding`: every step runs in the HIP kernels behind the C ABI, tensors are accepted for their
device memory, shape and strides, and there is no fallback.  All calls are asynchronous on ``stream`` (default: torch's current
stream) and allocate nothing.

A cache is a pair of tensors with the logical shape [pages][key heads][page size][d] (whatever the order in memory: a view with
other strides will do), for the page functions [layers][pages][key heads][page size][d]; float16, bfloat16 or E4M3 (float8_e4m3fn, or
uint8 for the raw bytes).  Tokens are [tokens][heads][d], a batch of sequences is described by ``q_start`` [S + 1], ``kv_len`` [S] and
``table`` [S][entries], all int32 on the device: see the header.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding

FP16, BF16, E4M3 = 0, 1, 2
HALF, INTERLEAVED = 0, 1
PLAIN, LINEAR, BASE, PARTS = 0, 1, 2, 3
MAX_LIST = 8192

_TYPES = {torch.float16: FP16, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3, torch.uint8: E4M3}
_vp, _ci, _cl, _cf, _cd = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_double


class _Pages(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("layer_stride", _cl), ("page_stride", _cl), ("head_stride", _cl),
                ("token_stride", _cl), ("layers", _ci), ("pages", _ci), ("heads", _ci), ("page_size", _ci), ("d", _ci), ("dtype", _ci)]


class _Batch(ctypes.Structure):
    _fields_ = [("q_start", _vp), ("kv_len", _vp), ("table", _vp), ("sequences", _ci), ("tokens", _ci), ("table_width", _ci), ("table_stride", _ci),
                ("max_q", _ci), ("max_kv", _ci)]


class _Rows(ctypes.Structure):
    _fields_ = [("p", _vp), ("token_stride", _cl), ("head_stride", _cl)]


class _Tensor(ctypes.Structure):
    _fields_ = [("p", _vp), ("batch_stride", _cl), ("head_stride", _cl), ("token_stride", _cl)]


class _Book(ctypes.Structure):
    _fields_ = [("ref", _vp), ("table", _vp), ("kv_len", _vp), ("pages", _ci), ("rows", _ci), ("table_width", _ci), ("table_stride", _ci),
                ("page_size", _ci)]


class KvCacheError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("kv_cache call failed with code %d: %s" % (code, text))
        self.code = code


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        p = ctypes.POINTER
        lib.kv_strerror.restype = ctypes.c_char_p
        lib.kv_strerror.argtypes = [_ci]
        attn = [p(_Pages), p(_Batch), p(_Rows), p(_Rows), _vp, _ci, _cf]
        append = [p(_Pages), p(_Batch)] + [p(_Rows)] * 4 + [_ci, _vp, _ci, _ci, _cf]
        turn = [p(_Tensor), p(_Tensor), _ci, _ci, _ci, _ci, _vp, _cl, _vp, _ci, _ci, _cf]
        for name, args in (("attn_paged", attn + [_ci, _ci, _vp, _cl, _vp]), ("attn_paged_check_args", attn + [_ci, _vp, _cl]),
                           ("kv_append", append + [_ci, _vp]), ("kv_append_check_args", append + [_ci]),
                           ("rope", turn + [_ci, _ci, _vp]), ("rope_check_args", turn + [_ci]),
                           ("rope_frequencies", [p(_cd), _ci, _cd, _ci, _cd, _cd, _cd, _cd]),
                           ("kv_reserve", [p(_Book), _vp, _vp, _ci, _vp, _vp]), ("kv_free", [p(_Book), _vp, _ci, _vp]),
                           ("kv_fork", [p(_Pages), p(_Book), _vp, _vp, _ci, _vp, _vp]), ("kv_compact", [p(_Pages), p(_Book), _vp, _cl, _vp]),
                           ("kv_copy_pages", [p(_Pages), _vp, _vp, _ci, _vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = _ci, args
        lib.attn_paged_workspace.restype, lib.attn_paged_workspace.argtypes = _cl, [p(_Pages), p(_Batch), _ci]
        lib.kv_compact_workspace.restype, lib.kv_compact_workspace.argtypes = _cl, [_ci]
        _lib = lib
    return _lib


def _check(rc: int) -> None:
    if rc != 0:
        raise KvCacheError(rc, _load().kv_strerror(rc).decode())


def _device(x, what):
    if not x.is_cuda:
        raise ValueError("%s: device tensors are taken; got one on %s" % (what, x.device))
    if x.device.index != torch.cuda.current_device():
        raise ValueError("%s: on %s, and the call goes to the current device, %d" % (what, x.device, torch.cuda.current_device()))
    return x.data_ptr()


def _fast():
    """The extension that makes plain calls without the interpreter's share; what it does not take (NotImplemented) goes through the code here."""
    return binding._fast or binding._load_fast()


def _int(x):
    """A number for an int of the C ABI, which ctypes would cut to its lower 32 bits."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise KvCacheError(-5, _load().kv_strerror(-5).decode())
    return x


def _array(x, dtype, what, shape=None):
    """Address of a contiguous tensor of a type (and shape); None passes."""
    if x is None:
        return None
    if x.dtype != dtype or not x.is_contiguous() or (shape is not None and tuple(x.shape) != shape):
        raise ValueError("%s: a contiguous %s tensor%s is wanted; got %s %s" % (what, dtype, "" if shape is None else " of shape %s" % (shape,), x.dtype, tuple(x.shape)))
    return _device(x, what)


def _unit(x, what):
    """The last dimension lies without gaps."""
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError("%s: the elements of a head must be contiguous; strides %s" % (what, tuple(x.stride())))


def _type(x, what):
    if x.dtype not in _TYPES:
        raise ValueError("%s: type %s is not supported" % (what, x.dtype))
    return _TYPES[x.dtype]


def _pages(k, v, k_scale=None, v_scale=None, layers=False):
    if k.dim() != 4 + layers or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride():
        raise ValueError("k and v caches: two tensors of one type, shape and strides, %s[pages][heads][page size][d]; got %s and %s" % (
            "[layers]" if layers else "", tuple(k.shape), tuple(v.shape)))
    _unit(k, "cache")
    n, h, t, d = map(_int, k.shape[-4:])
    s = k.stride()
    return _Pages(_device(k, "k cache"), _device(v, "v cache"), _array(k_scale, torch.float32, "k_scale", (h,)), _array(v_scale, torch.float32, "v_scale", (h,)),
                  s[0] if layers else 0, s[-4], s[-3], s[-2], _int(k.shape[0]) if layers else 1, n, h, t, d, _type(k, "cache"))


def _batch(q_start, kv_len, table, tokens, max_q, max_kv):
    n, tokens, max_q, max_kv = map(_int, (kv_len.shape[0], tokens, max_q, max_kv))
    if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != n or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table: int32 [sequences][entries], entries contiguous; got %s %s" % (table.dtype, tuple(table.shape)))
    return _Batch(_array(q_start, torch.int32, "q_start", (n + 1,)), _array(kv_len, torch.int32, "kv_len", (n,)), _device(table, "table"), n, tokens, _int(table.shape[1]),
                  _int(table.stride(0)) if n > 1 else 0, max_q, max_kv)


def _rows(x, what, shape=None, dtype=None):
    if x.dim() != 3 or (shape is not None and tuple(x.shape) != shape) or (dtype is not None and x.dtype != dtype):
        raise ValueError("%s: [tokens][heads][d]%s wanted; got %s %s" % (what, "" if shape is None else " = %s %s" % (dtype, shape), x.dtype, tuple(x.shape)))
    _unit(x, what)
    return _Rows(_device(x, what), x.stride(0), x.stride(1))


def _stream(stream):
    return binding._stream_handle(stream)


def attn_paged_workspace(q, k_cache, sequences, max_q, max_kv) -> int:
    """Bytes of workspace of a call of ``attn_paged`` with these tokens, this cache (k or v) and these bounds."""
    cache = _Pages(heads=_int(k_cache.shape[1]), d=_int(k_cache.shape[3]), dtype=_type(k_cache, "cache"))
    sequences, tokens, max_q, max_kv = map(_int, (sequences, q.shape[0], max_q, max_kv))
    n = _load().attn_paged_workspace(cache, _Batch(sequences=sequences, tokens=tokens, max_q=max_q, max_kv=max_kv), _int(q.shape[1]))
    if n < 0:
        raise KvCacheError(-2, "no call takes these sizes")
    return n


def attn_paged(q, k_cache, v_cache, q_start, kv_len, table, o, lse, max_q, max_kv, scale, causal=True, k_scale=None, v_scale=None, workspace=None,
               stream=None) -> None:
    """Attention of the new tokens of a packed batch over a paged cache: ``q``, ``o`` [tokens][heads][d], ``lse`` float32 [tokens][heads] or None.

    ``max_q`` and ``max_kv`` bound the new tokens and the length of any sequence.  ``workspace``: a uint8 tensor of at least
    ``attn_paged_workspace`` bytes (None where that is 0)."""
    rc = _fast().attn_paged(q, k_cache, v_cache, q_start, kv_len, table, o, lse, max_q, max_kv, scale, causal, k_scale, v_scale, workspace, stream)
    if rc is not NotImplemented:
        return _check(rc)
    tokens, heads, d = q.shape
    rq, ro = _rows(q, "q"), _rows(o, "o", tuple(q.shape), q.dtype)
    if d != k_cache.shape[-1]:
        raise ValueError("q has heads of %d elements, the cache of %d" % (d, k_cache.shape[-1]))
    _check(_load().attn_paged(_pages(k_cache, v_cache, k_scale, v_scale), _batch(q_start, kv_len, table, tokens, max_q, max_kv), rq, ro,
                              _array(lse, torch.float32, "lse", (tokens, heads)), _int(heads), scale, int(bool(causal)), _type(q, "q"),
                              _array(workspace, torch.uint8, "workspace"), 0 if workspace is None else workspace.numel(), _stream(stream)))


def rope_frequencies(rot, base=10000.0, scaling=PLAIN, factor=1.0, trained=0.0, low=1.0, high=32.0) -> torch.Tensor:
    """Radians per position of each pair, float64 [rot / 2] on the CPU: as they are, or for a context ``factor`` times the trained one (LINEAR: positions
    squeezed; BASE: a larger base; PARTS: pair by pair, by the turns that it makes in ``trained`` positions)."""
    freq = (_cd * max(1, min(rot, 1024) // 2))()              # (more is refused)
    rot = _int(rot)
    _check(_load().rope_frequencies(freq, rot, base, scaling, factor, trained, low, high))
    return torch.tensor(list(freq), dtype=torch.float64)


def rope(x, y, freq, pos=None, layout=HALF, amplitude=1.0, inverse=False, stream=None) -> None:
    """``y`` = ``x`` turned by its positions: [batch][heads][tokens][d], any strides (``y`` may be ``x``).

    ``freq`` float64 [rot / 2] on the device: the first rot elements of a head are turned, the others copied.  ``pos`` int32 [batch][tokens] or
    [tokens] (None: 0, 1, ...).  ``inverse`` turns back, which is the gradient of ``x`` for a gradient of ``y``."""
    rc = _fast().rope(x, y, freq, pos, layout, amplitude, inverse, stream)
    if rc is not NotImplemented:
        return _check(rc)
    if x.dim() != 4 or x.shape != y.shape or x.dtype != y.dtype:
        raise ValueError("x and y: two tensors of one type and shape [batch][heads][tokens][d]; got %s and %s" % (tuple(x.shape), tuple(y.shape)))
    _unit(x, "x")
    _unit(y, "y")
    b, h, n, d = map(_int, x.shape)
    if pos is not None and tuple(pos.shape) not in ((b, n), (n,)):
        raise ValueError("pos: [batch][tokens] or [tokens]; got %s" % (tuple(pos.shape),))
    stride = n if pos is not None and pos.dim() == 2 else 0
    _check(_load().rope(_Tensor(_device(x, "x"), *x.stride()[:3]), _Tensor(_device(y, "y"), *y.stride()[:3]), b, h, n, d, _array(pos, torch.int32, "pos"), stride,
                        _array(freq, torch.float64, "freq"), _int(2 * freq.numel()), _int(layout), amplitude, int(bool(inverse)), _type(x, "x"), _stream(stream)))


def kv_append(k, v, k_cache, v_cache, q_start, kv_len, table, max_q, max_kv, q=None, q_out=None, freq=None, layout=HALF, amplitude=1.0, k_scale=None,
              v_scale=None, stream=None) -> None:
    """New tokens into the cache: ``k``, ``v`` [tokens][key heads][d], K turned by its position if ``freq`` (as for ``rope``) is given, and ``q``
    [tokens][heads][d] turned into ``q_out`` beside it.  ``kv_len`` counts the new tokens already."""
    rc = _fast().kv_append(k, v, k_cache, v_cache, q_start, kv_len, table, max_q, max_kv, q, q_out, freq, layout, amplitude, k_scale, v_scale, stream)
    if rc is not NotImplemented:
        return _check(rc)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out: both or neither")
    tokens = k.shape[0]
    shape = (tokens, k_cache.shape[1], k_cache.shape[3])
    rk, rv = _rows(k, "k", shape, k.dtype), _rows(v, "v", shape, k.dtype)
    rq = ro = _Rows()
    if q is not None:
        rq, ro = _rows(q, "q", (tokens, q.shape[1], shape[2]), k.dtype), _rows(q_out, "q_out", tuple(q.shape), k.dtype)
    _check(_load().kv_append(_pages(k_cache, v_cache, k_scale, v_scale), _batch(q_start, kv_len, table, tokens, max_q, max_kv), rk, rv, rq, ro,
                             0 if q is None else _int(q.shape[1]), _array(freq, torch.float64, "freq"), 0 if freq is None else _int(2 * freq.numel()), _int(layout),
                             amplitude,
                             _type(k, "k"), _stream(stream)))


def _book(ref, table, kv_len, page_size):
    rows = _int(kv_len.shape[0])
    if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != rows or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table: int32 [rows][entries], entries contiguous; got %s %s" % (table.dtype, tuple(table.shape)))
    return _Book(_array(ref, torch.int32, "ref"), _device(table, "table"), _array(kv_len, torch.int32, "kv_len"), _int(ref.numel()), rows, _int(table.shape[1]),
                 _int(table.stride(0)) if rows > 1 else 0, _int(page_size))


def _list(x, n, what):
    _int(n)
    return _array(x, torch.int32, what, (n,))


def kv_reserve(ref, table, kv_len, rows, new_len, missing, page_size, stream=None) -> None:
    """Rows get pages for ``new_len`` tokens in all, lowest free page first; ``missing`` int32 [1]: how many were not there.

    Their entries are -1 and stay so, though ``kv_len`` counts the tokens: after a call that missed pages give them back (``kv_free``), or set the ``kv_len`` of
    the rows to ``page_size`` times the entries that they have and call again."""
    rc = _fast().kv_reserve(ref, table, kv_len, rows, new_len, missing, page_size, stream)
    if rc is not NotImplemented:
        return _check(rc)
    n = rows.numel()
    _check(_load().kv_reserve(_book(ref, table, kv_len, page_size), _list(rows, n, "rows"), _list(new_len, n, "new_len"), n, _array(missing, torch.int32, "missing"),
                              _stream(stream)))


def kv_free(ref, table, kv_len, rows, page_size, stream=None) -> None:
    """The pages of rows are given back."""
    rc = _fast().kv_free(ref, table, kv_len, rows, page_size, stream)
    if rc is not NotImplemented:
        return _check(rc)
    n = rows.numel()
    _check(_load().kv_free(_book(ref, table, kv_len, page_size), _list(rows, n, "rows"), n, _stream(stream)))


def kv_fork(k_cache, v_cache, ref, table, kv_len, src, dst, missing, stream=None) -> None:
    """Rows ``dst`` become continuations of rows ``src``: full pages shared, a last page that is not full copied."""
    rc = _fast().kv_fork(k_cache, v_cache, ref, table, kv_len, src, dst, missing, stream)
    if rc is not NotImplemented:
        return _check(rc)
    n = src.numel()
    _check(_load().kv_fork(_pages(k_cache, v_cache, layers=True), _book(ref, table, kv_len, k_cache.shape[3]), _list(src, n, "src"), _list(dst, n, "dst"), n,
                           _array(missing, torch.int32, "missing"), _stream(stream)))


def kv_compact_workspace(pages) -> int:
    """Bytes of workspace of ``kv_compact`` for a cache of so many pages."""
    return _load().kv_compact_workspace(_int(pages))


def kv_compact(k_cache, v_cache, ref, table, kv_len, workspace, stream=None) -> None:
    """Pages in use move to the lowest numbers, with contents, counts and table entries."""
    rc = _fast().kv_compact(k_cache, v_cache, ref, table, kv_len, workspace, stream)
    if rc is not NotImplemented:
        return _check(rc)
    _check(_load().kv_compact(_pages(k_cache, v_cache, layers=True), _book(ref, table, kv_len, k_cache.shape[3]), _array(workspace, torch.uint8, "workspace"),
                              workspace.numel(), _stream(stream)))


def kv_copy_pages(k_cache, v_cache, src, dst, stream=None) -> None:
    """Pages ``src`` are copied to pages ``dst``, all layers, keys and values."""
    rc = _fast().kv_copy_pages(k_cache, v_cache, src, dst, stream)
    if rc is not NotImplemented:
        return _check(rc)
    n = src.numel()
    _check(_load().kv_copy_pages(_pages(k_cache, v_cache, layers=True), _list(src, n, "src"), _list(dst, n, "dst"), n, _stream(stream)))

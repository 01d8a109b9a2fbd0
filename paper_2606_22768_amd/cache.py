"""Attention over paged caches in microscaled 4-bit floating point: the C calls
fgd_mx4_cache_*, fgd_mx4_attend, fgd_extend_pages and fgd_truncate_pages, and
tensor-level calls on top of them.  A decoding turn:

    starts, positions, slots = extend_pages(tables, lengths, counts, free, free_count, cache.page, tokens)
    q, k = rotate_heads(q, k, positions, freqs, q_weight, k_weight)
    mx4_cache_write(cache, k, v, slots)
    o = mx4_attend(q, cache, tables, lengths, starts)

all on the GPU, so that turns can be captured into a graph.  Under a stream the
calls behave as those of mx4.py do.
"""

from __future__ import annotations

import ctypes
import math

from . import DTYPES, FGD_F32, _check, _dev, _stream, lib
from .heads import _array, _at, _form, _heads, _keep, _known
from .mx4 import _check_workspace, _current, _on, _on_gpu

_I64 = ctypes.c_int64


class fgd_mx4_cache(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("page", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("pages", ctypes.c_int64), ("data", ctypes.c_void_p),
                ("reserved", ctypes.c_int64)]

    def __init__(self, page=0, heads=0, head_dim=0, pages=0, data=None):
        super().__init__(ctypes.sizeof(fgd_mx4_cache), page, heads, head_dim, pages, _dev(data), 0)


class fgd_attention(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("sequences", ctypes.c_int32),
                ("table_width", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("window", ctypes.c_int32),
                ("tokens", ctypes.c_int64), ("most_queries", ctypes.c_int64), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32)]

    def __init__(self, dtype=FGD_F32, sequences=0, table_width=0, q_heads=0, window=0, tokens=0, most_queries=0,
                 scale=1.0):
        super().__init__(ctypes.sizeof(fgd_attention), DTYPES.get(dtype, dtype), sequences, table_width, q_heads,
                         window, tokens, most_queries, scale, 0)


class fgd_pages(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("page", ctypes.c_int32), ("requests", ctypes.c_int32),
                ("table_width", ctypes.c_int32), ("table_stride", ctypes.c_int64), ("tables", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("free", ctypes.c_void_p), ("free_count", ctypes.c_void_p),
                ("capacity", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    def __init__(self, page=0, requests=0, table_width=0, table_stride=0, tables=None, lengths=None, free=None,
                 free_count=None, capacity=0):
        super().__init__(ctypes.sizeof(fgd_pages), page, requests, table_width, table_stride, _dev(tables),
                         _dev(lengths), _dev(free), _dev(free_count), capacity, 0)


# --------------------------------------------------------------- raw C ABI

def fgd_mx4_cache_size(cache) -> int:
    n = _I64()
    _check(lib.fgd_mx4_cache_size(ctypes.byref(cache), ctypes.byref(n)), "fgd_mx4_cache_size")
    return n.value


def fgd_mx4_cache_write(cache, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, dtype, tokens, slots,
                        stream=None):
    _check(lib.fgd_mx4_cache_write(ctypes.byref(cache), _dev(k), k_token_stride, k_head_stride, _dev(v),
                                   v_token_stride, v_head_stride, DTYPES.get(dtype, dtype), tokens, _dev(slots),
                                   _stream(stream)), "fgd_mx4_cache_write")


def fgd_mx4_cache_read(cache, slots, tokens, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, dtype,
                       stream=None):
    _check(lib.fgd_mx4_cache_read(ctypes.byref(cache), _dev(slots), tokens, _dev(k), k_token_stride, k_head_stride,
                                  _dev(v), v_token_stride, v_head_stride, DTYPES.get(dtype, dtype), _stream(stream)),
           "fgd_mx4_cache_read")


def fgd_mx4_attend(cache, sizes, q, q_token_stride, q_head_stride, tables, table_stride, lengths, starts, out,
                   out_token_stride, out_head_stride, workspace=None, workspace_bytes=0, stream=None):
    """The C call; `cache` and `sizes` are fgd_mx4_cache and fgd_attention structures."""
    _check(lib.fgd_mx4_attend(ctypes.byref(cache), ctypes.byref(sizes), _dev(q), q_token_stride, q_head_stride,
                              _dev(tables), table_stride, _dev(lengths), _dev(starts), _dev(out), out_token_stride,
                              out_head_stride, _dev(workspace), workspace_bytes, _stream(stream)), "fgd_mx4_attend")


def fgd_mx4_attend_workspace_size(cache, sizes) -> int:
    n = _I64()
    _check(lib.fgd_mx4_attend_workspace_size(ctypes.byref(cache), ctypes.byref(sizes), ctypes.byref(n)),
           "fgd_mx4_attend_workspace_size")
    return n.value


def fgd_extend_pages(pages, counts, tokens, starts, positions, slots, stream=None):
    """The C call; `pages` is an fgd_pages structure."""
    _check(lib.fgd_extend_pages(ctypes.byref(pages), _dev(counts), tokens, _dev(starts), _dev(positions), _dev(slots),
                                _stream(stream)), "fgd_extend_pages")


def fgd_truncate_pages(pages, keep, stream=None):
    _check(lib.fgd_truncate_pages(ctypes.byref(pages), _dev(keep), _stream(stream)), "fgd_truncate_pages")


# ----------------------------------------------------------- tensor level

def _int(name, v, lo, hi):
    """A whole number of a C type's range (ctypes would take its lower bits)."""
    try:
        n = int(v)
    except (OverflowError, ValueError):  # infinity, NaN
        n = None
    if n is None or n != v:
        raise ValueError(f"{name}: expected a whole number, got {v}")
    if not lo <= n <= hi:
        raise ValueError(f"{name}: {v} is outside [{lo}, {hi}]")
    return n


class Mx4Cache:
    """A cache of keys and values in microscaled 4-bit floating point: `pages`
    pages of `page` tokens (a power of two, 16 at least) with `heads` heads of
    `dim` elements (a multiple of 32, 256 at most).  `data` is its device array
    (uint8, laid out as fgd.h says), allocated when not given; its bytes need
    no initial value."""

    __slots__ = ("_data", "_form", "_c")

    def __init__(self, pages, page, heads, dim, device=None, data=None):
        import torch

        pages = _int("pages", pages, 0, 0x7fffffff)
        page, heads, dim = (_int(n, v, 1, 0x7fffffff) for n, v in (("page", page), ("heads", heads), ("dim", dim)))
        need = fgd_mx4_cache_size(fgd_mx4_cache(page, heads, dim, pages))
        if data is None:
            data = torch.empty(need, dtype=torch.uint8, device="cuda" if device is None else device)
        else:
            at = data.device if device is None else torch.device(device)
            if at.index is None and at.type == data.device.type:  # "cuda": whichever it is on
                at = data.device
            _array("data", data, torch.uint8, at)
            if data.numel() != need:
                raise ValueError(f"data: expected {need} bytes, got {data.numel()}")
        self._data = data
        self._form = (pages, page, heads, dim, data.device)
        self._c = fgd_mx4_cache(page, heads, dim, pages, data.data_ptr())

    # Fixed for a cache's life: the kernels read as many bytes as they say.
    data = property(lambda self: self._data)
    pages = property(lambda self: self._form[0])
    page = property(lambda self: self._form[1])
    heads = property(lambda self: self._form[2])
    dim = property(lambda self: self._form[3])
    device = property(lambda self: self._form[4])

    @property
    def nbytes(self):
        return self._data.numel()

    def __repr__(self):
        return (f"Mx4Cache(pages={self.pages}, page={self.page}, heads={self.heads}, dim={self.dim}, "
                f"device={self.device})")


_SETTINGS = (type(None), float, int)  # of which equal values mean equal calls


def _is_cache(c):
    if not isinstance(c, Mx4Cache):
        raise TypeError(f"cache: expected an Mx4Cache, got {type(c).__name__}")
    return c


def _tokens(name, t, cache, like=None):
    """(dtype code, tokens, heads) of heads that the cache can hold."""
    if getattr(t, "ndim", 3) != 3:
        raise ValueError(f"{name}: expected [tokens][heads][dim], got shape {tuple(t.shape)}")
    code, _, tokens, heads, dim = _heads(name, t, like)
    if dim != cache.dim:
        raise ValueError(f"{name}: expected heads of {cache.dim} elements, got {dim}")
    return code, tokens, heads


def _slots(slots, tokens, device):
    import torch

    _array("slots", slots, torch.int64, device)
    if slots.dim() != 1 or slots.shape[0] != tokens:
        raise ValueError(f"slots: expected shape [{tokens}], got {tuple(slots.shape)}")


def mx4_cache_write(cache, k, v, slots, stream=None):
    """Writes keys and values k, v [T][heads][dim] (float32 or bfloat16, heads
    contiguous) to the cache's slots (int64 [T], slot s being token s % page of
    page s // page).  A slot outside the cache, as -1, is passed over; slots
    that are written must differ."""
    _is_cache(cache)
    key = None
    if stream is None:
        try:
            key = (cache._form, _form(k), _form(v), _form(slots), "write")
            plan = _known(key)
        except AttributeError:  # no tensors: the checks say so
            key = plan = None
        if plan is not None:
            index, code, T, kt, kh, vt, vh = plan
            _check(lib.fgd_mx4_cache_write(ctypes.byref(cache._c), k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, code, T,
                                           slots.data_ptr(), _current(index)), "fgd_mx4_cache_write")
            return
    code, T, heads = _tokens("k", k, cache)
    _tokens("v", v, cache, k)
    for name, t in (("k", k), ("v", v)):
        if t.shape[1] != cache.heads:
            raise ValueError(f"{name}: expected {cache.heads} heads, got {t.shape[1]}")
    _slots(slots, T, cache.device)
    _on_gpu("cache", cache.data, None)
    _on_gpu("k", k, cache.device)
    with _on(cache.device, stream):
        fgd_mx4_cache_write(cache._c, k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1), code, T, slots,
                            _current(cache.device))
    if key is not None:
        _keep(key, cache.device.index, code, T, k.stride(0), k.stride(1), v.stride(0), v.stride(1))


def mx4_cache_read(cache, slots, dtype="f32", stream=None):
    """The values (k, v), [T][heads][dim] of `dtype` ("f32", "bf16" or torch's),
    that slots (int64 [T]) hold; zeros for a slot outside the cache."""
    import torch

    _is_cache(cache)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}.get(dtype, dtype)
    if t not in (torch.float32, torch.bfloat16):
        raise TypeError(f"dtype: expected 'f32' or 'bf16', got {dtype!r}")
    if not isinstance(slots, torch.Tensor):
        raise TypeError(f"slots: expected a torch tensor, got {type(slots).__name__}")
    T = slots.shape[0] if slots.dim() == 1 else -1
    _slots(slots, T, cache.device)
    _on_gpu("cache", cache.data, None)
    with _on(cache.device, stream):
        both = torch.empty((2, T, cache.heads, cache.dim), dtype=t, device=cache.device)
        k, v = both.unbind()
        fgd_mx4_cache_read(cache._c, slots, T, k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1),
                           "f32" if t == torch.float32 else "bf16", _current(cache.device))
    return k, v


def _tables(tables, device):
    """(requests, width, stride) of block tables."""
    import torch

    if not isinstance(tables, torch.Tensor):
        raise TypeError(f"tables: expected a torch tensor, got {type(tables).__name__}")
    if tables.dtype != torch.int32:
        raise TypeError(f"tables: expected {torch.int32}, got {tables.dtype}")
    if tables.dim() != 2:
        raise ValueError(f"tables: expected [requests][pages], got shape {tuple(tables.shape)}")
    if tables.device != device:
        raise ValueError(f"tables: expected a tensor on {device}, got {tables.device}")
    B, W = tables.shape
    if W > 1 and B and tables.stride(1) != 1:
        raise ValueError("tables: rows must be contiguous")
    if B > 1 and tables.stride(0) < W:
        raise ValueError("tables: rows must not overlap")
    return B, W, tables.stride(0) if B > 1 else W


def _ints(name, t, n, device):
    import torch

    _array(name, t, torch.int32, device)
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{name}: expected shape [{n}], got {tuple(t.shape)}")


def mx4_attend(q, cache, tables, lengths, starts=None, max_q=None, scale=None, window=0, out=None, workspace=None,
               stream=None):
    """Attention of queries q [T][heads][dim] (float32 or bfloat16, heads
    contiguous; a multiple of the cache's heads, neighbours sharing one) over
    the cache, causal: sequence b has lengths[b] keys (int32 [B]), on the pages
    that tables[b] lists (int32 [B][W]), and the queries [starts[b], starts[b +
    1]) (int32 [B + 1]), the last of which stands at its last key.  Without
    starts every sequence has one query.  With a window a query sees the last
    `window` keys only.  `scale` is 1 / sqrt(dim) unless given.  max_q, the
    most queries that a sequence has, steers the launch where it is known.
    Rows of no sequence stay as they are in `out`; in a new tensor they hold
    nothing of use.  The workspace (a uint8 device tensor of
    fgd_mx4_attend_workspace_size bytes) is allocated when not given."""
    import torch

    _is_cache(cache)
    key = None
    if out is None and workspace is None and stream is None and type(window) is int and \
            type(scale) in _SETTINGS and type(max_q) in _SETTINGS:
        try:
            key = (cache._form, _form(q), _form(tables), _form(lengths), _form(starts), max_q, scale, window, "attend")
            plan = _known(key)
        except AttributeError:  # no tensors: the checks say so
            key = plan = None
        if plan is not None:
            index, sizes, need, qt, qh, stride, ot, oh = plan
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            work = q.new_empty(need, dtype=torch.uint8) if need else None
            _check(lib.fgd_mx4_attend(ctypes.byref(cache._c), ctypes.byref(sizes), q.data_ptr(), qt, qh,
                                      tables.data_ptr(), stride, lengths.data_ptr(), _at(starts), out.data_ptr(), ot,
                                      oh, _at(work), need, _current(index)), "fgd_mx4_attend")
            return out
    code, T, heads = _tokens("q", q, cache)
    dev = cache.device
    if heads == 0 or heads % cache.heads:
        raise ValueError(f"q: expected a multiple of {cache.heads} heads, got {heads}")
    B, W, stride = _tables(tables, dev)
    _ints("lengths", lengths, B, dev)
    if starts is not None:
        _ints("starts", starts, B + 1, dev)
    elif T != B:
        raise ValueError(f"q: expected {B} rows, one for each sequence, got {T} (several need starts)")
    if out is not None:
        _heads("out", out, q)
        if out.shape != q.shape:
            raise ValueError(f"out: expected shape {tuple(q.shape)}, got {tuple(out.shape)}")
    window = _int("window", window, 0, math.inf)
    if starts is None:
        most = 1
    elif max_q is None:
        most = min(T, -(-2 * T // max(B, 1)))  # twice the mean
    else:
        most = min(_int("max_q", max_q, 0, 1 << 62), T)
    _on_gpu("cache", cache.data, None)
    _on_gpu("q", q, dev)
    sizes = fgd_attention(code, B, W, heads, min(window, 0x7fffffff), T, most,
                          cache.dim ** -0.5 if scale is None else float(scale))
    need = fgd_mx4_attend_workspace_size(cache._c, sizes)
    if workspace is not None:
        _check_workspace(workspace, need, dev)
    with _on(dev, stream):
        out = torch.empty(q.shape, dtype=q.dtype, device=dev) if out is None else out
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        fgd_mx4_attend(cache._c, sizes, q, q.stride(0), q.stride(1), tables, stride, lengths, starts, out,
                       out.stride(0), out.stride(1), workspace,
                       0 if workspace is None else workspace.numel() * workspace.element_size(), _current(dev))
    if key is not None:
        _keep(key, dev.index, sizes, need, q.stride(0), q.stride(1), stride, out.stride(0), out.stride(1))
    return out


def _state(plan, tables, lengths, free, free_count):
    """The C structure of a plan's sizes with these arrays."""
    page, B, W, stride, capacity = plan
    return fgd_pages(page, B, W, stride, tables.data_ptr(), lengths.data_ptr(), free.data_ptr(), free_count.data_ptr(),
                     capacity)


def _pages(tables, lengths, free, free_count, page):
    """(device, requests, sizes) of the state, checked."""
    import torch

    if not isinstance(lengths, torch.Tensor):
        raise TypeError(f"lengths: expected a torch tensor, got {type(lengths).__name__}")
    dev = lengths.device
    B, W, stride = _tables(tables, dev)
    _ints("lengths", lengths, B, dev)
    _array("free", free, torch.int32, dev)
    if free.dim() != 1:
        raise ValueError(f"free: expected one axis, got shape {tuple(free.shape)}")
    _ints("free_count", free_count, 1, dev)
    return dev, B, (_int("page", page, 1, 0x7fffffff), B, W, stride, free.shape[0])


def extend_pages(tables, lengths, counts, free, free_count, page, tokens, stream=None):
    """Room for counts[b] (int32 [B]) further tokens of every request: takes
    pages from the top of the stack free[:free_count[0]] (int32), adds them to
    tables (int32 [B][W]), lets lengths (int32 [B]) grow, all in place, and
    returns (starts int32 [B + 1], positions int32 [tokens], slots int64
    [tokens]) of the new tokens, of which there may be `tokens` at most.  A
    request that cannot be served wholly keeps its length and gets no tokens;
    the rule stands at fgd_extend_pages in fgd.h.  Behind the last token
    positions are 0 and slots -1, which mx4_cache_write passes over."""
    import torch

    key = None
    if stream is None and type(page) is int and type(tokens) is int:
        try:
            key = (_form(tables), _form(lengths), _form(counts), _form(free), _form(free_count), page, tokens, "extend")
            plan = _known(key)
        except AttributeError:  # no tensors: the checks say so
            key = plan = None
        if plan is not None:
            index, B, sizes = plan
            starts, positions, slots = counts.new_empty(B + 1), counts.new_empty(tokens), \
                counts.new_empty(tokens, dtype=torch.int64)
            _check(lib.fgd_extend_pages(ctypes.byref(_state(sizes, tables, lengths, free, free_count)),
                                        counts.data_ptr(), tokens, starts.data_ptr(), positions.data_ptr(),
                                        slots.data_ptr(), _current(index)), "fgd_extend_pages")
            return starts, positions, slots
    dev, B, sizes = _pages(tables, lengths, free, free_count, page)
    _ints("counts", counts, B, dev)
    tokens = _int("tokens", tokens, 0, 0x7fffffff)
    _on_gpu("lengths", lengths, None)
    with _on(dev, stream):
        starts = torch.empty(B + 1, dtype=torch.int32, device=dev)
        positions = torch.empty(tokens, dtype=torch.int32, device=dev)
        slots = torch.empty(tokens, dtype=torch.int64, device=dev)
        fgd_extend_pages(_state(sizes, tables, lengths, free, free_count), counts, tokens, starts, positions, slots,
                         _current(dev))
    if key is not None:
        _keep(key, dev.index, B, sizes)
    return starts, positions, slots


def truncate_pages(tables, lengths, keep, free, free_count, page, stream=None):
    """Shortens requests to keep[b] (int32 [B]) tokens, in place: 0 for one that
    is done, its length or more for one that stays as it is.  Pages without a
    token left go back on the stack, their entries in tables become -1."""
    key = None
    if stream is None and type(page) is int:
        try:
            key = (_form(tables), _form(lengths), _form(keep), _form(free), _form(free_count), page, "truncate")
            plan = _known(key)
        except AttributeError:  # no tensors: the checks say so
            key = plan = None
        if plan is not None:
            index, sizes = plan
            _check(lib.fgd_truncate_pages(ctypes.byref(_state(sizes, tables, lengths, free, free_count)),
                                          keep.data_ptr(), _current(index)), "fgd_truncate_pages")
            return
    dev, B, sizes = _pages(tables, lengths, free, free_count, page)
    _ints("keep", keep, B, dev)
    _on_gpu("lengths", lengths, None)
    with _on(dev, stream):
        fgd_truncate_pages(_state(sizes, tables, lengths, free, free_count), keep, _current(dev))
    if key is not None:
        _keep(key, dev.index, sizes)

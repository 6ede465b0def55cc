"""A cache of keys and values in 8-bit pages, and the attention of single tokens
over all or chosen ones of them: Python binding of the paged section of
``include/frog.h`` (the formulas and the limits stand there).  Argument checks
and marshalling only; serving operators, which take no gradients.
"""
from __future__ import annotations

import ctypes as C

import torch
from torch.autograd.graph import increment_version

from . import _check, lib
from .attention import _D, _I, _P, _TYPES, _launch, _need, _no_gradient, _on, _own_workspace, _packer, _plain, _rows, _values, _workspace

CACHE_E4M3, CACHE_INT8 = 0, 1
_CODES = {torch.float8_e4m3fn: CACHE_E4M3, torch.int8: CACHE_INT8}
_STORAGE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}

_CACHE = [("cache." + n, _P) for n in ("k", "v", "k_exp", "v_exp", "bounds")] + [("cache.num_pages", _I)] + \
         [("cache." + n, _D) for n in ("kv_heads", "page", "d", "storage")]


class WriteArgs(C.Structure):
    _fields_ = [*_CACHE, *_rows("k", 2), *_rows("v", 2), ("starts", _P), ("pages", _P), ("lengths", _P), ("batch", _I), ("tokens", _I),
                ("pages_per_request", _I), ("type", _D)]


class ReadArgs(C.Structure):
    _fields_ = [*_CACHE, *_rows("k", 3), *_rows("v", 3), ("pages", _P), ("lengths", _P), ("batch", _I), ("slots", _I),
                ("pages_per_request", _I), ("type", _D)]


class SelectArgs(C.Structure):
    _fields_ = [*_CACHE, *_rows("q", 2), ("pages", _P), ("lengths", _P), ("chosen", _P), ("ws", _P), ("ws_bytes", _I), ("batch", _I),
                ("pages_per_request", _I), ("keep", _I), ("first", _I), ("recent", _I), ("heads", _D), ("type", _D)]


class PagedArgs(C.Structure):
    _fields_ = [*_CACHE, *_rows("q", 2), ("pages", _P), ("lengths", _P), ("chosen", _P), ("lr", _P), ("slopes", _P), *_rows("out", 2),
                ("lse", _P), ("ws", _P), ("ws_bytes", _I), ("batch", _I), ("pages_per_request", _I), ("num_chosen", _I), ("heads", _D),
                ("type", _D), ("scale", C.c_float), ("cap", C.c_float)]


_pack_write, _pack_read, _pack_select, _pack_paged = (_packer(c) for c in (WriteArgs, ReadArgs, SelectArgs, PagedArgs))


class PagedCache:
    """Pages of keys and values in 8 bits: every row of d values as d codes and
    one power of two.

    k, v: codes [num_pages, kv_heads, page, d], float8_e4m3fn or int8; k_exp,
    v_exp: uint8 [num_pages, kv_heads, page], the power plus 127; bounds:
    bfloat16 [num_pages, kv_heads, 2, d], the least and the largest key of every
    channel of a page (None: not kept; :func:`select_pages` needs them).  All
    contiguous on one GPU.  page 16, 32, 64, 128 or 256; d 32, 64, 96 or 128.
    The tensors are the cache: a program that keeps them elsewhere (saved,
    moved) makes a new PagedCache of them."""

    __slots__ = ("_tensors", "_tail", "_written")

    def __init__(self, k, v, k_exp, v_exp, bounds=None):
        _need(k.dim() == 4 and k.dtype in _CODES and k.is_cuda, "k: codes [num_pages, kv_heads, page, d] of float8_e4m3fn or int8 on a GPU are wanted")
        n, h, page, d = k.shape
        _plain("k", k, k.dtype, k.shape, k)
        _plain("v", v, k.dtype, k.shape, k)
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            _plain(name, t, torch.uint8, (n, h, page), k)
        if bounds is not None:
            _plain("bounds", bounds, torch.bfloat16, (n, h, 2, d), k)
        _need(page in (16, 32, 64, 128, 256), f"page {page}: 16, 32, 64, 128 or 256")
        _need(d in (32, 64, 96, 128), f"d {d}: 32, 64, 96 or 128")
        # (not to be replaced one by one: the kernels take their sizes from here)
        self._tensors = (k, v, k_exp, v_exp, bounds)
        self._tail = (n, h, page, d, _CODES[k.dtype])
        self._written = [t for t in self._tensors if t is not None and not t.is_inference()]

    k, v, k_exp, v_exp, bounds = (property(lambda self, i=i: self._tensors[i]) for i in range(5))
    device = property(lambda self: self._tensors[0].device)
    shape = property(lambda self: self._tail[:4], doc="num_pages, kv_heads, page, d")

    @classmethod
    def empty(cls, num_pages, kv_heads, d, *, page=64, storage="e4m3", bounds=True, device="cuda"):
        """A cache of rows of value 0.  storage: "int8" (normally distributed rows of 128 are off by 0.9 % of their
        norm) or "e4m3" (2.6 %, and no more for the other values of a row with one far above them)."""
        if storage not in _STORAGE:
            raise ValueError(f"storage {storage!r}: one of {sorted(_STORAGE)}")
        k, v = (torch.zeros((num_pages, kv_heads, page, d), dtype=torch.uint8, device=device).view(_STORAGE[storage]) for _ in range(2))
        ke, ve = (torch.full((num_pages, kv_heads, page), 27, dtype=torch.uint8, device=device) for _ in range(2))
        return cls(k, v, ke, ve, torch.zeros((num_pages, kv_heads, 2, d), dtype=torch.bfloat16, device=device) if bounds else None)

    def _head(self):
        k, v, ke, ve, b = self._tensors
        return (k.data_ptr(), v.data_ptr(), ke.data_ptr(), ve.data_ptr(), 0 if b is None else b.data_ptr(), *self._tail)

    def _run(self, call, stream, *inputs):
        """`call()`, enqueued on `stream` (None: the current one)."""
        return call() if stream is None else _on(stream, call, (*self._tensors, *inputs))


def _table(cache, pages, lengths):
    """Pointers of the requests' page table and lengths, and their numbers."""
    if pages.dim() != 2:
        raise ValueError("pages: [batch, pages_per_request] is wanted")
    b, width = pages.shape
    like = cache._tensors[0]
    return _plain("pages", pages, torch.int32, (b, width), like), _plain("lengths", lengths, torch.int32, (b,), like), b, width


def _query(q, cache, batch):
    kind, d = _TYPES.get(q.dtype), cache._tail[3]
    if kind is None or q.dim() != 3 or q.shape[0] != batch or q.shape[2] != d or q.get_device() != cache._tensors[0].get_device():
        raise ValueError(f"q {tuple(q.shape)} of {q.dtype} on {q.device}: [{batch}, heads, {d}] of float32, float16 or bfloat16 on "
                         f"{cache.device} is wanted")
    if q.stride(2) != 1:
        raise ValueError("q: the last axis must have stride 1")
    return kind


def _most_workspace(batch, heads, d, rows):
    """Bytes that an attention call over ``rows`` rows a request takes at most: a part has 256 of them or more, and keeps an
    output, a maximum and a sum of every query row."""
    return batch * heads * (d + 2) * 4 * -(-rows // 256)


def cache_write(cache, k, v, pages, lengths, *, starts=None, stream=None):
    """Append rows to the requests of a cache, quantised.

    k, v [tokens, kv_heads, d], float32, float16 or bfloat16, rows on 16-byte
    boundaries.  pages int32 [batch, pages_per_request]: every request's pages
    in order; lengths int32 [batch]: the requests' rows with the new ones.
    starts int32 [batch + 1]: request b's new rows are starts[b] .. starts[b + 1]
    - 1, its last ones (None: tokens / batch each).  A page belongs to the
    request that writes it, which lists it once.  The bounds of a page written from its row 0 on are
    those of the new rows, else they widen the old ones."""
    _no_gradient(("k", "v"), (k, v))
    kind = _values(("k", "v"), (k, v), (3, 3))
    t, (_, h, _, d) = k.shape[0], cache._tail[:4]
    if k.shape != (t, h, d) or v.shape != k.shape or k.get_device() != cache._tensors[0].get_device():
        raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)} on {k.device}: twice [tokens, {h}, {d}] on {cache.device} are wanted")
    table, rows, b, width = _table(cache, pages, lengths)
    args = _pack_write(*cache._head(), k.data_ptr(), *k.stride()[:2], v.data_ptr(), *v.stride()[:2],
                       0 if starts is None else _plain("starts", starts, torch.int32, (b + 1,), k), table, rows, b, t, width, kind)

    def run():
        _launch(lib().frog_cache_write, args, k.device)
        return ()

    cache._run(run, stream, k, v, pages, lengths, starts)
    if cache._written:
        increment_version(cache._written)      # (written by address: autograd has to hear of it)


def cache_read(cache, pages, lengths, slots=None, *, dtype=torch.bfloat16, stream=None):
    """The first ``slots`` rows (None: all that the table has room for) of every
    request: k, v [batch, slots, kv_heads, d] of ``dtype``, 0 past a length; as
    :func:`attend` takes them."""
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"dtype {dtype}: float32, float16 or bfloat16")
    table, rows, b, width = _table(cache, pages, lengths)
    _, h, page, d, _ = cache._tail
    slots = width * page if slots is None else slots
    _need(slots >= 0, "slots is negative")

    def run():
        k = torch.empty((b, slots, h, d), dtype=dtype, device=pages.device)
        v = torch.empty_like(k)
        strides = (slots * h * d, h * d, d)
        _launch(lib().frog_cache_read, _pack_read(*cache._head(), k.data_ptr(), *strides, v.data_ptr(), *strides, table, rows, b, slots, width,
                                                  kind), pages.device)
        return k, v

    return cache._run(run, stream, pages, lengths)


def select_pages(q, cache, pages, lengths, keep, *, first=0, recent=1, stream=None):
    """The ``keep`` pages of every (request, kv head) that a token has to look
    at: the first ``first``, the newest ``recent``, and of the others those with
    the largest bound on the head's scores, q [batch, heads, d], summed over the
    heads that share the kv head (equal: the lower page).  Returns int32 [batch,
    kv_heads, keep]: numbers of pages within the request, ascending, -1 behind
    them, for ``chosen`` of :func:`attend_paged`.  The bound is one of q . k: a
    distance bias, an ``lr`` or a negative scale of that call is not in it."""
    _no_gradient(("q",), (q,))
    table, rows, b, width = _table(cache, pages, lengths)
    kind = _query(q, cache, b)
    kv = cache._tail[1]
    _need(cache.bounds is not None, "the cache keeps no bounds")
    if not (0 <= first and 0 <= recent and first + recent <= keep):
        raise ValueError(f"first {first}, recent {recent}, keep {keep}: first + recent <= keep is wanted")

    def run():
        chosen = lengths.new_empty((b, kv, keep))
        head = (*cache._head(), q.data_ptr(), *q.stride()[:2], table, rows, chosen.data_ptr())
        tail = (b, width, keep, first, recent, q.shape[1], kind)
        args, ws, L = _pack_select(*head, 0, 0, *tail), None, lib()
        if _own_workspace(b * kv * width > 2 ** 24):
            ws, at = _workspace(L.frog_select_pages_workspace, args, q.device)
            args = _pack_select(*head, *at, *tail)
        _launch(L.frog_select_pages, args, q.device)
        return (chosen,)

    return cache._run(run, stream, q, pages, lengths)[0]


def attend_paged(q, cache, pages, lengths, *, chosen=None, lr=None, scale=None, cap=0.0, slopes=None, return_lse=False, stream=None):
    """Attention of one token per request, q [batch, heads, d], over the rows of
    its pages, or over the ``chosen`` ones (int32 [batch, kv_heads, n], as
    :func:`select_pages` gives them; an entry of -1 takes as long as a page).  A
    table much wider than the longest request costs time.  lr int32 [batch, 2]: the interval of rows
    a request sees (None: all).  scale, cap and slopes [heads] as for
    :func:`attend`; the query stands on the request's last row.  Several tokens
    of one request at once are several requests of the same pages with lengths
    that grow by one.  Returns out [batch, heads, d], and lse [batch, heads]
    with return_lse."""
    _no_gradient(("q", "slopes"), (q, slopes))
    table, rows, b, width = _table(cache, pages, lengths)
    kind = _query(q, cache, b)
    h, kv, page, d = q.shape[1], *cache._tail[1:4]
    num = 0
    if chosen is not None:
        num = chosen.shape[-1] if chosen.dim() else 0
        # (an empty list is not none: any address that is not null, of which nothing is read)
        chosen_at = _plain("chosen", chosen, torch.int32, (b, kv, num), q) or rows

    def run():
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = torch.empty((b, h), dtype=torch.float32, device=q.device) if return_lse else None
        head = (*cache._head(), q.data_ptr(), *q.stride()[:2], table, rows, 0 if chosen is None else chosen_at,
                0 if lr is None else _plain("lr", lr, torch.int32, (b, 2), q),
                0 if slopes is None else _plain("slopes", slopes, torch.float32, (h,), q), out.data_ptr(), h * d, d,
                0 if lse is None else lse.data_ptr())
        tail = (b, width, num, h, kind, d ** -0.5 if scale is None else scale, cap)
        args, ws, L = _pack_paged(*head, 0, 0, *tail), None, lib()
        # (the listed pages, or else the table's width, are what a call is cut by)
        most = _most_workspace(b, h, d, (width if chosen is None else num) * page)
        if _own_workspace(most > 2 ** 26 and L.frog_attend_paged_workspace(args) > 2 ** 26):
            ws, at = _workspace(L.frog_attend_paged_workspace, args, q.device)
            args = _pack_paged(*head, *at, *tail)
        _launch(L.frog_attend_paged, args, q.device)
        return out, lse

    out, lse = cache._run(run, stream, q, pages, lengths, chosen, lr, slopes)
    return (out, lse) if return_lse else out

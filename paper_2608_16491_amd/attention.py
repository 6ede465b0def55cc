"""Attention over rows kept in attribute order, and the upkeep of the cache
that holds them: Python binding of the attention section of ``include/frog.h``
(the formulas and the limits stand there).  Argument checks and marshalling
only; the gradients go through ``torch.autograd``.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import STORAGE_BF16, STORAGE_F16, STORAGE_F32, FrogError, _check, lib

_TYPES = {torch.float32: STORAGE_F32, torch.float16: STORAGE_F16, torch.bfloat16: STORAGE_BF16}
_P, _I, _D = C.c_void_p, C.c_int64, C.c_int32


def _rows(name, strides):
    return [(name, _P), (name + "_stride", _I * strides)]


class AttendArgs(C.Structure):
    _fields_ = [*_rows("q", 3), *_rows("k", 3), *_rows("v", 3), *_rows("out", 3), ("lr", _P), ("lr_stride", _I), ("slopes", _P),
                ("at_q", _P), ("at_q_stride", _I), ("at_k", _P), ("at_k_stride", _I * 2), ("lse", _P), ("w_in", _P), ("w_out", _P),
                *_rows("dout", 3), *_rows("dq", 3), *_rows("dk", 3), *_rows("dv", 3), ("ws", _P), ("ws_bytes", _I), ("batch", _I),
                ("queries", _I), ("keys", _I), ("heads", _D), ("kv_heads", _D), ("d", _D), ("type", _D), ("scale", C.c_float),
                ("cap", C.c_float)]


class SharedArgs(C.Structure):
    _fields_ = [*_rows("q", 2), *_rows("k", 2), *_rows("v", 2), *_rows("k_pages", 3), *_rows("v_pages", 3), ("pages", _P),
                ("lengths", _P), ("lr", _P), ("slopes", _P), *_rows("out", 2), ("lse", _P), ("ws", _P), ("ws_bytes", _I),
                ("batch", _I), ("prefix", _I), ("num_pages", _I), ("pages_per_request", _I), ("page", _D), ("heads", _D),
                ("kv_heads", _D), ("d", _D), ("type", _D), ("scale", C.c_float), ("cap", C.c_float)]


class EvictArgs(C.Structure):
    _fields_ = [*_rows("k", 3), *_rows("v", 3), ("weights", _P), ("positions", _P), ("lengths", _P), ("k_out", _P), ("v_out", _P),
                ("weights_out", _P), ("positions_out", _P), ("lengths_out", _P), ("ws", _P), ("ws_bytes", _I), ("batch", _I),
                ("slots", _I), ("keep", _I), ("recent", _I), ("heads", _D), ("d", _D), ("type", _D)]


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _tensor(name, t, dtype, shape, device, packed=True):
    """`t` is None or a tensor of this type, shape and device (packed: contiguous)."""
    if t is None:
        return
    _need(t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.device == device and (not packed or t.is_contiguous()),
          f"{name}: {dtype} {tuple(shape)} on {device}{', contiguous' if packed else ''} is wanted, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _values(name, t, dtype, dims, device):
    """A tensor of rows: its last axis has no gaps."""
    _need(t.dim() == dims and t.dtype == dtype and t.device == device, f"{name}: {dims} axes of {dtype} on {device} are wanted, "
          f"not {t.dim()} of {t.dtype} on {t.device}")
    _need(t.shape[-1] < 2 or t.stride(-1) == 1, f"{name}: the last axis must have stride 1")


def _start(q):
    _need(q.is_cuda, f"q is on {q.device}: a GPU tensor is wanted")
    _need(q.dtype in _TYPES, f"q is {q.dtype}: float32, float16 or bfloat16")


def _put(a, name, t):
    if t is not None:
        setattr(a, name, t.data_ptr())
        setattr(a, name + "_stride", t.stride()[:-1])


def _at(t):
    return None if t is None else t.data_ptr()


def _workspace(a, bytes_, device):
    """The call's workspace, from torch's allocator (so that a captured graph keeps it)."""
    if bytes_ < 0:
        _check(bytes_)
    if bytes_ == 0:
        return None
    ws = torch.empty(bytes_, dtype=torch.uint8, device=device)
    a.ws, a.ws_bytes = ws.data_ptr(), bytes_
    return ws


def _launch(fn, a, stream, device, tensors):
    """Enqueue on `stream` (default: the current one of the device); memory that another stream's allocator pool holds is kept
    until `stream` is done with it."""
    here = torch.cuda.current_stream(device)
    s = here if stream is None else stream
    _need(s.device == device, f"the stream is on {s.device}, the tensors on {device}")
    with torch.cuda.device(device):
        _check(fn(C.byref(a), s.cuda_stream))
    if s != here:
        for t in tensors:
            if t is not None:
                t.record_stream(s)


class _Call:
    """The checked arguments of one attention call, apart from its outputs."""

    def __init__(self, q, k, v, lr, scale, cap, slopes, at_q, at_k):
        _start(q)
        _values("q", q, q.dtype, 4, q.device)
        _values("k", k, q.dtype, 4, q.device)
        _values("v", v, q.dtype, 4, q.device)
        b, tq, h, d = q.shape
        tk, kv = k.shape[1], k.shape[2]
        _need(k.shape == (b, tk, kv, d) and v.shape == k.shape, f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}: "
              "[batch, queries, heads, d] and twice [batch, keys, kv_heads, d] are wanted")
        _need((slopes is None) == (at_q is None) == (at_k is None), "slopes, at_q and at_k go together")
        self.dev, self.shape, self.kv = q.device, (b, tq, h, d, tk), kv
        self.extra = (lr, slopes, at_q, at_k)
        a = self.a = AttendArgs()
        if lr is not None:
            _tensor("lr", lr, torch.int32, (tq, 2) if lr.dim() == 2 else (b, tq, 2), q.device)
            a.lr, a.lr_stride = lr.data_ptr(), 0 if lr.dim() == 2 else 2 * tq
        if slopes is not None:
            _tensor("slopes", slopes, torch.float32, (h,), q.device)
            _tensor("at_q", at_q, torch.float32, (b, tq), q.device)
            _tensor("at_k", at_k, torch.float32, (b, tk) if at_k.dim() == 2 else (b, kv, tk), q.device)
            _need(not slopes.requires_grad, "slopes take no gradient")
            a.slopes, a.at_q, a.at_k, a.at_q_stride = slopes.data_ptr(), at_q.data_ptr(), at_k.data_ptr(), tq
            a.at_k_stride = (tk, 0) if at_k.dim() == 2 else (kv * tk, tk)
        a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type = b, tq, tk, h, kv, d, _TYPES[q.dtype]
        a.scale, a.cap = d ** -0.5 if scale is None else scale, cap
        _put(a, "q", q)
        _put(a, "k", k)
        _put(a, "v", v)

    def forward(self, q, k, v, want_lse, w_in, w_out, stream):
        a, (b, tq, h, d, tk) = self.a, self.shape
        out = torch.empty((b, tq, h, d), dtype=q.dtype, device=self.dev)
        lse = torch.empty((b, h, tq), dtype=torch.float32, device=self.dev) if want_lse else None
        _put(a, "out", out)
        a.lse, a.w_in, a.w_out = _at(lse), _at(w_in), _at(w_out)
        ws = _workspace(a, lib().frog_attend_workspace(C.byref(a), 0), self.dev)
        _launch(lib().frog_attend, a, stream, self.dev, (q, k, v, *self.extra, out, lse, w_in, w_out, ws))
        return out, lse

    def backward(self, q, k, v, out, lse, dout):
        a = self.a
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=self.dev) for t in (q, k, v))
        for name, t in (("q", q), ("k", k), ("v", v), ("out", out), ("dout", dout), ("dq", dq), ("dk", dk), ("dv", dv)):
            _put(a, name, t)
        a.lse, a.w_in, a.w_out, a.ws, a.ws_bytes = lse.data_ptr(), None, None, None, 0
        ws = _workspace(a, lib().frog_attend_workspace(C.byref(a), 1), self.dev)
        _launch(lib().frog_attend_backward, a, None, self.dev, (ws,))
        return dq, dk, dv


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, call, w_in, w_out, stream):
        out, lse = call.forward(q, k, v, True, w_in, w_out, stream)
        ctx.call = call
        ctx.save_for_backward(q, k, v, out, lse, *(t for t in call.extra if t is not None))
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, _):
        q, k, v, out, lse = ctx.saved_tensors[:5]
        size = 16 // dout.element_size()
        if dout.stride(-1) != 1 or dout.data_ptr() % 16 or any(s % size for s in dout.stride()[:-1]):
            dout = dout.contiguous()
        return (*ctx.call.backward(q, k, v, out, lse, dout), None, None, None, None)


def attend(q, k, v, lr=None, *, scale=None, cap=0.0, slopes=None, at_q=None, at_k=None, weights=None, weights_out=None,
           return_lse=False, stream=None):
    """Attention of queries over rank intervals of the keys.

    q [batch, queries, heads, d]; k, v [batch, keys, kv_heads, d], kv_heads a
    divisor of heads, all float32, float16 or bfloat16, any strides whose rows
    start on 16-byte boundaries, d 32, 64, 96 or 128.  lr: int32
    [batch, queries, 2] or [queries, 2], the interval [l, r] of keys every query
    sees (:func:`rank_bounds` writes such; empty: the output is 0); None: all.
    scale: 1 / sqrt(d) by default.  cap > 0: scores are cap tanh(score / cap).
    slopes [heads] with at_q [batch, queries] and at_k [batch, keys] or
    [batch, kv_heads, keys], float32: scores fall by slope |at_q - at_k|.
    weights: float32 [batch, kv_heads, keys]; the call then also returns these
    plus the weight each key received, summed over queries and the group's
    heads, in a new tensor or in weights_out (may be ``weights``).

    Returns out [batch, queries, heads, d], followed by lse [batch, heads,
    queries] (return_lse) and the new weights (weights given).  q, k and v
    take gradients; lse and weights do not."""
    call = _Call(q, k, v, lr, scale, cap, slopes, at_q, at_k)
    b, tq, h, d, tk = call.shape
    if weights is not None:
        _tensor("weights", weights, torch.float32, (b, call.kv, tk), call.dev)
        _tensor("weights_out", weights_out, torch.float32, (b, call.kv, tk), call.dev)
        if weights_out is None:
            weights_out = torch.empty_like(weights)
    else:
        _need(weights_out is None, "weights_out needs weights")
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        out, lse = _Attend.apply(q, k, v, call, weights, weights_out, stream)
    else:
        out, lse = call.forward(q, k, v, return_lse, weights, weights_out, stream)
    if not return_lse and weights is None:
        return out
    return (out,) + ((lse,) if return_lse else ()) + ((weights_out,) if weights is not None else ())


def attend_shared(q, k, v, k_pages, v_pages, pages, lengths, *, lr=None, scale=None, cap=0.0, slopes=None, return_lse=False,
                  stream=None):
    """One query token per request over a prefix shared by all, then its own
    tail.  q [batch, heads, d]; k, v [prefix, kv_heads, d]; k_pages, v_pages
    [num_pages, page, kv_heads, d]; pages int32 [batch, pages_per_request]: the
    pages of every request's tail in order; lengths int32 [batch]: the tails'
    rows.  lr int32 [batch, 2]: the interval of the prefix a request sees
    (None: all).  slopes [heads]: scores fall with the distance of the query,
    which stands on the last row of its tail.  Returns out [batch, heads, d],
    and lse [batch, heads] with return_lse."""
    _start(q)
    dev = q.device
    for name, t, dims in (("q", q, 3), ("k", k, 3), ("v", v, 3), ("k_pages", k_pages, 4), ("v_pages", v_pages, 4)):
        _values(name, t, q.dtype, dims, dev)
    b, h, d = q.shape
    tk, kv = k.shape[:2]
    _need(k.shape == (tk, kv, d) and v.shape == k.shape and k_pages.shape[2:] == (kv, d) and v_pages.shape == k_pages.shape,
          f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}, pages {tuple(k_pages.shape)}, {tuple(v_pages.shape)}: "
          "[batch, heads, d], twice [prefix, kv_heads, d], twice [num_pages, page, kv_heads, d] are wanted")
    _need(pages.dim() == 2, "pages: [batch, pages_per_request] is wanted")
    _tensor("pages", pages, torch.int32, (b, pages.shape[1]), dev)
    _tensor("lengths", lengths, torch.int32, (b,), dev)
    _tensor("lr", lr, torch.int32, (b, 2), dev)
    _tensor("slopes", slopes, torch.float32, (h,), dev)
    out = torch.empty((b, h, d), dtype=q.dtype, device=dev)
    lse = torch.empty((b, h), dtype=torch.float32, device=dev) if return_lse else None
    a = SharedArgs()
    for name, t in (("q", q), ("k", k), ("v", v), ("k_pages", k_pages), ("v_pages", v_pages), ("out", out)):
        _put(a, name, t)
    a.pages, a.lengths, a.lr, a.slopes, a.lse = pages.data_ptr(), lengths.data_ptr(), _at(lr), _at(slopes), _at(lse)
    a.batch, a.prefix, a.num_pages, a.pages_per_request, a.page = b, tk, k_pages.shape[0], pages.shape[1], k_pages.shape[1]
    a.heads, a.kv_heads, a.d, a.type = h, kv, d, _TYPES[q.dtype]
    a.scale, a.cap = d ** -0.5 if scale is None else scale, cap
    ws = _workspace(a, lib().frog_attend_shared_workspace(C.byref(a)), dev)
    _launch(lib().frog_attend_shared, a, stream, dev, (q, k, v, k_pages, v_pages, pages, lengths, lr, slopes, out, lse, ws))
    return (out, lse) if return_lse else out


def evict(k, v, weights, positions, lengths, keep, *, recent=0, stream=None):
    """Shorten caches to ``keep`` rows per (sequence, head): the last ``recent``
    and the heaviest of the others (ties: the lower slot), in slot order.
    k, v [batch, slots, heads, d]; weights float32 and positions int32 (None:
    the slots) [batch, heads, slots]; lengths int32 [batch].  Returns new
    (k, v, weights, positions, lengths) with ``keep`` slots; those past a
    length hold 0, 0, 0 and -1."""
    _need(k.is_cuda and k.dtype in _TYPES, f"k is {k.dtype} on {k.device}: float32, float16 or bfloat16 on a GPU is wanted")
    dev = k.device
    _values("k", k, k.dtype, 4, dev)
    _values("v", v, k.dtype, 4, dev)
    _need(v.shape == k.shape, f"k {tuple(k.shape)}, v {tuple(v.shape)}: the same shape is wanted")
    b, t, h, d = k.shape
    _tensor("weights", weights, torch.float32, (b, h, t), dev)
    _tensor("positions", positions, torch.int32, (b, h, t), dev)
    _tensor("lengths", lengths, torch.int32, (b,), dev)
    _need(0 <= recent <= keep <= t, f"recent {recent}, keep {keep}, slots {t}: 0 <= recent <= keep <= slots is wanted")
    k_out, v_out = (torch.empty((b, keep, h, d), dtype=k.dtype, device=dev) for _ in range(2))
    w_out = torch.empty((b, h, keep), dtype=torch.float32, device=dev)
    p_out = torch.empty((b, h, keep), dtype=torch.int32, device=dev)
    n_out = torch.empty((b,), dtype=torch.int32, device=dev)
    a = EvictArgs()
    _put(a, "k", k)
    _put(a, "v", v)
    a.weights, a.positions, a.lengths = weights.data_ptr(), _at(positions), lengths.data_ptr()
    a.k_out, a.v_out, a.weights_out, a.positions_out = k_out.data_ptr(), v_out.data_ptr(), w_out.data_ptr(), p_out.data_ptr()
    a.lengths_out = n_out.data_ptr()
    a.batch, a.slots, a.keep, a.recent, a.heads, a.d, a.type = b, t, keep, recent, h, d, _TYPES[k.dtype]
    ws = _workspace(a, lib().frog_evict_workspace(C.byref(a)), dev)
    _launch(lib().frog_evict, a, stream, dev, (k, v, weights, positions, lengths, k_out, v_out, w_out, p_out, n_out, ws))
    return k_out, v_out, w_out, p_out, n_out

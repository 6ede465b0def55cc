"""Attention over rows kept in attribute order, and the upkeep of the cache
that holds them: Python binding of the attention section of ``include/frog.h``
(the formulas and the limits stand there).  Argument checks and marshalling
only; the gradients go through ``torch.autograd``.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch
from torch.autograd import forward_ad

from . import STORAGE_BF16, STORAGE_F16, STORAGE_F32, _check, lib

_TYPES = {torch.float32: STORAGE_F32, torch.float16: STORAGE_F16, torch.bfloat16: STORAGE_BF16}
_P, _I, _D = C.c_void_p, C.c_int64, C.c_int32


def _rows(name, strides):
    return [(name, _P), (name + "_stride", _I * strides)]


class AttendArgs(C.Structure):
    _fields_ = [*_rows("q", 3), *_rows("k", 3), *_rows("v", 3), *_rows("out", 3), ("lr", _P), ("lr_stride", _I), ("slopes", _P),
                ("at_q", _P), ("at_q_stride", _I), ("at_k", _P), ("at_k_stride", _I * 2), ("lse", _P), ("w_in", _P), ("w_out", _P),
                *_rows("dout", 3), *_rows("dq", 3), *_rows("dk", 3), *_rows("dv", 3), ("ws", _P), ("ws_bytes", _I), ("batch", _I),
                ("queries", _I), ("keys", _I), ("heads", _D), ("kv_heads", _D), ("d", _D), ("type", _D), ("scale", C.c_float),
                ("cap", C.c_float), ("out_low", _P)]


class SharedArgs(C.Structure):
    _fields_ = [*_rows("q", 2), *_rows("k", 2), *_rows("v", 2), *_rows("k_pages", 3), *_rows("v_pages", 3), ("pages", _P),
                ("lengths", _P), ("lr", _P), ("slopes", _P), *_rows("out", 2), ("lse", _P), ("ws", _P), ("ws_bytes", _I),
                ("batch", _I), ("prefix", _I), ("num_pages", _I), ("pages_per_request", _I), ("page", _D), ("heads", _D),
                ("kv_heads", _D), ("d", _D), ("type", _D), ("scale", C.c_float), ("cap", C.c_float)]


class EvictArgs(C.Structure):
    _fields_ = [*_rows("k", 3), *_rows("v", 3), ("weights", _P), ("positions", _P), ("lengths", _P), ("k_out", _P), ("v_out", _P),
                ("weights_out", _P), ("positions_out", _P), ("lengths_out", _P), ("ws", _P), ("ws_bytes", _I), ("batch", _I),
                ("slots", _I), ("keep", _I), ("recent", _I), ("heads", _D), ("d", _D), ("type", _D)]


def _packer(cls):
    """Writes the values of a struct's fields, arrays spread out, in order."""
    codes = {_P: "P", _I: "q", _D: "i", C.c_float: "f"}
    fmt = "".join(codes[t] if t in codes else codes[t._type_] * t._length_ for _, t in cls._fields_)
    out = struct.Struct("@" + fmt + "0q")
    assert out.size == C.sizeof(cls)
    return out.pack


_pack_attend, _pack_shared, _pack_evict = (_packer(c) for c in (AttendArgs, SharedArgs, EvictArgs))
# the raw handle of the current stream, without the stream object built around it where torch offers that
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _need(ok, text):
    """(where the text is put together from values, the test stands at the call: it costs microseconds)"""
    if not ok:
        raise ValueError(text)


def _plain(name, t, dtype, shape, like):
    """`t` is a contiguous tensor of this type and shape on the device of `like`."""
    if t.dtype != dtype or t.shape != shape or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{name}: {dtype} {tuple(shape)} on {like.device}, contiguous, is wanted, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _values(names, tensors, dims):
    """Tensors of rows: of one supported type, on one GPU, their last axes without gaps."""
    first = tensors[0]
    dtype, device = first.dtype, first.get_device()
    kind = _TYPES.get(dtype)
    if device < 0 or kind is None:
        raise ValueError(f"{names[0]} is {dtype} on {first.device}: float32, float16 or bfloat16 on a GPU is wanted")
    for name, t, n in zip(names, tensors, dims):
        if t.dtype != dtype or t.get_device() != device or t.dim() != n:
            raise ValueError(f"{name}: {n} axes of {dtype} on {first.device} are wanted, not {t.dim()} of {t.dtype} on {t.device}")
        if t.stride(-1) != 1 and t.shape[-1] > 1:
            raise ValueError(f"{name}: the last axis must have stride 1")
    return kind


def _launch(fn, args, device):
    """Enqueue on the device's current stream."""
    index = device.index
    if _device() == index:
        rc = fn(args, _current(index))
    else:
        with torch.cuda.device(index):
            rc = fn(args, _current(index))
    if rc:
        _check(rc)


def _on(stream, call, inputs):
    """The tensors `call()` returns, with its work enqueued on `stream` (None: the current one of the inputs' device).  On
    another stream than the current one the call allocates from that stream's memory, which no earlier work of the current
    stream may still use; and inputs and outputs are kept until both streams are done with them."""
    if stream is None:
        return call()
    device = inputs[0].device
    _need(stream.device == device, f"the stream is not on {device}")
    here = torch.cuda.current_stream(device)
    if stream == here:
        return call()
    with torch.cuda.stream(stream):
        outs = call()
    for t in inputs:
        if t is not None:
            t.record_stream(stream)
    for t in outs:
        if t is not None:
            t.record_stream(here)
    return outs


def _no_tangent(names, tensors):
    """No derivative of forward mode enters a kernel: it would be left out of the result."""
    if getattr(forward_ad, "_current_level", 0) < 0:      # (outside dual levels, without a look at the tensors)
        return
    for name, t in zip(names, tensors):
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{name} carries a tangent: forward-mode derivatives are not supported")


def _no_gradient(names, tensors):
    _no_tangent(names, tensors)
    if torch.is_grad_enabled():
        for name, t in zip(names, tensors):
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} takes no gradient: detach it, or call under torch.no_grad()")


def _own_workspace(large):
    """Whether a call takes its workspace from torch rather than the library's buffer of the stream: a captured graph has to
    keep it, and the library would keep a large one for good."""
    return large or torch.cuda.is_current_stream_capturing()


def _workspace(query, args, device):
    n = query(args)
    if n < 0:
        _check(n)
    ws = torch.empty(n, dtype=torch.uint8, device=device) if n else None
    return ws, (ws.data_ptr(), n) if n else (0, 0)


_NONE4 = (0, 0, 0, 0)
_NO_GRADS = _NONE4 * 4


class _Call:
    """The checked arguments of one attention call, apart from its outputs."""

    __slots__ = ("device", "shape", "rows", "masks", "tail")

    def __init__(self, q, k, v, lr, scale, cap, slopes, at_q, at_k):
        kind = _values(("q", "k", "v"), (q, k, v), (4, 4, 4))
        _no_gradient(("slopes", "at_q", "at_k"), (slopes, at_q, at_k))
        b, tq, h, d = q.shape
        _, tk, kv, _ = ks = k.shape
        if ks != (b, tk, kv, d) or v.shape != ks:
            raise ValueError(f"q {tuple(q.shape)}, k {tuple(ks)}, v {tuple(v.shape)}: [batch, queries, heads, d] and twice "
                             "[batch, keys, kv_heads, d] are wanted")
        self.device, self.shape = q.device, (b, tq, h, d, tk, kv)
        self.rows = (q.data_ptr(), *q.stride()[:3], k.data_ptr(), *k.stride()[:3], v.data_ptr(), *v.stride()[:3])
        lrs = (0, 0)
        if lr is not None:
            one = lr.dim() == 2
            lrs = (_plain("lr", lr, torch.int32, (tq, 2) if one else (b, tq, 2), q), 0 if one else 2 * tq)
        bias = (0, 0, 0, 0, 0, 0)
        if slopes is not None:
            _need(at_q is not None and at_k is not None, "slopes, at_q and at_k go together")
            f, one = torch.float32, at_k.dim() == 2
            bias = (_plain("slopes", slopes, f, (h,), q), _plain("at_q", at_q, f, (b, tq), q), tq,
                    _plain("at_k", at_k, f, (b, tk) if one else (b, kv, tk), q), tk if one else kv * tk, 0 if one else tk)
        else:
            _need(at_q is None and at_k is None, "slopes, at_q and at_k go together")
        self.masks = lrs + bias
        self.tail = (b, tq, tk, h, kv, d, kind, d ** -0.5 if scale is None else scale, cap)

    def forward(self, q, want_lse, w_in, w_out, want_low=False):
        b, tq, h, d, tk, kv = self.shape
        out = torch.empty((b, tq, h, d), dtype=q.dtype, device=self.device)
        low = torch.empty_like(out) if want_low else None
        lse = torch.empty((b, h, tq), dtype=torch.float32, device=self.device) if want_lse else None
        head = (*self.rows, out.data_ptr(), tq * h * d, h * d, d, *self.masks, 0 if lse is None else lse.data_ptr(),
                0 if w_in is None else w_in.data_ptr(), 0 if w_out is None else w_out.data_ptr(), *_NO_GRADS)
        tail = (*self.tail, 0 if low is None else low.data_ptr())
        args, ws, L = _pack_attend(*head, 0, 0, *tail), None, lib()
        if _own_workspace(w_out is not None and max(q.numel() // d, kv * 64) * tk > 2 ** 22):
            ws, at = _workspace(lambda x: L.frog_attend_workspace(x, 0), args, self.device)
            args = _pack_attend(*head, *at, *tail)
        _launch(L.frog_attend, args, self.device)
        return out, lse, low

    def backward(self, q, k, v, out, low, lse, dout):
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=self.device) for t in (q, k, v))
        grads = (x for t in (dout, dq, dk, dv) for x in (t.data_ptr(), *t.stride()[:3]))
        head = (*self.rows, out.data_ptr(), *out.stride()[:3], *self.masks, lse.data_ptr(), 0, 0, *grads)
        tail = (*self.tail, 0 if low is None else low.data_ptr())
        args, ws, L = _pack_attend(*head, 0, 0, *tail), None, lib()
        n = L.frog_attend_workspace(args, 1)
        if _own_workspace(n > 2 ** 26):
            ws, at = _workspace(lambda x: n, args, self.device)
            args = _pack_attend(*head, *at, *tail)
        _launch(L.frog_attend_backward, args, self.device)
        return dq, dk, dv


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, call, mask, w_in, w_out, kept):
        # (16-bit rows: the gradient takes the output with what its rounding left)
        out, lse, low = call.forward(q, True, w_in, w_out, q.element_size() == 2)
        kept.append(lse)
        lr, ctx.scale, ctx.cap, *bias = mask
        ctx.save_for_backward(q, k, v, out, low, lse, lr, *bias)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        # (the tensors may have moved since: hooks on saved tensors, recomputation)
        q, k, v, out, low, lse, lr, *bias = ctx.saved_tensors
        _no_tangent(("the gradient of the output",), (dout,))
        size = 16 // dout.element_size()
        if dout.stride(-1) != 1 or dout.data_ptr() % 16 or any(s % size for s in dout.stride()[:-1]):
            # (a copy in new memory: contiguous() returns a tensor that only starts off a boundary as it is)
            dout = dout.clone(memory_format=torch.contiguous_format)
        if low is not None and low.stride() != out.stride():       # (read at the same places)
            out, low = out.contiguous(), low.contiguous()
        call = _Call(q, k, v, lr, ctx.scale, ctx.cap, *bias)
        return (*call.backward(q, k, v, out, low, lse, dout), None, None, None, None, None)


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

    stream: where the work is enqueued (default: the current stream); inputs
    written on another stream have to be waited for there, as for any kernel.

    Returns out [batch, queries, heads, d], followed by lse [batch, heads,
    queries] (return_lse) and the new weights (weights given).  q, k and v
    take gradients; lse and weights do not, and no argument a tangent of
    forward mode (ValueError)."""
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _no_tangent(("q", "k", "v", "slopes", "at_q", "at_k", "weights", "weights_out"), (q, k, v, slopes, at_q, at_k, weights, weights_out))
    mask = (lr, scale, cap, slopes, at_q, at_k)
    call = _Call(q, k, v, *mask)
    if weights is not None:
        b, _, _, _, tk, kv = call.shape
        _plain("weights", weights, torch.float32, (b, kv, tk), q)
        _no_gradient(("weights", "weights_out"), (weights, weights_out))
        if weights_out is not None:
            _plain("weights_out", weights_out, torch.float32, (b, kv, tk), q)
    else:
        _need(weights_out is None, "weights_out needs weights")
    grad = torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad)

    def run():
        new = torch.empty_like(weights) if weights is not None and weights_out is None else weights_out
        if not grad:
            return (*call.forward(q, return_lse, weights, new)[:2], new)
        kept = []
        return _Attend.apply(q, k, v, call, mask, weights, new, kept), kept[0], new

    out, lse, new = _on(stream, run, (q, k, v, lr, slopes, at_q, at_k, weights, weights_out))
    if weights_out is not None and not weights_out.is_inference():
        torch.autograd.graph.increment_version(weights_out)      # (written by address: autograd has to hear of it)
    if not return_lse and weights is None:
        return out
    return (out,) + ((lse,) if return_lse else ()) + ((new,) if weights is not None else ())


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
    _no_gradient(("q", "k", "v", "k_pages", "v_pages", "slopes"), (q, k, v, k_pages, v_pages, slopes))
    kind = _values(("q", "k", "v", "k_pages", "v_pages"), (q, k, v, k_pages, v_pages), (3, 3, 3, 4, 4))
    b, h, d = q.shape
    tk, kv, _ = k.shape
    num, page, _, _ = k_pages.shape
    if k.shape != (tk, kv, d) or v.shape != k.shape or k_pages.shape != (num, page, kv, d) or v_pages.shape != k_pages.shape:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}, pages {tuple(k_pages.shape)}, {tuple(v_pages.shape)}: "
                         "[batch, heads, d], twice [prefix, kv_heads, d], twice [num_pages, page, kv_heads, d] are wanted")
    _need(pages.dim() == 2, "pages: [batch, pages_per_request] is wanted")
    outs = _on(stream, lambda: _attend_shared(kind, q, k, v, k_pages, v_pages, pages, lengths, lr, scale, cap, slopes, return_lse),
               (q, k, v, k_pages, v_pages, pages, lengths, lr, slopes))
    return outs if return_lse else outs[0]


def _attend_shared(kind, q, k, v, k_pages, v_pages, pages, lengths, lr, scale, cap, slopes, return_lse):
    b, h, d = q.shape
    tk, kv, _ = k.shape
    num, page, _, _ = k_pages.shape
    width, device = pages.shape[1], q.device
    out = torch.empty((b, h, d), dtype=q.dtype, device=device)
    lse = torch.empty((b, h), dtype=torch.float32, device=device) if return_lse else None
    head = (q.data_ptr(), *q.stride()[:2], k.data_ptr(), *k.stride()[:2], v.data_ptr(), *v.stride()[:2], k_pages.data_ptr(),
            *k_pages.stride()[:3], v_pages.data_ptr(), *v_pages.stride()[:3], _plain("pages", pages, torch.int32, (b, width), q),
            _plain("lengths", lengths, torch.int32, (b,), q), 0 if lr is None else _plain("lr", lr, torch.int32, (b, 2), q),
            0 if slopes is None else _plain("slopes", slopes, torch.float32, (h,), q), out.data_ptr(), h * d, d,
            0 if lse is None else lse.data_ptr())
    tail = (b, tk, num, width, page, h, kv, d, kind, d ** -0.5 if scale is None else scale, cap)
    args, ws, L = _pack_shared(*head, 0, 0, *tail), None, lib()
    if _own_workspace(q.numel() > 2 ** 22):
        ws, at = _workspace(L.frog_attend_shared_workspace, args, device)
        args = _pack_shared(*head, *at, *tail)
    _launch(L.frog_attend_shared, args, device)
    return out, lse


def evict(k, v, weights, positions, lengths, keep, *, recent=0, stream=None):
    """Shorten caches to ``keep`` rows per (sequence, head): the last ``recent``
    and the heaviest of the others (ties: the lower slot), in slot order.
    k, v [batch, slots, heads, d]; weights float32 and positions int32 (None:
    the slots) [batch, heads, slots]; lengths int32 [batch].  Returns new
    (k, v, weights, positions, lengths) with ``keep`` slots; those past a
    length hold 0, 0, 0 and -1."""
    _no_gradient(("k", "v", "weights"), (k, v, weights))
    kind = _values(("k", "v"), (k, v), (4, 4))
    b, t, h, d = k.shape
    if v.shape != k.shape or not 0 <= recent <= keep <= t:
        raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}, recent {recent}, keep {keep}: the same shape and "
                         "0 <= recent <= keep <= slots are wanted")
    return _on(stream, lambda: _evict(kind, k, v, weights, positions, lengths, keep, recent), (k, v, weights, positions, lengths))


def _evict(kind, k, v, weights, positions, lengths, keep, recent):
    b, t, h, d = k.shape
    device = k.device
    k_out, v_out = (torch.empty((b, keep, h, d), dtype=k.dtype, device=device) for _ in range(2))
    w_out = torch.empty((b, h, keep), dtype=torch.float32, device=device)
    p_out = torch.empty((b, h, keep), dtype=torch.int32, device=device)
    n_out = torch.empty((b,), dtype=torch.int32, device=device)
    head = (k.data_ptr(), *k.stride()[:3], v.data_ptr(), *v.stride()[:3], _plain("weights", weights, torch.float32, (b, h, t), k),
            0 if positions is None else _plain("positions", positions, torch.int32, (b, h, t), k),
            _plain("lengths", lengths, torch.int32, (b,), k), k_out.data_ptr(), v_out.data_ptr(), w_out.data_ptr(), p_out.data_ptr(),
            n_out.data_ptr())
    tail = (b, t, keep, recent, h, d, kind)
    args, ws, L = _pack_evict(*head, 0, 0, *tail), None, lib()
    if _own_workspace(b * h * keep > 2 ** 22):
        ws, at = _workspace(L.frog_evict_workspace, args, device)
        args = _pack_evict(*head, *at, *tail)
    _launch(L.frog_evict, args, device)
    return k_out, v_out, w_out, p_out, n_out

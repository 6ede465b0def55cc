"""The attention operators in 64 bits, and how far a computation in 32 bits
with factors rounded to the rows' type may be from them.

Error bounds (u: half a unit in the last place of the type; e = 2^-24):
a score's error is that of a sum of d products, of the cap (its tanh is
computed to a few e, times the cap) and of the bias:
  es = scale (d + 2) e sum|q k| + 8 e cap + 4 e (|z| + |slope (aq - ak)|)
so a weight is off by the factor 2 max(es) (its own error and its sum's) plus
n e for the sum, and u where it is rounded; sums of n products add n e of the
sum of magnitudes; an output is rounded once more."""
import math

import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}
TINY = {torch.float32: 1e-36, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-36}   # below it a value of the type is lost
E = 2.0 ** -24


class Attention:
    """Forward and gradients of one call, in float64, with error bounds."""

    def __init__(self, q, k, v, lr=None, scale=None, cap=0.0, slopes=None, at_q=None, at_k=None, dout=None):
        self.type = q.dtype
        dev = q.device
        b, tq, h, d = q.shape
        tk, kv = k.shape[1:3]
        g = h // kv
        scale = d ** -0.5 if scale is None else scale
        place = torch.arange(tk, device=dev)
        if lr is None:
            lr = torch.tensor([0, tk - 1], device=dev, dtype=torch.int32).expand(tq, 2)
        lr = lr.expand(b, tq, 2).long()
        seen = ((place >= lr[..., :1]) & (place <= lr[..., 1:])).unsqueeze(1)          # [b, 1, tq, tk]
        used = seen.any(2).view(b, tk, 1, 1)                                           # rows some interval meets
        Q = q.double().transpose(1, 2)
        K, V = (torch.where(used, x.double(), 0).transpose(1, 2).repeat_interleave(g, 1) for x in (k, v))
        x = Q @ K.transpose(2, 3) * scale
        mag = Q.abs() @ K.abs().transpose(2, 3) * abs(scale)
        t = torch.tanh(x / cap) if cap else None
        z = cap * t if cap else x
        bias = torch.zeros_like(z)
        if slopes is not None:
            ak = at_k.double()
            ak = (ak.unsqueeze(1).expand(b, kv, tk) if ak.dim() == 2 else ak).repeat_interleave(g, 1)
            bias = slopes.double().view(1, h, 1, 1) * (at_q.double().view(b, 1, tq, 1) - ak.unsqueeze(2)).abs()
        z = z - bias
        es = (d + 2) * E * mag + 8 * E * cap + 4 * E * (z.abs() + bias)
        es = torch.where(seen, es, 0).amax(-1, keepdim=True) if tk else es.new_zeros((b, h, tq, 1))
        z = z.masked_fill(~seen, -math.inf)
        some = seen.any(-1, keepdim=True)
        top = torch.where(some, z.amax(-1, keepdim=True), 0.0) if tk else es
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        p = torch.where(some, p / total.clamp(min=1e-300), 0.0)
        u, n = U[self.type], tk
        o = p @ V
        ep = 2 * es + (n + 8) * E                      # relative error of a weight before it is rounded
        self.out = o.transpose(1, 2)
        self.out_err = ((ep + u + n * E) * (p @ V.abs()) * 1.05 + u * o.abs() + TINY[self.type] * (1 + V.abs().sum(2, keepdim=True))).transpose(1, 2)
        self.lse = torch.where(some, top + torch.log(total.clamp(min=1e-300)), -math.inf).squeeze(-1)
        self.lse_err = (es + (n + 8) * E + 4 * E * self.lse.abs().nan_to_num(0, 0, 0).unsqueeze(-1)).squeeze(-1).expand_as(self.lse)
        self.weights = p.view(b, kv, g * tq, tk).sum(2)
        self.weights_err = ((ep + (tq * g + 8) * E) * p).view(b, kv, g * tq, tk).sum(2)
        if dout is None:
            return
        G = torch.where(some, dout.double().transpose(1, 2), 0.0)
        dp = G @ V.transpose(2, 3)
        delta = (G * o).sum(-1, keepdim=True)
        dt = (1 - t * t) if cap else torch.ones_like(x)
        dx = p * (dp - delta) * dt
        # dp: a sum of d products; delta: the same, from the rounded output
        part = (d + 2) * E * (G.abs() @ V.abs().transpose(2, 3)) + (G.abs() * (self.out_err.transpose(1, 2) + (d + 2) * E * o.abs())).sum(-1, keepdim=True)
        et = 4 * es / cap + 1e-6 if cap else 0.0       # 1 - tanh^2 = 4 r (1 - r)
        # u |dx| + TINY: dx is rounded to the type as a factor of the next product
        edx = (p * dt * part + (ep + et + 4 * E) * dx.abs()) * 1.05 + u * dx.abs() + TINY[self.type]
        edx = torch.where(seen, edx, 0.0)
        a = abs(scale)
        dq, dk, dv = dx @ K * scale, dx.transpose(2, 3) @ Q * scale, p.transpose(2, 3) @ G

        def fold(y):
            return y.view(b, kv, g, tk, d).sum(2).transpose(1, 2)

        self.dq = dq.transpose(1, 2)
        self.dq_err = ((edx + (tk + 2) * E * dx.abs()) @ K.abs() * a + u * dq.abs() + TINY[self.type]).transpose(1, 2)
        rows = tq * g + 2
        self.dk, self.dv = fold(dk), fold(dv)
        self.dk_err = fold((edx + rows * E * dx.abs()).transpose(2, 3) @ Q.abs() * a) + u * self.dk.abs() + TINY[self.type]
        ev = torch.where(seen, (ep + u + rows * E) * p * 1.05 + TINY[self.type], 0.0)
        self.dv_err = fold(ev.transpose(2, 3) @ G.abs()) + u * self.dv.abs() + TINY[self.type]


def near(got, want, err, what=""):
    """Every element within its own bound; infinities equal."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(got[~fin], want[~fin]), what
    off = (got - want).abs()[fin]
    bad = ~(off <= err.expand_as(want)[fin])
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / err.expand_as(want)[fin].clamp(min=1e-300)).nan_to_num(math.inf).max()):.3g} of its bound"


def intervals(kind, b, tq, tk, seed=0):
    """int32 [b, tq, 2] intervals of a mask, some outside [0, tk) where it is "wild"."""
    g = torch.Generator().manual_seed(seed)
    i = torch.arange(tq).expand(b, tq)
    at = i + tk - tq
    if kind == "causal":
        lo, hi = torch.zeros_like(i), at
    elif kind == "window":
        lo, hi = (at - 5).clamp(min=0), at
    elif kind == "prefix":
        lo, hi = torch.zeros_like(i), at.clamp(min=tk // 3)
    elif kind == "documents":
        cut = torch.sort(torch.randint(0, tk + 1, (b, 3), generator=g), -1)[0]
        start = (at.unsqueeze(-1) >= cut.unsqueeze(1)).long() * cut.unsqueeze(1)
        lo, hi = start.amax(-1), at
    elif kind == "lengths":
        n = torch.randint(0, tk + 1, (b, 1), generator=g)
        lo, hi = torch.zeros_like(i), (n - tq + i)
    elif kind == "wild":
        lo = torch.randint(-tk, tk + 3, (b, tq), generator=g)
        hi = lo + torch.randint(-3, tk + 3, (b, tq), generator=g)
    elif kind == "empty":
        lo, hi = torch.ones_like(i), torch.zeros_like(i)
    else:
        return None
    return torch.stack([lo, hi], -1).to(torch.int32).contiguous()


def select(weights, length, keep, recent):
    """Slots kept of one cache: the newest, and of the others the heaviest (ties: the lowest slot; NaN last)."""
    recent = min(recent, length)
    old = [(-w if w == w else math.inf, w != w, i) for i, w in enumerate(weights[: length - recent])]
    first = [i for _, _, i in sorted(old)[: max(0, min(keep - recent, len(old)))]]
    return sorted(first) + list(range(length - recent, length))

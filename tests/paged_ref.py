"""A cache in 8-bit pages in 64 bits and plain Python: quantisation, appending,
reading back, the choice of pages, and attention with error bounds."""
import math

import torch

LIMIT = {"e4m3": 448.0, "int8": 127.0}
U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}
TINY = {torch.float32: 1e-36, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-36}
E = 2.0 ** -24


def quantise(x, store):
    """Codes (float64) and power bytes (int64) of rows in float64, from the definition."""
    a = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    a = torch.where(fine, a, 1.0)
    e = torch.full(a.shape, -100, dtype=torch.int64)
    for i, v in enumerate(a.flatten().tolist()):
        n = -100
        while v > LIMIT[store] * 2.0 ** n:
            n += 1
        e.view(-1)[i] = n
    y = torch.where(fine.unsqueeze(-1), x, 0.0) * torch.exp2(-e.double()).unsqueeze(-1)
    if store == "e4m3":
        # the nearest of all codes, ties to the even one
        unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        codes = torch.round(y / unit) * unit
    else:
        codes = torch.round(y)
    return codes, torch.where(fine, e + 127, 255)


class Cache:
    """The same arrays on the host, values as float64."""

    def __init__(self, cache):
        self.store = "int8" if cache.k.dtype == torch.int8 else "e4m3"
        self.pages, self.kv, self.page, self.d = cache.shape
        self.codes = {x: getattr(cache, x).cpu().to(torch.float32).double() for x in ("k", "v")}
        self.exps = {x: getattr(cache, x + "_exp").cpu().long() for x in ("k", "v")}
        self.bounds = None if cache.bounds is None else cache.bounds.cpu().double()

    def value(self, x, page, h, row):
        if int(self.exps[x][page, h, row]) == 255:
            return torch.full((self.d,), math.nan, dtype=torch.float64)
        return self.codes[x][page, h, row] * 2.0 ** (int(self.exps[x][page, h, row]) - 127)

    def values(self, x, page):
        """[kv_heads, page, d]"""
        e = self.exps[x][page]
        y = self.codes[x][page] * torch.exp2(e.double() - 127).unsqueeze(-1)
        return torch.where((e == 255).unsqueeze(-1), math.nan, y)

    def write(self, k, v, pages, lengths, starts=None):
        k, v = k.cpu().double(), v.cpu().double()
        b, width = pages.shape
        starts = [i * (k.shape[0] // b) for i in range(b + 1)] if starts is None else starts.tolist()
        q = {"k": quantise(k, self.store), "v": quantise(v, self.store)}
        for i in range(b):
            count = starts[i + 1] - starts[i]
            met = {}
            for t in range(count):
                at = int(lengths[i]) - count + t
                if at < 0 or at >= width * self.page:
                    continue
                p = int(pages[i, at // self.page])
                if not 0 <= p < self.pages:
                    continue
                for x in ("k", "v"):
                    self.codes[x][p, :, at % self.page] = q[x][0][starts[i] + t]
                    self.exps[x][p, :, at % self.page] = q[x][1][starts[i] + t]
                met.setdefault(p, []).append(at % self.page)
            if self.bounds is not None:
                for p, rows in met.items():
                    y = self.values("k", p)[:, rows]                    # [kv_heads, rows, d]
                    low, high = y.amin(1), y.amax(1)                   # (NaN where a row is)
                    if rows[0]:
                        low, high = torch.minimum(low, self.bounds[p, :, 0]), torch.maximum(high, self.bounds[p, :, 1])
                    # (held in bfloat16, which has every value but 64 2^122, the one above the range of 32 bits)
                    self.bounds[p] = torch.stack([low, high], 1).to(torch.bfloat16).double()

    def same(self, cache):
        """Whether the GPU's arrays hold exactly this."""
        other = Cache(cache)
        for x in ("k", "v"):
            assert torch.equal(other.exps[x], self.exps[x]), f"powers of {x}"
            assert torch.equal(other.codes[x], self.codes[x]), f"codes of {x}"
        if self.bounds is not None:
            assert torch.equal(torch.isnan(other.bounds), torch.isnan(self.bounds)), "bounds that are not a number"
            assert torch.equal(other.bounds.nan_to_num(0.0), self.bounds.nan_to_num(0.0)), "bounds"

    def rows(self, x, pages, h, numbers):
        """Values [rows, d] of pages `numbers` of one request, and their places; pages that are none have none."""
        got, place = [], []
        for n in numbers:
            if not 0 <= n < len(pages) or not 0 <= int(pages[n]) < self.pages:
                continue
            got.append(self.values(x, int(pages[n]))[h])
            place.append(n * self.page + torch.arange(self.page))
        if not got:
            return torch.zeros((0, self.d), dtype=torch.float64), torch.zeros((0,), dtype=torch.long)
        return torch.cat(got), torch.cat(place)

    def read(self, pages, lengths, slots, dtype):
        b = pages.shape[0]
        out = [torch.zeros((b, slots, self.kv, self.d), dtype=torch.float64) for _ in range(2)]
        for i in range(b):
            for t in range(min(slots, int(lengths[i]), pages.shape[1] * self.page)):
                p = int(pages[i, t // self.page])
                if 0 <= p < self.pages:
                    for y, x in zip(out, ("k", "v")):
                        y[i, t] = self.values(x, p)[:, t % self.page]
        return [y.to(dtype) for y in out]

    def select(self, q, pages, lengths, keep, first, recent):
        b, h, _ = q.shape
        q = q.cpu().double()
        out = torch.full((b, self.kv, keep), -1, dtype=torch.int32)
        for i in range(b):
            n = -(-max(0, min(int(lengths[i]), pages.shape[1] * self.page)) // self.page)
            at = pages[i, :n].long()
            none = (at < 0) | (at >= self.pages)
            for j in range(self.kv):
                heads = q[i, j * (h // self.kv):(j + 1) * (h // self.kv)]
                # (sums of 64-bit products: their order moves a score rounded to 32 bits in one of 2^28)
                low, high = self.bounds[at.clamp(0, self.pages - 1), j].unbind(1)
                scores = (heads.clamp(min=0).sum(0) * high + heads.clamp(max=0).sum(0) * low).sum(-1).float().tolist()
                rank = []
                for p, s in enumerate(scores):
                    if p < first or p >= n - recent:
                        key = (-2, 0.0)
                    elif none[p]:
                        key = (2, 0.0)
                    else:
                        key = (-1, 0.0) if s != s else (0, -s)
                    rank.append((*key, p))
                kept = sorted(p for _, _, p in sorted(rank)[:keep])
                out[i, j, :len(kept)] = torch.tensor(kept, dtype=torch.int32)
        return out

    def attend(self, q, pages, lengths, chosen=None, lr=None, scale=None, cap=0.0, slopes=None):
        """out, its bound, lse, its bound.

        A score's error (e = 2^-24): sums of up to 3 d products, the product with the power (exact), with the scale, the
        cap (its tanh to a few e) and the bias; a weight is off by twice the largest of these, its sum's rounding, and
        2^-16 (16-bit queries: two bf16 factors, each rounded by 2^-8) or 2^-24 (three); the output is rounded once."""
        b, h, d = q.shape
        kind, group = q.dtype, h // self.kv
        scale = d ** -0.5 if scale is None else scale
        out, err = torch.zeros((b, h, d), dtype=torch.float64), torch.zeros((b, h, d), dtype=torch.float64)
        lse, lerr = torch.full((b, h), -math.inf, dtype=torch.float64), torch.zeros((b, h), dtype=torch.float64)
        q = q.cpu().double()
        part = 2.0 ** -24 if kind == torch.float32 else 2.0 ** -16
        for i in range(b):
            n = max(0, min(int(lengths[i]), pages.shape[1] * self.page))
            lo, hi = (0, n - 1) if lr is None else (max(0, int(lr[i, 0])), min(n - 1, int(lr[i, 1])))
            for j in range(self.kv):
                numbers = range(-(-n // self.page)) if chosen is None else chosen[i, j].tolist()
                K, place = self.rows("k", pages[i], j, numbers)
                V, _ = self.rows("v", pages[i], j, numbers)
                seen = (place >= lo) & (place <= hi)
                K, V, place = K[seen], V[seen], place[seen]
                m = len(place)
                if not m:
                    continue
                for g in range(j * group, (j + 1) * group):
                    x, mag = K @ q[i, g] * scale, K.abs() @ q[i, g].abs() * abs(scale)
                    z = cap * torch.tanh(x / cap) if cap else x
                    bias = float(slopes[g]) * (n - 1 - place).abs().double() if slopes is not None else torch.zeros_like(z)
                    z = z - bias
                    es = float(((3 * d + 6) * E * mag + 8 * E * cap + 4 * E * (z.abs() + bias)).max())
                    s = torch.logsumexp(z, 0)
                    p = torch.exp(z - s)
                    out[i, g] = p @ V
                    weight = 2 * es + (m + 8) * E + part + 3 * m * E
                    err[i, g] = weight * (p @ V.abs()) * 1.05 + U[kind] * out[i, g].abs() + TINY[kind]
                    lse[i, g] = s
                    lerr[i, g] = es + (m + 8) * E + 4 * E * s.abs()
        return out, err, lse, lerr

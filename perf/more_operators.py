"""Cases of the operators around a cache of keys and values in 8-bit pages:
writing rows into it (quantised, with the least and the largest key of every
page), reading them back, attention of one new token per request over it, and
the choice of the pages a token has to look at.

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same
ranges, ``prepare`` makes from a seed what a program has in hand before the
call, ``run`` is one pass (the plain form in elementary 32-bit operations, or,
where ``own`` is true, the library's calls), ``exact`` the result in 64 bits
and ``work`` the bytes and operations no implementation can do without.

A case is a dict of plain values:

  op       "write", "read", "select" or "attend"
  type     "bf16", "fp16" or "fp32": queries, and rows before and after the cache
  store    "e4m3" or "int8": a row is 8-bit codes times one power of two
  batch    requests, of lengths spread up to
  tokens   rows of the longest one (one of eight or more requests is empty)
  new      "write": rows the longest request adds (the others in proportion)
  heads, kv_heads, d
  page     rows of a page
  keep     "select": pages chosen for each kv head, the first and the newest
           among them; "attend": pages chosen (0: every row is seen)
  cap      scores are cap tanh(score / cap), 0: not capped
  bias     scores fall with the distance, a slope per head
  window   "attend": the newest rows a token sees, 0: all
"""
import math

import torch

own = False

_KEYS = ("op", "type", "store", "batch", "tokens", "new", "heads", "kv_heads", "d", "page", "keep", "cap", "bias", "window")
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_LIMIT = {"e4m3": 448.0, "int8": 127.0}
_LEAST = -100                                # least exponent of a row


def _case(name=None, **kw):
    c = dict(op="attend", type="bf16", store="e4m3", batch=1, tokens=1000, new=0, heads=8, kv_heads=8, d=128, page=64, keep=0, cap=0.0,
             bias=False, window=0)
    c.update(kw)
    assert set(c) == set(_KEYS)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new row of every conversation of a batch, as each step of decoding adds it: latency
        _case("new_rows", op="write", batch=32, tokens=2000, new=1, heads=32),
        # prompts of many lengths that arrive together
        _case("prompts", op="write", batch=12, tokens=16_000, new=16_000, heads=32),
        # pieces of prompts in single precision, behind what their requests hold, rows of an odd width
        _case("pieces", op="write", type="fp32", store="int8", batch=5, tokens=2100, new=701, heads=3, kv_heads=3, d=96, page=16),
        # two short conversations read back: latency
        _case("read_short", op="read", type="fp16", store="int8", batch=2, tokens=300, heads=2, kv_heads=2, d=64, page=16),
        # long conversations read back for the next piece of their prompts
        _case("read_long", op="read", batch=4, tokens=50_000, heads=32),
        # the pages one token of one long conversation looks at: latency
        _case("select_one", op="select", tokens=20_001, heads=32, keep=32),
        # the same for many long conversations
        _case("select_many", op="select", batch=48, tokens=60_000, heads=32, page=32, keep=128),
        # one token of one conversation of a thousand tokens: latency
        _case("one_more", tokens=1001, heads=16, kv_heads=4),
        # the next token of many conversations of all lengths
        _case("many_more", batch=32, tokens=40_000, heads=32),
        # every head with keys of its own, capped scores
        _case("own_keys", type="fp16", store="int8", batch=24, tokens=5000, heads=12, kv_heads=12, d=64, page=32, cap=30.0),
        # the next token of many long conversations, over chosen pages alone
        _case("chosen_pages", store="int8", batch=48, tokens=60_000, heads=32, keep=64),
        # a small model in single precision, nearer tokens preferred, a window
        _case("near_rows", type="fp32", store="int8", batch=3, tokens=777, heads=8, kv_heads=2, d=32, page=16, bias=True, window=256),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(("write", "write", "read", "select", "select", "attend", "attend", "attend", "attend"))
    kv = rng.choice((1, 2, 3, 4, 8, 12))
    heads = kv * rng.choice((1, 2, 4, 7, 8, 16, 24))
    c = dict(op=op, type=rng.choice(("bf16", "bf16", "fp16", "fp32")), store=rng.choice(("e4m3", "int8")), heads=heads, kv_heads=kv,
             d=rng.choice((32, 64, 96, 128, 128)), page=rng.choice((16, 32, 64, 64, 128, 256)))
    # (of fewer pages a selection says little)
    tokens = _log(rng, 32 * c["page"] if op == "select" else 1, 60_000)
    # values of a cache's keys, which a pass over it walks
    most = 50_000_000 if op in ("write", "read") else 500_000_000
    batch = _log(rng, 1, max(1, min(48, most // (tokens * kv * c["d"]))))
    pages = -(-tokens // c["page"])
    if op == "write":
        new = rng.choice((1, 1, _log(rng, 1, tokens), tokens))
        return _case(**c, batch=batch, tokens=tokens, new=new)
    if op == "select":
        return _case(**c, batch=batch, tokens=tokens, keep=_log(rng, 4, min(pages // 2, 512)))
    if op == "attend":
        c.update(cap=rng.choice((0.0, 0.0, 30.0)), bias=rng.random() < 0.25)
        if rng.random() < 0.35:
            c["keep"] = _log(rng, 1, min(pages, 256))
        elif rng.random() < 0.3:
            c["window"] = _log(rng, 1, tokens)
    return _case(**c, batch=batch, tokens=tokens)


# ------------------------------------------------------------------ structure of a case

def _lengths(case):
    """Rows of every request, spread evenly up to the longest; one of eight or more is empty."""
    b, most = case["batch"], case["tokens"]
    out = [max(1, most * (i + 1) // b) for i in range(b)]
    return [0] + out[1:] if b >= 8 else out


def _added(case):
    """Of these, the rows a "write" adds to every request."""
    return [min(n, max(1, n * case["new"] // case["tokens"])) if n else 0 for n in _lengths(case)]


def _pages_of(rows, page):
    return -(-rows // page)


def _kept(case):
    """Pages chosen of every request."""
    return [min(case["keep"], _pages_of(n, case["page"])) for n in _lengths(case)]


def _seen(case):
    """Rows every request's token sees."""
    out = _lengths(case)
    if case["keep"]:
        # the newest page, which is chosen, holds what the others leave
        p = case["page"]
        out = [min(n, (k - 1) * p + n - (_pages_of(n, p) - 1) * p) if n else 0 for n, k in zip(out, _kept(case))]
    return [min(n, case["window"]) for n in out] if case["window"] else out


def work(case):
    e = 4 if case["type"] == "fp32" else 2
    b, h, kv, d, p = (case[x] for x in ("batch", "heads", "kv_heads", "d", "page"))
    if case["op"] == "write":
        new = sum(_added(case))
        # pages met, whose bounds are written
        met = sum(_pages_of(n, p) - (n - m) // p for n, m in zip(_lengths(case), _added(case)) if m)
        return {"bytes": 2 * new * kv * (d * e + d + 1) + 4 * d * kv * met, "flops": 6 * new * kv * d}
    if case["op"] == "read":
        rows = sum(_lengths(case))
        return {"bytes": 2 * kv * (rows * (d + 1) + b * case["tokens"] * d * e), "flops": 2 * rows * kv * d}
    if case["op"] == "select":
        pages = sum(_pages_of(n, p) for n in _lengths(case))
        return {"bytes": kv * (4 * d * pages + 4 * b * case["keep"]) + b * h * d * e, "flops": 4 * pages * kv * d}
    rows = sum(_seen(case))
    return {"bytes": 2 * rows * kv * (d + 1) + 2 * b * h * d * e, "flops": 4 * rows * h * d}


# ------------------------------------------------------------------ inputs

def _quantise(x, store):
    """The codes of rows (the last axis) and their exponents' bytes."""
    bits = x.abs().amax(-1).view(torch.int32)
    # x = m 2^n with 1 <= m < 2; the limits are 1.75 2^8 and (1 + 63/64) 2^6
    top, part = (8, 0x600000) if store == "e4m3" else (6, 0x7E0000)
    e = ((bits >> 23) - 127 - top + ((bits & 0x7FFFFF) > part).int()).clamp(min=_LEAST)
    y = x * _power(127 - e).unsqueeze(-1)
    return (y if store == "e4m3" else torch.round(y)).to(_CODES[store]), (e + 127).to(torch.uint8)


def _power(byte):
    """2^(byte - 127)"""
    return (byte.int() << 23).view(torch.float32)


def _values(codes, exps):
    return codes.float() * _power(exps).unsqueeze(-1)


def prepare(case, seed):
    g = torch.Generator().manual_seed(int(seed) * 2 + 1)
    dev = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 2)
    b, h, kv, d, page, store = (case[x] for x in ("batch", "heads", "kv_heads", "d", "page", "store"))
    kind = _TYPES[case["type"]]
    order = torch.randperm(b, generator=g).tolist()
    n = [_lengths(case)[i] for i in order]
    used = [_pages_of(x, page) for x in n]
    width, total = max(used), sum(used) + 3

    # what a model's keys are like: a few channels far larger than the others, tokens of unequal norm
    channels = torch.where(torch.rand((kv, d), generator=dev, device="cuda") < 0.04, 6.0, 1.0)

    def rows(*shape):
        x = torch.randn((*shape, kv, d), generator=dev, device="cuda") * channels
        return x * torch.exp(0.4 * torch.randn((*shape, kv, 1), generator=dev, device="cuda"))

    # the requests' pages lie anywhere; entries past a request's own are none
    free = torch.randperm(total, generator=g)
    pages = torch.full((b, width), -1, dtype=torch.int32)
    at = 0
    for i, m in enumerate(used):
        pages[i, :m] = free[at:at + m].to(torch.int32)
        at += m
    cache = {x: torch.empty((total, kv, page, d), dtype=_CODES[store], device="cuda") for x in ("k", "v")}
    cache.update({x + "_exp": torch.empty((total, kv, page), dtype=torch.uint8, device="cuda") for x in ("k", "v")})
    cache["bounds"] = torch.empty((total, kv, 2, d), dtype=torch.bfloat16, device="cuda") if case["op"] in ("write", "select") else None
    step = max(1, 2 ** 28 // (page * kv * d))
    for first in range(0, total, step):
        m = min(total, first + step) - first
        for x in ("k", "v"):
            codes, exps = _quantise(rows(m, page).transpose(1, 2).contiguous(), store)
            cache[x][first:first + m], cache[x + "_exp"][first:first + m] = codes, exps
            if x == "k" and cache["bounds"] is not None:
                y = _values(codes, exps)
                cache["bounds"][first:first + m] = torch.stack([y.amin(2), y.amax(2)], 2).to(torch.bfloat16)
    state = {"case": case, "cache": cache, "pages": pages.cuda(), "lengths": torch.tensor(n, dtype=torch.int32).cuda()}
    if case["op"] == "write":
        new = [_added(case)[i] for i in order]
        starts = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        state.update(k=rows(sum(new)).to(kind), v=rows(sum(new)).to(kind), starts=starts.cuda())
    elif case["op"] in ("select", "attend"):
        state["q"] = (torch.randn((b, h, d), generator=dev, device="cuda") * 1.5).to(kind)
    if case["op"] == "attend":
        state["slopes"] = torch.exp2(-8.0 * torch.arange(1, h + 1, device="cuda") / h) if case["bias"] else None
        state["chosen"] = state["lr"] = None
        if case["keep"]:
            # of the pages of each request some at random and the newest, for every kv head others
            chosen = torch.full((b, kv, case["keep"]), -1, dtype=torch.int32)
            for i, m in enumerate(used):
                k = min(m, case["keep"])
                if k:
                    chosen[i, :, :k] = torch.stack([torch.cat([torch.randperm(m - 1, generator=g)[: k - 1].sort()[0], torch.tensor([m - 1])])
                                                    for _ in range(kv)]).to(torch.int32)
            state["chosen"] = chosen.cuda()
        if case["window"]:
            state["lr"] = torch.stack([(state["lengths"] - case["window"]).clamp(min=0), state["lengths"] - 1], -1)
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    return {"write": _write, "read": _read, "select": _select, "attend": _attend}[case["op"]](case, state)


def _library(s):
    """The library, and the handle of the cache, which a program makes once and keeps."""
    import paper_2608_16491_amd as F
    if "handle" not in s:
        s["handle"] = F.PagedCache(**s["cache"])
    return F, s["handle"]


def _write(case, s):
    c = s["cache"]
    if own:
        F, handle = _library(s)
        F.cache_write(handle, s["k"], s["v"], s["pages"], s["lengths"], starts=s["starts"])
        return c["k"], c["v"], c["k_exp"], c["v_exp"], c["bounds"]
    token = torch.arange(s["k"].shape[0], device="cuda")
    request = torch.searchsorted(s["starts"][1:].contiguous(), token, right=True)
    place = s["lengths"][request] - s["starts"][request + 1] + token
    page, row = s["pages"][request, place // case["page"]].long(), place % case["page"]
    for x in ("k", "v"):
        codes, exps = _quantise(s[x].float(), case["store"])
        c[x].view(torch.uint8)[page, :, row] = codes.view(torch.uint8)
        c[x + "_exp"][page, :, row] = exps
        if x == "k":
            # a page begun anew forgets what it held
            y, bounds = _values(codes, exps), c["bounds"].float()
            begun = torch.zeros(bounds.shape[0] + 1, dtype=torch.bool, device="cuda")
            begun.index_fill_(0, torch.where(row == 0, page, bounds.shape[0]), True)
            bounds[:, :, 0].masked_fill_(begun[:-1].view(-1, 1, 1), math.inf)
            bounds[:, :, 1].masked_fill_(begun[:-1].view(-1, 1, 1), -math.inf)
            at = page.view(-1, 1, 1).expand_as(y)
            least = bounds[:, :, 0].contiguous().scatter_reduce_(0, at, y, "amin")
            most = bounds[:, :, 1].contiguous().scatter_reduce_(0, at, y, "amax")
            c["bounds"].copy_(torch.stack([least, most], 2))
    return c["k"], c["v"], c["k_exp"], c["v_exp"], c["bounds"]


def _read(case, s):
    kind, slots = _TYPES[case["type"]], case["tokens"]
    if own:
        F, handle = _library(s)
        return F.cache_read(handle, s["pages"], s["lengths"], slots, dtype=kind)
    c, at = s["cache"], s["pages"].clamp(min=0).long()
    live = (torch.arange(slots, device="cuda") < s["lengths"].unsqueeze(1)).view(-1, slots, 1, 1)
    out = []
    for x in ("k", "v"):
        y = _values(c[x].view(torch.uint8)[at].view(_CODES[case["store"]]), c[x + "_exp"][at]).to(kind)
        y = y.transpose(2, 3).flatten(1, 2)[:, :slots]                      # [batch, slots, kv_heads, d]
        out.append(torch.where(live, y, 0.0))
    return tuple(out)


def _select(case, s):
    if own:
        F, handle = _library(s)
        return F.select_pages(s["q"], handle, s["pages"], s["lengths"], case["keep"], first=1 if case["keep"] > 1 else 0, recent=1)
    b, h, d = s["q"].shape
    kv, keep = case["kv_heads"], case["keep"]
    # in 64 bits: a score next to the last one kept decides which page is
    q = s["q"].double().view(b, kv, h // kv, d)
    bounds = s["cache"]["bounds"][s["pages"].clamp(min=0).long()].double()   # [batch, width, kv_heads, 2, d]
    score = (bounds[:, :, :, 1] * q.clamp(min=0).sum(2).unsqueeze(1)).sum(-1) + (bounds[:, :, :, 0] * q.clamp(max=0).sum(2).unsqueeze(1)).sum(-1)
    score = score.float().transpose(1, 2)                                   # [batch, kv_heads, width]
    place = torch.arange(score.shape[-1], device="cuda")
    n = ((s["lengths"] + case["page"] - 1) // case["page"]).view(b, 1, 1)
    always = (place >= n - 1) | (place < (1 if keep > 1 else 0))
    score = score.masked_fill(always, math.inf).masked_fill(place >= n, -math.inf)
    kept = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :keep]
    none = score.shape[-1]
    kept = torch.sort(torch.where(torch.arange(keep, device="cuda") < n, kept, none), dim=-1)[0]
    return torch.where(kept < none, kept, -1).to(torch.int32)


def _attend(case, s):
    b, h, d = s["q"].shape
    if own:
        F, handle = _library(s)
        return F.attend_paged(s["q"], handle, s["pages"], s["lengths"], chosen=s["chosen"], lr=s["lr"], cap=case["cap"], slopes=s["slopes"])
    kv, page = case["kv_heads"], case["page"]
    pages, chosen = s["pages"].long(), s["chosen"]
    if chosen is None:
        k, v = (_values(*(s["cache"][x + y].view(torch.uint8)[pages.clamp(min=0)].view(s["cache"][x + y].dtype) for y in ("", "_exp")))
                .transpose(1, 2).flatten(2, 3) for x in ("k", "v"))            # [batch, kv_heads, rows, d]
        place = torch.arange(k.shape[2], device="cuda").view(1, 1, -1)
        held = torch.ones_like(place, dtype=torch.bool)
    else:
        at = pages.unsqueeze(1).expand(b, kv, -1).gather(2, chosen.clamp(min=0).long()).clamp(min=0)
        head = torch.arange(kv, device="cuda").view(1, kv, 1)
        k, v = (_values(*(s["cache"][x + y].view(torch.uint8)[at, head].view(s["cache"][x + y].dtype) for y in ("", "_exp"))).flatten(2, 3)
                for x in ("k", "v"))
        place = (chosen.unsqueeze(-1) * page + torch.arange(page, device="cuda")).flatten(2)
        held = (chosen >= 0).repeat_interleave(page, -1)
    n = s["lengths"].view(b, 1, 1)
    seen = held & (place < n)
    if s["lr"] is not None:
        seen = seen & (place >= s["lr"][:, 0].view(b, 1, 1)) & (place <= s["lr"][:, 1].view(b, 1, 1))
    z = torch.matmul(s["q"].float().view(b, kv, h // kv, d), k.transpose(2, 3)) * d ** -0.5
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    if case["bias"]:
        z = z - s["slopes"].view(1, kv, -1, 1) * (n - 1 - place).abs().unsqueeze(2)
    z = z.masked_fill(~seen.unsqueeze(2), -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-38)
    return torch.matmul(p, v).reshape(b, h, d).to(s["q"].dtype)


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "select":
        return None                      # page numbers: they are equal or not
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["op"]](case, s)


def _rounded64(y, store):
    """To the nearest code, ties to even."""
    if store == "int8":
        return torch.round(y)
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit


def _exact_write(case, s):
    """Request by request and page by page, as the rows come."""
    c = {x: t.double() for x, t in s["cache"].items()}
    page, starts = case["page"], s["starts"].tolist()
    for i, n in enumerate(s["lengths"].tolist()):
        first, last = n - (starts[i + 1] - starts[i]), n
        at = first
        while at < last:
            stop = min(last, (at // page + 1) * page)
            p, r = int(s["pages"][i, at // page]), slice(at % page, at % page + stop - at)
            t = slice(starts[i] + at - first, starts[i] + stop - first)
            for x in ("k", "v"):
                y = s[x][t].double().transpose(0, 1)
                e = torch.ceil(torch.log2((y.abs().amax(-1, keepdim=True) / _LIMIT[case["store"]]).clamp(min=2.0 ** _LEAST)))
                codes = _rounded64(y * torch.exp2(-e), case["store"])
                c[x][p, :, r], c[x + "_exp"][p, :, r] = codes, e.squeeze(-1) + 127
                if x == "k":
                    y = codes * torch.exp2(e)
                    low, high = y.amin(1), y.amax(1)
                    if at % page:
                        low, high = torch.minimum(low, c["bounds"][p, :, 0]), torch.maximum(high, c["bounds"][p, :, 1])
                    c["bounds"][p] = torch.stack([low, high], 1)
            at = stop
    whole = case["store"] == "int8"
    return None if whole else c["k"], None if whole else c["v"], None, None, c["bounds"]


def _rows64(s, name, case, i, used):
    """Rows of request i in the pages it holds: [kv_heads, rows, d]."""
    at = s["pages"][i, used].long()
    x = s["cache"][name].view(torch.uint8)[at].view(_CODES[case["store"]]).double() * torch.exp2(s["cache"][name + "_exp"][at].double() - 127).unsqueeze(-1)
    return x.transpose(0, 1).flatten(1, 2)


def _exact_read(case, s):
    out = [torch.zeros((case["batch"], case["tokens"], case["kv_heads"], case["d"]), dtype=torch.float64, device="cuda") for _ in range(2)]
    for i, n in enumerate(s["lengths"].tolist()):
        for y, x in zip(out, ("k", "v")):
            y[i, :n] = _rows64(s, x, case, i, slice(0, _pages_of(n, case["page"])))[:, :n].transpose(0, 1)
    return tuple(out)


def _exact_attend(case, s):
    b, h, d = s["q"].shape
    kv, page = case["kv_heads"], case["page"]
    out = torch.zeros((b, h, d), dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lengths"].tolist()):
        for j in range(kv if n else 0):
            if s["chosen"] is None:
                used = torch.arange(_pages_of(n, page), device="cuda")
            else:
                used = s["chosen"][i, j][s["chosen"][i, j] >= 0].long()
            place = (used.view(-1, 1) * page + torch.arange(page, device="cuda")).flatten()
            seen = place < n
            if case["window"]:
                seen &= place >= n - case["window"]
            at = s["pages"][i, used].long()
            k, v = (s["cache"][x].view(torch.uint8)[at, j].view(_CODES[case["store"]]).double().flatten(0, 1)[seen]
                    * torch.exp2(s["cache"][x + "_exp"][at, j].double().flatten()[seen] - 127).unsqueeze(1) for x in ("k", "v"))
            q = s["q"][i, j * (h // kv):(j + 1) * (h // kv)].double()
            z = q @ k.t() / math.sqrt(d)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["bias"]:
                z = z - s["slopes"][j * (h // kv):(j + 1) * (h // kv)].double().view(-1, 1) * (n - 1 - place[seen]).double()
            out[i, j * (h // kv):(j + 1) * (h // kv)] = torch.softmax(z, -1) @ v
    return out

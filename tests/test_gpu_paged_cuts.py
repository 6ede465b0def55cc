"""The cache in 8-bit pages in calls large enough for the kernels and rules that
small ones do not meet."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import paged as G  # noqa: E402
from tests.attention_ref import near  # noqa: E402
from tests.paged_ref import Cache  # noqa: E402


def say(*what):
    print("[gpu]", *what, flush=True)


# ------------------------------------------------------------------ workspaces

@pytest.mark.parametrize("b,h,kv,page,width,num,own", [
    (64, 32, 8, 16, 1, 16_384, True),           # a list far longer than the table: 130 MiB
    (1, 64, 1, 256, 20_000, None, True),        # a wide table: 79 MiB
    (1, 64, 1, 256, 20_000, 3, False),          # the same under a short list, which takes none
    (1, 64, 1, 256, 10_000, None, True),        # as many parts, half as long: 320,000 tiles of both blocks, 64 a part
    (1, 64, 1, 256, 5000, None, False),         # 40 MiB
    (2, 8, 2, 64, 64, None, False),
])
def test_only_workspaces_to_64_mib_stay_with_the_library(monkeypatch, b, h, kv, page, width, num, own):
    say("workspace", b, h, kv, page, width, num)
    d = 128
    cache = F.PagedCache.empty(3, kv, d, page=page, bounds=False)
    g = torch.Generator(device="cuda").manual_seed(b)
    k, v = (torch.randn((b * 5, kv, d), generator=g, device="cuda") for _ in range(2))
    pages = torch.full((b, width), -1, dtype=torch.int32, device="cuda")
    pages[-1, 0] = 1                            # (one request with rows: a page is one request's)
    n = torch.full((b,), 5, dtype=torch.int32, device="cuda")
    F.cache_write(cache, k, v, pages, n)
    q = torch.randn((b, h, d), generator=g, device="cuda").bfloat16()
    chosen = None
    if num is not None:
        chosen = torch.full((b, kv, num), -1, dtype=torch.int32, device="cuda")
        chosen[:, :, -1] = 0
    asked, taken = [], []
    rule, launch = G._own_workspace, G._launch

    def looked(large):
        asked.append(bool(large))
        return rule(large)

    def launched(fn, args, device):
        a = G.PagedArgs.from_buffer_copy(args)
        taken.append((a.ws_bytes, F.lib().frog_attend_paged_workspace(C.byref(a))))
        return launch(fn, args, device)

    monkeypatch.setattr(G, "_own_workspace", looked)
    monkeypatch.setattr(G, "_launch", launched)
    out = F.attend_paged(q, cache, pages, n, chosen=chosen)
    monkeypatch.undo()
    (given, needed), = taken
    assert asked == [own] and (needed > 2 ** 26) == own and given == (needed if own else 0)
    # one page of five rows: the same as over a table of that page alone
    small = F.attend_paged(q, cache, pages[:, :1].contiguous(), n)
    assert small[-1].any() and not small[:-1].any()
    assert torch.equal(out, small)


# ------------------------------------------------------------------ many small pages written

LIMIT = {"e4m3": 448.0, "int8": 127.0}
ONE_WAVE = {32: 64, 64: 32, 96: 32, 128: 16}      # largest page whose rows a wavefront has in four rounds


def quantised(x, store):
    """Codes (float64) and bytes of rows in float64: the least power of at least -100 that the largest magnitude fits."""
    fine = torch.isfinite(x).all(-1)
    x = torch.where(fine.unsqueeze(-1), x, 0.0)
    a = x.abs().amax(-1)
    e = torch.ceil(torch.log2((a / LIMIT[store]).clamp(min=2.0 ** -110)))
    e = torch.where(a > LIMIT[store] * torch.exp2(e), e + 1, e)
    e = torch.where(a <= LIMIT[store] * torch.exp2(e - 1), e - 1, e).clamp(min=-100)
    y = x * torch.exp2(-e).unsqueeze(-1)
    if store == "e4m3":
        unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = torch.round(y / unit) * unit
    else:
        y = torch.round(y)
    return y, torch.where(fine, e + 127, 255.0)


class Arrays:
    """The cache's arrays in 64 bits on the host, all rows of a call at a time."""

    def __init__(self, cache):
        self.store = "int8" if cache.k.dtype == torch.int8 else "e4m3"
        self.of(cache)

    def of(self, cache):
        self.t = {x: getattr(cache, x).cpu().float().double() for x in ("k", "v", "k_exp", "v_exp", "bounds")}

    def write(self, k, v, pages, lengths, starts):
        num, kv, page, d = self.t["k"].shape
        b, width = pages.shape
        starts, lengths = starts.long(), lengths.long()
        token = torch.arange(int(starts[0]), int(starts[-1]))
        request = torch.searchsorted(starts[1:].contiguous(), token, right=True)
        place = lengths[request] - starts[request + 1] + token
        inside = (place >= 0) & (place < width * page)
        at = torch.where(inside, pages[request, (place // page).clamp(0, width - 1)].long(), -1)
        inside &= (at >= 0) & (at < num)
        token, at, row = token[inside], at[inside], place[inside] % page
        for x, t in (("k", k), ("v", v)):
            codes, byte = quantised(t[token].double(), self.store)
            self.t[x][at, :, row] = codes
            self.t[x + "_exp"][at, :, row] = byte
            if x == "k":
                value = torch.where((byte == 255).unsqueeze(-1), torch.nan, codes * torch.exp2(byte - 127).unsqueeze(-1))
                old = self.t["bounds"]
                begun = at[row == 0]
                old[begun, :, 0], old[begun, :, 1] = torch.inf, -torch.inf
                index = at.view(-1, 1, 1).expand_as(value)
                # (amin and amax hand a NaN on)
                least = old[:, :, 0].contiguous().scatter_reduce_(0, index, value, "amin")
                most = old[:, :, 1].contiguous().scatter_reduce_(0, index, value, "amax")
                # a head with a row that is not finite has no bounds in any channel
                lost = torch.zeros((num, kv), dtype=torch.bool)
                lost[at] |= False
                lost.view(-1)[(at.unsqueeze(1) * kv + torch.arange(kv))[byte == 255]] = True
                least[lost], most[lost] = torch.nan, torch.nan
                self.t["bounds"] = torch.stack([least, most], 2)

    def same(self, cache):
        for x, want in self.t.items():
            got = getattr(cache, x).cpu().float().double()
            assert torch.equal(torch.isnan(got), torch.isnan(want)), x
            wrong = (got.nan_to_num(0.0) != want.nan_to_num(0.0)).nonzero()
            assert len(wrong) == 0, (x, len(wrong), wrong[:3].tolist())


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d,page", [(32, 16), (32, 64), (64, 16), (64, 32), (96, 16), (96, 32), (128, 16)])
def test_many_small_pages(kind, store, d, page):
    """Pages that a wavefront writes alone: prompts, pieces and single rows behind them, in a call of 4,096 (page, head) and more."""
    say("small pages", kind, store, d, page)
    assert page <= ONE_WAVE[d]
    b, kv, width = 300, 7, max(2, 64 // page)
    g = torch.Generator().manual_seed(d + page)
    total = b * width + 5
    pages = torch.randperm(total, generator=g)[: b * width].view(b, width).to(torch.int32)
    pages[3, 1], pages[8, 0], pages[9, -1] = -1, total, -2 ** 31
    cache = F.PagedCache.empty(total, kv, d, page=page, storage=store)
    ref = Arrays(cache)
    n = torch.zeros(b, dtype=torch.long)
    for step, most in enumerate((40, 1, 20, page)):
        new = torch.randint(0, most + 1, (b,), generator=g) if step != 1 else torch.ones(b, dtype=torch.long)
        new[0], new[1] = most, 0
        n = (n + new).clamp(max=width * page)
        length = n.clone()
        if step == 2:
            length[5], length[6], length[7] = new[5] - 3, 2 ** 30, -1    # rows before a request's start, past its pages, of none
        starts = torch.cat([torch.zeros(1, dtype=torch.long), new.cumsum(0)]).to(torch.int32)
        tokens = int(starts[-1])
        assert (tokens // page + 2 * b) * kv >= 4096
        k, v = (torch.randn((tokens, kv, d), generator=g) * torch.exp(torch.randn((tokens, kv, 1), generator=g)) for _ in range(2))
        k[..., 1] *= 7.0
        if step != 1:
            k[tokens // 2, 2, d - 1], k[tokens // 3, 0, 0], v[tokens // 2 + 1, 1, 5] = torch.nan, -torch.inf, torch.inf
        k, v = k.to(kind), v.to(kind)
        F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), length.to(torch.int32).cuda(), starts=starts.cuda())
        ref.write(k, v, pages, length, starts)
        ref.same(cache)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_small_pages_in_one_call_or_several(store):
    """The same rows by one wavefront a page and, in calls of fewer requests, by four."""
    b, kv, d, page = 520, 4, 64, 32
    g = torch.Generator().manual_seed(4)
    n = torch.randint(1, 2 * page + 1, (b,), generator=g)
    pages = torch.randperm(2 * b, generator=g).view(b, 2).to(torch.int32).cuda()
    one, many = (F.PagedCache.empty(2 * b, kv, d, page=page, storage=store) for _ in range(2))
    k, v = (torch.randn((int(n.sum()), kv, d), generator=g).half().cuda() for _ in range(2))
    starts = torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)])
    length = n.to(torch.int32).cuda()
    assert (len(k) // page + 2 * b) * kv >= 4096
    F.cache_write(one, k, v, pages, length, starts=starts.to(torch.int32).cuda())
    for i in range(0, b, 65):
        s = starts[i:i + 66]
        assert (int(s[-1] - s[0]) // page + 130) * kv < 4096
        F.cache_write(many, k[s[0]:s[-1]], v[s[0]:s[-1]], pages[i:i + 65], length[i:i + 65], starts=(s - s[0]).to(torch.int32).cuda())
    for x in ("k", "v", "k_exp", "v_exp", "bounds"):
        assert torch.equal(getattr(one, x).view(torch.uint8), getattr(many, x).view(torch.uint8)), x


# ------------------------------------------------------------------ many requests that are not split

@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("h,kv,d,page,width", [(2, 2, 32, 16, 65), (8, 2, 128, 64, 64), (8, 1, 96, 256, 16), (26, 2, 64, 32, 100),
                                               (36, 2, 128, 16, 256), (40, 1, 64, 128, 32)])
def test_requests_of_many_pairs_are_whole(kind, h, kv, d, page, width):
    """512 and more (request, kv head) pairs, tables of 65 to 256 tiles: a workgroup walks a whole request."""
    say("whole requests", kind, h, kv, d, page, width)
    b, rows = 512 // kv + 3, width * page
    assert 64 < rows // 16 <= 256 and b * kv >= 512
    # (pages that many requests read)
    g = torch.Generator().manual_seed(h + d)
    total = 40 * 64 // page + 30
    cache = F.PagedCache.empty(total, kv, d, page=page, storage="int8" if h % 8 else "e4m3", bounds=False)
    k, v = ((torch.randn((total * page, kv, d), generator=g) * torch.exp(0.5 * torch.randn((total * page, kv, 1), generator=g))).to(kind).cuda() for _ in range(2))
    F.cache_write(cache, k, v, torch.arange(total, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([total * page], dtype=torch.int32).cuda())
    pages = torch.randint(0, total, (b, width), generator=g, dtype=torch.int32)
    pages[5, width // 2] = -1
    n = torch.randint(1, rows + 1, (b,), generator=g, dtype=torch.int32)
    n[0], n[1], n[2], n[3], n[4], n[5] = rows, 0, rows - 1, 1, 2 ** 30, rows - 17
    q = (torch.randn((b, h, d), generator=g) * 1.2).to(kind)
    lo = torch.randint(-5, rows, (b,), generator=g, dtype=torch.int32)
    lr = torch.stack([lo, lo + torch.randint(-1, rows, (b,), generator=g, dtype=torch.int32)], -1)
    lr[0], lr[2] = torch.tensor([0, rows - 1]), torch.tensor([rows - 2, rows + 9])
    slopes = torch.exp2(-8.0 * torch.arange(1, h + 1) / h)
    at, ref = [0, 1, 2, 3, 4, 5, b // 3, b // 2, b - 1], Cache(cache)
    for kw in ({}, {"lr": lr}, {"lr": lr, "cap": 12.0, "slopes": slopes}):
        args = {x: y.cuda() if torch.is_tensor(y) else y for x, y in kw.items()}
        out, lse = F.attend_paged(q.cuda(), cache, pages.cuda(), n.cuda(), return_lse=True, **args)
        want, err, lw, le = ref.attend(q[at], pages[at], n[at], **{x: y[at] if x == "lr" else y for x, y in kw.items()})
        near(out[at].cpu(), want, err, f"out {list(kw)}")
        near(lse[at].cpu(), lw, le, f"lse {list(kw)}")


# ------------------------------------------------------------------ more workgroups than a launch takes

def test_attention_and_selection_in_several_launches():
    """2^21 requests of 8 kv heads over a few pages: 2^33 threads and more, against the same requests in a call of 4,096."""
    g = torch.Generator(device="cuda").manual_seed(0)
    kv, d, page, few, b = 8, 32, 16, 4096, 2 ** 21 + 7
    say("several launches", b)
    cache = F.PagedCache.empty(64, kv, d, page=page)
    k, v = (torch.randn((64 * page, kv, d), generator=g, device="cuda") for _ in range(2))
    every = torch.arange(64, dtype=torch.int32, device="cuda").view(1, -1)
    F.cache_write(cache, k, v, every, torch.full((1,), 64 * page, dtype=torch.int32, device="cuda"))
    pages = torch.randint(0, 64, (few, 3), generator=g, device="cuda", dtype=torch.int32)
    n = torch.randint(0, 3 * page + 1, (few,), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn((few, 2 * kv, d), generator=g, device="cuda").bfloat16()
    at = torch.randint(0, few, (b,), generator=g, device="cuda")
    want, lse = F.attend_paged(q, cache, pages, n, return_lse=True)
    chosen = F.select_pages(q, cache, pages, n, 2)
    out, got = F.attend_paged(q[at], cache, pages[at], n[at], return_lse=True)
    assert torch.equal(out, want[at]) and torch.equal(got, lse[at])
    assert torch.equal(F.select_pages(q[at], cache, pages[at], n[at], 2), chosen[at])


def test_rows_in_several_launches():
    """2^21 requests of a row of 16 heads written, 2^24 blocks of 16 rows read, against parts of them in calls of their own."""
    g = torch.Generator(device="cuda").manual_seed(1)
    kv, d, b = 16, 32, 2 ** 21 + 3
    say("rows in several launches", b)
    cache = F.PagedCache.empty(b, kv, d, page=16, storage="int8")
    x = torch.randn((b, kv, d), generator=g, device="cuda").bfloat16()
    pages = torch.randperm(b, generator=g, device="cuda").to(torch.int32).view(b, 1)
    one = torch.ones(b, dtype=torch.int32, device="cuda")
    F.cache_write(cache, x, -x, pages, one)
    small = F.PagedCache.empty(1000, kv, d, page=16, storage="int8")
    own = torch.arange(1000, dtype=torch.int32, device="cuda").view(-1, 1)
    for i in (0, b // 2, b - 1000):
        F.cache_write(small, x[i:i + 1000], -x[i:i + 1000], own, one[:1000])
        where = pages[i:i + 1000, 0].long()
        for name in ("k", "v", "k_exp", "v_exp", "bounds"):
            assert torch.equal(getattr(cache, name)[where], getattr(small, name)), (name, i)
    k, v = F.cache_read(cache, pages, one, 1)
    # (a code is off by half a step of at most 1 / 63.5 of the largest magnitude: what it is above, half the limit)
    assert ((k[:, 0].float() - x.float()).abs().amax(-1) <= x.float().abs().amax(-1) / 127).all() and torch.equal(k, -v)
    del cache, small, x, k, v, pages, one
    b, width = 2 ** 20 + 5, 17
    cache = F.PagedCache.empty(64, 1, d, page=16)
    k = torch.randn((1024, 1, d), generator=g, device="cuda")
    every = torch.arange(64, dtype=torch.int32, device="cuda").view(1, -1)
    F.cache_write(cache, k, -k, every, torch.full((1,), 1024, dtype=torch.int32, device="cuda"))
    pages = torch.randint(0, 64, (b, width), generator=g, device="cuda", dtype=torch.int32)
    n = torch.randint(0, 16 * width + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    k, v = F.cache_read(cache, pages, n, 16 * width)
    for i in (0, b // 2, 2 ** 24 // width - 1000, b - 2000):
        some = F.cache_read(cache, pages[i:i + 2000], n[i:i + 2000], 16 * width)
        assert torch.equal(k[i:i + 2000], some[0]) and torch.equal(v[i:i + 2000], some[1]), i

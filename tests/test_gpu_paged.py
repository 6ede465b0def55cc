"""The cache in 8-bit pages against its definition: rows written and read back
exactly, the same pages chosen, attention within its error bound."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from tests.attention_ref import Attention, near  # noqa: E402
from tests.paged_ref import Cache  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
NAN_CODE = {"e4m3": 0x7F, "int8": 0x80}


def say(*what):
    print("[gpu]", *what, flush=True)


def rand_rows(g, kind, *shape):
    x = torch.randn(shape, generator=g) * torch.exp(torch.randn((*shape[:-1], 1), generator=g))
    x[..., 0] *= 9.0
    return x.to(TYPES[kind])


def table(g, b, width, extra=3):
    return torch.randperm(b * width + extra, generator=g)[: b * width].view(b, width).to(torch.int32), b * width + extra


def ragged(g, b, most):
    n = torch.randint(0, most + 1, (b,), generator=g)
    n[torch.randint(0, b, (1,), generator=g)] = most
    if b > 2:
        n[torch.randint(0, b, (1,), generator=g)] = 0
    return n


def filled(kind, store, b, most, kv, d, page, seed=0, lengths=None, bounds=True):
    """A cache with rows of `b` requests in it, and its tables."""
    g = torch.Generator().manual_seed(seed)
    n = ragged(g, b, most) if lengths is None else torch.tensor(lengths)
    width = max(1, -(-int(n.max()) // page)) + seed % 2
    pages, total = table(g, b, width)
    cache = F.PagedCache.empty(total, kv, d, page=page, storage=store, bounds=bounds)
    starts = torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)]).to(torch.int32)
    k, v = (rand_rows(g, kind, int(starts[-1]), kv, d) for _ in range(2))
    lengths = n.to(torch.int32)
    if len(k):
        F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), lengths.cuda(), starts=starts.cuda())
    return cache, k, v, pages, lengths, starts


# ------------------------------------------------------------------ rows in and out

@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("b,most,kv,d,page", [(1, 1, 1, 32, 16), (3, 70, 2, 128, 16), (5, 150, 3, 96, 64), (9, 33, 1, 64, 32), (2, 600, 4, 64, 256),
                                              (70, 20, 2, 32, 16)])
def test_rows(kind, store, b, most, kv, d, page):
    say("rows", kind, store, b, most, kv, d, page)
    cache, k, v, pages, n, starts = filled(kind, store, b, most, kv, d, page, seed=b)
    ref = Cache(F.PagedCache.empty(cache.shape[0], kv, d, page=page, storage=store))
    ref.write(k, v, pages, n, starts)
    ref.same(cache)
    # appended row by row and in pieces
    g = torch.Generator().manual_seed(7)
    for step in range(3):
        new = torch.randint(0, (1, 4, page + 3)[step] + 1, (b,), generator=g)
        new = torch.minimum(new, pages.shape[1] * page - n)
        starts = torch.cat([torch.zeros(1, dtype=torch.long), new.cumsum(0)]).to(torch.int32)
        k, v = (rand_rows(g, kind, int(starts[-1]), kv, d) for _ in range(2))
        n = (n + new).to(torch.int32)
        if len(k):
            F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), n.cuda(), starts=starts.cuda())
            ref.write(k, v, pages, n, starts)
    ref.same(cache)
    for dtype in TYPES.values():
        slots = most // 2 + 3
        for got, want in zip(F.cache_read(cache, pages.cuda(), n.cuda(), slots, dtype=dtype), ref.read(pages, n, slots, dtype)):
            assert got.dtype == dtype and torch.equal(got.cpu(), want)
    got = F.cache_read(cache, pages.cuda(), n.cuda())
    assert got[0].shape == (b, pages.shape[1] * page, kv, d)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_every_code_and_power(store):
    # rows whose largest magnitude stands just at, below and above the limit of a power, over the whole range of fp32
    limit = 448.0 if store == "e4m3" else 127.0
    rows = []
    for e in list(range(-126, -90, 3)) + list(range(-20, 21)) + [100, 118, 119, 120, 121]:
        for up in (-1, 0, 1):
            a = torch.tensor(limit).mul(2.0 ** e).float() if e > -126 else torch.tensor(1e-38)
            if not torch.isfinite(a):
                continue
            a = (a.view(torch.int32) + up).view(torch.float32)
            x = torch.linspace(-1, 1, 32) * a
            x[5] = a
            rows.append(x)
    # every code of one power, and the middles between neighbours
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn if store == "e4m3" else torch.int8).float()
    codes = codes[torch.isfinite(codes) & (codes.abs() <= limit)].sort()[0]
    for block in torch.cat([codes, (codes[1:] + codes[:-1]) / 2]).split(31):
        rows.append(torch.cat([block, torch.full((32 - len(block),), limit)]))
    rows += [torch.zeros(32), torch.full((32,), 1e-45), -torch.zeros(32), torch.full((32,), 2.0 ** -101)]
    odd = torch.randn(3, 32)
    odd[0, 3], odd[1, 31], odd[2, 0] = math.inf, -math.inf, math.nan
    x = torch.cat([torch.stack(rows), odd]).view(-1, 1, 32)
    n = len(x)
    say("codes and powers", store, n)
    cache = F.PagedCache.empty(-(-n // 16), 1, 32, page=16, storage=store)
    pages, lengths = torch.arange(cache.shape[0], dtype=torch.int32).view(1, -1), torch.tensor([n], dtype=torch.int32)
    ref = Cache(cache)
    F.cache_write(cache, x.cuda(), (x * -0.5).cuda(), pages.cuda(), lengths.cuda())
    ref.write(x, x * -0.5, pages, lengths)
    ref.same(cache)
    got = F.cache_read(cache, pages.cuda(), lengths.cuda(), n, dtype=torch.float32)[0][0, :, 0].cpu()
    # a largest magnitude a just above 127 2^121 has the power 122 and the code 64, of value 2^128: above what 32 bits hold
    over = (x[:-3, 0].abs() > 127 * 2.0 ** 121) if store == "int8" else torch.zeros((n - 3, 32), dtype=torch.bool)
    assert torch.isnan(got[-3:]).all() and torch.equal(torch.isfinite(got[:-3]), ~over)
    step = 2.0 ** -4 if store == "e4m3" else 0.0       # e4m3: relative to the value, int8: to the largest
    top = x[:-3, 0].abs().amax(-1, keepdim=True).double()
    allowed = step * x[:-3, 0].abs().double() + (top * 2.0 ** -17 if store == "e4m3" else top / 127) + 2.0 ** -101
    assert (((got[:-3].double() - x[:-3, 0].double()).abs() <= allowed) | over).all()


def test_bounds_hold_every_row_and_say_what_is_not_a_number():
    cache, k, v, pages, n, starts = filled("bf16", "int8", 4, 100, 2, 64, 32, seed=4)
    x = k[:1].clone()
    x[0, 1, 7] = math.nan
    ref = Cache(cache)
    i = int(n.argmax())
    more = torch.zeros(5, dtype=torch.int32)
    more[i + 1:] = 1
    m = n.clone()
    m[i] = 99                                       # a row in the middle of the last page
    F.cache_write(cache, x.cuda(), x.cuda(), pages.cuda(), m.cuda(), starts=more.cuda())
    ref.write(x, x, pages, m, more)
    ref.same(cache)
    at = int(pages[i, 98 // 32])
    assert torch.isnan(cache.bounds[at, 1]).all() and torch.isfinite(cache.bounds[at, 0]).all()
    # once more beside it, and the page begun anew
    for length in (100, 97):
        m[i] = length
        F.cache_write(cache, k[:1].cuda(), k[:1].cuda(), pages.cuda(), m.cuda(), starts=more.cuda())
        ref.write(k[:1], k[:1], pages, m, more)
        ref.same(cache)
    assert torch.isfinite(cache.bounds[at]).all()


def test_rows_that_have_no_place_are_left_out():
    # lengths below the new rows, above the pages, pages that are none, starts that skip rows
    g = torch.Generator().manual_seed(3)
    pages, total = table(g, 5, 3)
    pages[2, 1], pages[3, 0] = -1, total
    cache = F.PagedCache.empty(total, 2, 64, page=16)
    ref = Cache(cache)
    starts = torch.tensor([3, 23, 63, 100, 130, 130], dtype=torch.int32)
    lengths = torch.tensor([7, 55, 40, 30, 48], dtype=torch.int32)
    k, v = rand_rows(g, "bf16", 140, 2, 64), rand_rows(g, "bf16", 140, 2, 64)
    F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), lengths.cuda(), starts=starts.cuda())
    ref.write(k, v, pages, lengths, starts)
    ref.same(cache)
    for got, want in zip(F.cache_read(cache, pages.cuda(), lengths.cuda(), 60), ref.read(pages, lengths, 60, torch.bfloat16)):
        assert torch.equal(got.cpu(), want)
    # equal shares, one request a padding with no rows
    lengths = torch.tensor([10, 0, 30, 20, 48], dtype=torch.int32)
    F.cache_write(cache, k[:10].cuda(), v[:10].cuda(), pages.cuda(), lengths.cuda())
    ref.write(k[:10], v[:10], pages, lengths)
    ref.same(cache)


def test_strided_rows_and_other_streams():
    g = torch.Generator().manual_seed(5)
    pages, total = table(g, 3, 4)
    both = rand_rows(g, "fp16", 60, 2 * 3, 96).cuda()          # keys and values side by side, as one product leaves them
    k, v = both[:, :3], both[:, 3:]
    lengths = torch.tensor([20, 20, 20], dtype=torch.int32).cuda()
    one, two = (F.PagedCache.empty(total, 3, 96, page=16, storage="int8") for _ in range(2))
    F.cache_write(one, k, v, pages.cuda(), lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    F.cache_write(two, k.contiguous(), v.transpose(0, 1).contiguous().transpose(0, 1), pages.cuda(), lengths, stream=side)
    read = F.cache_read(two, pages.cuda(), lengths, 20, stream=side)
    side.synchronize()
    for x in ("k", "v", "k_exp", "v_exp", "bounds"):
        assert torch.equal(getattr(one, x).cpu().float(), getattr(two, x).cpu().float()), x
    assert all(torch.equal(x, y) for x, y in zip(read, F.cache_read(one, pages.cuda(), lengths, 20)))


def test_versions():
    cache = F.PagedCache.empty(2, 1, 32, page=16)
    before = cache.k._version, cache.bounds._version
    x = torch.ones(1, 1, 32, device="cuda")
    F.cache_write(cache, x, x, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    assert cache.k._version > before[0] and cache.bounds._version > before[1]


# ------------------------------------------------------------------ pages chosen

@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("b,most,h,kv,d,page", [(1, 5, 1, 1, 32, 16), (3, 900, 8, 2, 128, 16), (5, 2000, 3, 3, 96, 64), (2, 3000, 28, 4, 64, 32)])
def test_select(kind, b, most, h, kv, d, page):
    say("select", kind, b, most, h, kv, d, page)
    cache, _, _, pages, n, _ = filled(kind, "e4m3" if d == 128 else "int8", b, most, kv, d, page, seed=b)
    q = rand_rows(torch.Generator().manual_seed(1), kind, b, h, d)
    ref = Cache(cache)
    width = pages.shape[1]
    for keep, first, recent in ((1, 0, 1), (1, 0, 0), (4, 1, 1), (4, 0, 4), (width, 0, 1), (width + 5, 2, 3), (max(1, width // 2), 0, 0)):
        got = F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), keep, first=first, recent=recent)
        assert got.dtype == torch.int32 and torch.equal(got.cpu(), ref.select(q, pages, n, keep, first, recent)), (keep, first, recent)
    assert F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), 0, recent=0).shape == (b, kv, 0)


def test_select_ties_and_what_is_not_a_number():
    pages, total = table(torch.Generator().manual_seed(2), 1, 40, extra=0)
    cache = F.PagedCache.empty(total, 2, 32, page=16)
    cache.bounds[:, :, 1] = 1.0
    cache.bounds[pages[0, 7].item()] = math.nan
    cache.bounds[pages[0, 21].item(), 1, 1] = 2.0
    cache.bounds[pages[0, 30].item(), 0, 1] = math.inf
    pages[0, 12] = -5
    lengths = torch.tensor([39 * 16 + 1], dtype=torch.int32)
    q = torch.ones(1, 4, 32)
    ref = Cache(cache)
    for keep in (1, 2, 3, 4, 10, 38, 39):
        for x in (q, -q, q * 0, q * math.nan):
            got = F.select_pages(x.cuda(), cache, pages.cuda(), lengths.cuda(), keep)
            assert torch.equal(got.cpu(), ref.select(x, pages, lengths, keep, 0, 1)), keep


@pytest.mark.parametrize("width", [2100, 3100, 8200])
def test_select_many_pages(width):
    # more pages than one workgroup keeps: scored by one launch, chosen by another, from registers or from memory
    g = torch.Generator().manual_seed(6)
    b, kv, d = 2, 2, 64
    pages, total = table(g, b, width)
    cache = F.PagedCache.empty(total, kv, d, page=16)
    q = rand_rows(g, "bf16", b, 6, d)
    for kind in ("all differ", "few values", "one value"):
        x = torch.randn(cache.bounds.shape, generator=g).sort(2)[0]
        # (of equal bounds only some pages' differ)
        x = x if kind == "all differ" else x[:1] * torch.ones((total, 1, 1, 1)) if kind == "one value" else x[torch.arange(total) % 7]
        cache.bounds.copy_(x)
        ref = Cache(cache)
        for n in ([width * 16, 5000], [0, 1], [width * 16 + 99, 2080 * 16]):
            n = torch.tensor(n, dtype=torch.int32)
            for keep in (1, 2, 200, 2050):
                first = 1 if keep > 1 else 0
                got = F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), keep, first=first)
                assert torch.equal(got.cpu(), ref.select(q, pages, n, keep, first, 1)), (kind, n, keep)


@pytest.mark.parametrize("width", [3, 63, 64, 65, 130, 1025, 2048])
def test_select_counts(width):
    # every number of pages kept about a wavefront's and a workgroup's share, scores with and without equals
    g = torch.Generator().manual_seed(width)
    pages, total = table(g, 1, width)
    cache = F.PagedCache.empty(total, 1, 32, page=16, storage="int8")
    q = rand_rows(g, "fp16", 1, 2, 32)
    n = torch.tensor([width * 16 - 5], dtype=torch.int32)
    for spread in (1, 3, total):
        cache.bounds.copy_(torch.randn(cache.bounds.shape, generator=g).sort(2)[0][torch.arange(total) % spread])
        ref = Cache(cache)
        for keep in sorted({1, 2, 3, width // 3, width // 2, width - 2, width - 1, width, width + 1} - {0}):
            for first, recent in ((0, 0), (0, 1), (1, keep - 1), (keep // 2, keep - keep // 2)):
                if first + recent <= keep:
                    got = F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), keep, first=first, recent=recent)
                    assert torch.equal(got.cpu(), ref.select(q, pages, n, keep, first, recent)), (spread, keep, first, recent)


# ------------------------------------------------------------------ attention

def check(q, cache, pages, n, **kw):
    out, lse = F.attend_paged(q.cuda(), cache, pages.cuda(), n.cuda(), **{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()}, return_lse=True)
    want, err, lw, le = Cache(cache).attend(q, pages, n, **kw)
    assert out.dtype == q.dtype
    near(out.cpu(), want, err, "out")
    near(lse.cpu(), lw, le, "lse")
    return out, lse


SHAPES = [(1, 1, 1, 1, 32, 16), (4, 37, 2, 2, 64, 16), (3, 700, 8, 2, 128, 64), (5, 1500, 21, 3, 96, 32), (2, 2600, 4, 1, 128, 256),
          (9, 130, 16, 1, 64, 128), (2, 900, 40, 2, 128, 16), (2, 400, 66, 2, 32, 64), (70, 60, 2, 1, 128, 16)]


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("b,most,h,kv,d,page", SHAPES)
def test_attend(kind, store, b, most, h, kv, d, page):
    say("attend", kind, store, b, most, h, kv, d, page)
    cache, _, _, pages, n, _ = filled(kind, store, b, most, kv, d, page, seed=b, bounds=False)
    g = torch.Generator().manual_seed(11)
    q = (torch.randn((b, h, d), generator=g) * 1.5).to(TYPES[kind])
    slopes = torch.exp2(-8.0 * torch.arange(1, h + 1) / h)
    lo = torch.randint(-3, most + 3, (b,), generator=g)
    lr = torch.stack([lo, lo + torch.randint(-2, most + 5, (b,), generator=g)], -1).to(torch.int32)
    width = pages.shape[1]
    check(q, cache, pages, n)
    check(q, cache, pages, n, lr=lr)
    check(q, cache, pages, n, cap=5.0, slopes=slopes, lr=lr, scale=0.3)
    check(q, cache, pages, n, slopes=slopes)
    # pages in any order, numbers that are none, one twice
    chosen = torch.randint(-2, width + 2, (b, kv, 6), generator=g).to(torch.int32)
    check(q, cache, pages, n, chosen=chosen)
    check(q, cache, pages, n, chosen=chosen, cap=80.0, lr=lr, slopes=slopes)
    out, lse = F.attend_paged(q.cuda(), cache, pages.cuda(), n.cuda(), chosen=chosen[:, :, :0].contiguous().cuda(), return_lse=True)
    assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 1023, 1024, 1025, 1100, 2047, 2049, 4100])
def test_lengths(n, page):
    cache, _, _, pages, lengths, _ = filled("bf16", "e4m3", 2, n, 1, 64, page, lengths=[n, max(1, n - 7)], bounds=False)
    q = torch.randn((2, 4, 64), generator=torch.Generator().manual_seed(n)).to(torch.bfloat16)
    check(q, cache, pages, lengths)
    check(q, cache, pages, lengths, lr=torch.tensor([[n - 1, n - 1], [0, 0]], dtype=torch.int32))


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_what_no_token_sees_may_hold_anything(kind, store):
    say("rows unseen", kind, store)
    cache, _, _, pages, n, _ = filled(kind, store, 4, 200, 2, 128, 32, seed=4, bounds=False)
    lr = torch.tensor([[20, 150], [30, 99], [5, 4], [0, 10 ** 9]], dtype=torch.int32)
    q = torch.randn((4, 6, 128), generator=torch.Generator().manual_seed(0)).to(TYPES[kind])
    ref = Cache(cache)
    ref = ref.attend(q, pages, n, lr=lr)
    seen = torch.zeros(cache.shape[0], 32, dtype=torch.bool)
    for i in range(4):
        for t in range(max(0, int(lr[i, 0])), min(int(n[i]), int(lr[i, 1]) + 1)):
            seen[pages[i, t // 32], t % 32] = True
    hide = (~seen).view(-1, 1, 32, 1).expand(cache.shape).cuda()
    for x in (cache.k, cache.v):
        x.view(torch.uint8).masked_fill_(hide, NAN_CODE[store])
    for x in (cache.k_exp, cache.v_exp):
        x.masked_fill_(hide[..., 0], 255)
    # entries past a request's rows are not looked at
    for i in range(4):
        pages[i, -(-int(n[i]) // 32):] = 2 ** 30
    out, lse = F.attend_paged(q.cuda(), cache, pages.cuda(), n.cuda(), lr=lr.cuda(), return_lse=True)
    near(out.cpu(), ref[0], ref[1], "out")
    near(lse.cpu(), ref[2], ref[3], "lse")


@pytest.mark.parametrize("page,most", [(16, 300), (64, 3000)])
def test_entries_that_are_no_page_and_lengths_past_the_table(page, most):
    cache, _, _, pages, n, _ = filled("bf16", "int8", 4, most, 2, 64, page, lengths=[most, most - 1, most // 2, 5], seed=1)
    pages[0, 2], pages[1, 0], pages[1, -1], pages[2, 1] = -1, cache.shape[0], -2 ** 31, 2 ** 31 - 1
    pages[3] = -1                                    # a request of no page at all
    n = n + torch.tensor([page * 9, 2 ** 30, 0, 0], dtype=torch.int32)
    q = torch.randn((4, 6, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    ref = Cache(cache)
    full = pages.shape[1] * page
    check(q, cache, pages, n)
    check(q, cache, pages, n, lr=torch.tensor([[0, full], [page // 2, full - 2], [page, 2 * page - 1], [0, 4]], dtype=torch.int32))
    for keep in (1, 3, pages.shape[1]):
        got = F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), keep)
        assert torch.equal(got.cpu(), ref.select(q, pages, n, keep, 0, 1))
        check(q, cache, pages, n, chosen=got.cpu())
    for got, want in zip(F.cache_read(cache, pages.cuda(), n.cuda(), full + 20), ref.read(pages, n, full + 20, torch.bfloat16)):
        assert torch.equal(got.cpu(), want)
    n[:] = torch.tensor([-1, -2 ** 31, 0, 0], dtype=torch.int32)
    out, lse = F.attend_paged(q.cuda(), cache, pages.cuda(), n.cuda(), return_lse=True)
    assert not out.any() and (lse == -math.inf).all()
    assert (F.select_pages(q.cuda(), cache, pages.cuda(), n.cuda(), 2) == -1).all()


def test_arguments_are_refused():
    cache, _, _, pages, n, _ = filled("bf16", "int8", 2, 50, 2, 64, 16, lengths=[50, 20])
    pages, n = pages.cuda(), n.cuda()
    q, k = torch.randn(2, 4, 64, device="cuda").bfloat16(), torch.randn(2, 2, 64, device="cuda").bfloat16()
    bad = [lambda: F.attend_paged(q[:1], cache, pages, n), lambda: F.attend_paged(q[..., :32], cache, pages, n), lambda: F.attend_paged(q.double(), cache, pages, n),
           lambda: F.attend_paged(q.cpu(), cache, pages, n), lambda: F.attend_paged(q, cache, pages.long(), n), lambda: F.attend_paged(q, cache, pages, n[:1]),
           lambda: F.attend_paged(q, cache, pages.t(), n), lambda: F.attend_paged(q, cache, pages, n, chosen=pages), lambda: F.attend_paged(q, cache, pages, n, lr=pages),
           lambda: F.attend_paged(q, cache, pages, n, slopes=torch.ones(3, device="cuda")), lambda: F.attend_paged(q.requires_grad_(), cache, pages, n),
           lambda: F.attend_paged(q.detach().transpose(1, 2).contiguous().transpose(1, 2), cache, pages, n),
           lambda: F.select_pages(q.detach(), cache, pages, n, 2, first=2), lambda: F.select_pages(q.detach(), cache, pages, n, 2, recent=-1),
           lambda: F.select_pages(q.detach(), F.PagedCache(cache.k, cache.v, cache.k_exp, cache.v_exp), pages, n, 2),
           lambda: F.cache_write(cache, k, k[:1], pages, n), lambda: F.cache_write(cache, k[..., :32], k[..., :32], pages, n),
           lambda: F.cache_write(cache, k, k.half(), pages, n), lambda: F.cache_write(cache, k, k, pages, n, starts=n),
           lambda: F.cache_write(cache, k.clone().requires_grad_(), k, pages, n), lambda: F.cache_read(cache, pages, n, -1),
           lambda: F.cache_read(cache, pages, n, dtype=torch.float64), lambda: F.PagedCache(cache.k, cache.v[:1], cache.k_exp, cache.v_exp),
           lambda: F.PagedCache(cache.k, cache.v, cache.k_exp, cache.v_exp.int()), lambda: F.PagedCache(cache.k.transpose(0, 1), cache.v, cache.k_exp, cache.v_exp),
           lambda: F.PagedCache.empty(2, 1, 64, page=48), lambda: F.PagedCache.empty(2, 1, 80)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", i)
    q = q.detach()
    three = torch.randn(3, 2, 64, device="cuda").bfloat16()
    for f in (lambda: F.cache_write(cache, three, three, pages, n),                                         # no equal shares
              lambda: F.attend_paged(torch.randn(2, 3, 64, device="cuda"), cache, pages, n),                # 3 heads over 2
              lambda: F.attend_paged(torch.randn(2, 4, 72, device="cuda")[..., 3:67], cache, pages, n),     # rows off a boundary
              lambda: F.attend_paged(q, cache, pages, n, cap=-1.0)):
        with pytest.raises(F.FrogError):
            f()


def test_a_row_that_is_not_a_number_reaches_who_sees_it():
    cache, _, _, pages, n, _ = filled("bf16", "e4m3", 2, 100, 2, 64, 16, lengths=[100, 90], bounds=False)
    x = torch.full((2, 2, 64), math.nan)
    x[1] = 1.0
    F.cache_write(cache, x.cuda(), x.cuda(), pages.cuda(), torch.tensor([51, 90], dtype=torch.int32).cuda())
    q = torch.randn(2, 4, 64).bfloat16().cuda()
    out = F.attend_paged(q, cache, pages.cuda(), n.cuda())
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()
    out = F.attend_paged(q, cache, pages.cuda(), n.cuda(), lr=torch.tensor([[51, 99], [0, 99]], dtype=torch.int32).cuda())
    assert torch.isfinite(out).all()


def test_scores_of_great_magnitude():
    # one key outweighs all, wherever it stands; weights of the others vanish
    for at in (0, 5, 700, 1499):
        cache = F.PagedCache.empty(50, 1, 64, page=32, storage="int8")
        pages, n = torch.arange(50, dtype=torch.int32).view(1, 50), torch.tensor([1500], dtype=torch.int32)
        k = torch.randn((1500, 1, 64), generator=torch.Generator().manual_seed(at))
        k[at] = 300.0
        v = torch.randn((1500, 1, 64), generator=torch.Generator().manual_seed(at + 1))
        F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), n.cuda())
        check(torch.full((1, 2, 64), 5.0), cache, pages, n)
        check(torch.full((1, 2, 64), -5.0), cache, pages, n)
        check(torch.full((1, 2, 64), 5.0), cache, pages, n, scale=-0.2)
        check(torch.full((1, 2, 64), 5.0), cache, pages, n, scale=0.0)


def test_the_same_pages_for_several_tokens():
    # four drafted tokens of one request: requests of the same pages
    cache, _, _, pages, n, _ = filled("bf16", "e4m3", 1, 300, 2, 128, 16, lengths=[300], bounds=False)
    q = torch.randn((4, 8, 128), generator=torch.Generator().manual_seed(2)).bfloat16()
    check(q, cache, pages.expand(4, -1).contiguous(), torch.tensor([297, 298, 299, 300], dtype=torch.int32))


def test_no_pages_and_no_requests():
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    cache = F.PagedCache.empty(0, 2, 64)
    pages, n = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.tensor([5, 100], dtype=torch.int32, device="cuda")
    out, lse = F.attend_paged(q, cache, pages, n, return_lse=True)
    assert not out.any() and (lse == -math.inf).all()
    assert (F.select_pages(q, cache, pages, n, 3) == -1).all()
    assert not any(x.any() for x in F.cache_read(cache, pages, n, 7))
    x = torch.ones(2, 2, 64, device="cuda")
    F.cache_write(cache, x, x, pages, n)
    cache = F.PagedCache.empty(4, 2, 64)
    assert F.attend_paged(q[:0], cache, pages[:0], n[:0]).shape == (0, 4, 64)
    assert F.cache_read(cache, pages[:0], n[:0], 3)[0].shape == (0, 3, 2, 64)
    assert not F.attend_paged(q, cache, pages[:, :0].contiguous(), n).any()
    F.cache_write(cache, x[:0], x[:0], pages, n)
    torch.cuda.synchronize()


@pytest.mark.parametrize("b,most", [(1, 900), (6, 5000)])
def test_graph_and_stream(b, most):
    cache, _, _, pages, n, _ = filled("bf16", "int8", b, most, 2, 128, 32, seed=2)
    pages, n = pages.cuda(), n.cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((b, h, 128), generator=g, device="cuda").bfloat16() for h in (8, 2, 2))
    m = (n - 1).clamp(min=1)

    def step():
        F.cache_write(cache, k, v, pages, m)
        chosen = F.select_pages(q, cache, pages, m, 12, first=1)
        return F.attend_paged(q, cache, pages, m), F.attend_paged(q, cache, pages, m, chosen=chosen), chosen, *F.cache_read(cache, pages, m, 100)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = F.attend_paged(q, cache, pages, m, stream=side)
    chosen = F.select_pages(q, cache, pages, m, 12, first=1, stream=side)
    side.synchronize()
    assert torch.equal(got, want[0]) and torch.equal(chosen, want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        q.normal_(generator=g)
        k.normal_(generator=g)
        m.copy_((n - 1 - i).clamp(min=1))
        graph.replay()
        torch.cuda.synchronize()
        got2 = [x.clone() for x in got]
        assert all(torch.equal(x, y) for x, y in zip(got2, step()))


def test_two_graphs_do_not_share_a_workspace():
    cache, _, _, pages, n, _ = filled("bf16", "e4m3", 3, 6000, 2, 64, 16, seed=2)
    pages, n = pages.cuda(), n.cuda()
    qs = [torch.randn(3, 4, 64, device="cuda").bfloat16() for _ in range(2)]
    want = [F.attend_paged(q, cache, pages, n) for q in qs]
    graphs, outs = [], []
    for q in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(F.attend_paged(q, cache, pages, n))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_threads_on_streams_of_their_own():
    import threading
    cache, _, _, pages, n, _ = filled("bf16", "int8", 3, 9000, 2, 64, 16, seed=2)
    pages, n = pages.cuda(), n.cuda()
    qs = [torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i in range(3)]
    want = [(F.attend_paged(q, cache, pages, n), F.select_pages(q, cache, pages, n, 20)) for q in qs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = F.attend_paged(qs[i], cache, pages, n), F.select_pages(qs[i], cache, pages, n, 20)
                torch.cuda.current_stream().synchronize()
                wrong.extend(i for x, y in zip(got, want[i]) if not torch.equal(x, y))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_cache_beyond_32_bit_offsets():
    # 5 GiB of keys: pages at both ends
    kv, d, page = 8, 128, 256
    total = 5 * 2 ** 30 // (kv * d * page)
    cache = F.PagedCache.empty(total, kv, d, page=page, storage="int8")
    pages = torch.tensor([[total - 1, 0, total // 2, total - 2]], dtype=torch.int32)
    n = torch.tensor([4 * 256 - 3], dtype=torch.int32)
    g = torch.Generator().manual_seed(8)
    k, v = rand_rows(g, "bf16", int(n), kv, d), rand_rows(g, "bf16", int(n), kv, d)
    F.cache_write(cache, k.cuda(), v.cuda(), pages.cuda(), n.cuda())
    small = F.PagedCache.empty(4, kv, d, page=page, storage="int8")
    own = torch.arange(4, dtype=torch.int32).view(1, 4)
    F.cache_write(small, k.cuda(), v.cuda(), own.cuda(), n.cuda())
    q = torch.randn((1, 16, d), generator=g).bfloat16().cuda()
    assert torch.equal(F.attend_paged(q, cache, pages.cuda(), n.cuda()), F.attend_paged(q, small, own.cuda(), n.cuda()))
    assert torch.equal(F.select_pages(q, cache, pages.cuda(), n.cuda(), 2), F.select_pages(q, small, own.cuda(), n.cuda(), 2))
    assert all(torch.equal(x, y) for x, y in zip(F.cache_read(cache, pages.cuda(), n.cuda()), F.cache_read(small, own.cuda(), n.cuda())))


@pytest.mark.parametrize("b,most,h,kv,d,page", [(1, 20_000, 4, 1, 32, 16), (2, 9000, 6, 2, 64, 128), (1, 6000, 20, 1, 32, 64), (20, 1500, 3, 3, 32, 16)])
def test_every_cut(b, most, h, kv, d, page):
    """Parts joined by one wavefront, by four, by sixteen; requests far shorter than the longest."""
    say("cut", b, most, h, kv, d, page)
    lengths = [most] + [(i * 977) % most for i in range(1, b)]
    cache, _, _, pages, n, _ = filled("fp16", "int8", b, most, kv, d, page, lengths=lengths, bounds=False)
    q = torch.randn((b, h, d), generator=torch.Generator().manual_seed(4)).half()
    check(q, cache, pages, n)
    lr = torch.stack([n // 3, n - 1 - n // 5], -1).to(torch.int32)
    check(q, cache, pages, n, lr=lr, cap=20.0)
    # the same rows by a list of all pages, in another order
    chosen = torch.randperm(pages.shape[1], generator=torch.Generator().manual_seed(5)).to(torch.int32).expand(b, kv, -1).contiguous()
    check(q, cache, pages, n, chosen=chosen)


def test_large_calls():
    # above 400,000 tiles (longer parts), and lists of pages for more than 256 (request, kv head) pairs (one workgroup
    # each): some requests against 64 bits, over the rows read back, which are exact in 32
    g = torch.Generator(device="cuda").manual_seed(3)
    b, kv, d, page, width = 72, 4, 64, 64, 400
    cache = F.PagedCache.empty(b * width // 8, kv, d, page=page, storage="int8", bounds=False)
    for x in (cache.k, cache.v):
        x.random_(-127, 128, generator=g)
    for x in (cache.k_exp, cache.v_exp):
        x.random_(118, 124, generator=g)
    pages = torch.randint(0, cache.shape[0], (b, width), generator=g, device="cuda", dtype=torch.int32)
    n = torch.randint(1, width * page + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn((b, 3 * kv, d), generator=g, device="cuda")
    chosen = torch.randint(0, width, (b, kv, 60), generator=g, device="cuda", dtype=torch.int32)
    whole = F.attend_paged(q, cache, pages, n)
    some = F.attend_paged(q, cache, pages, n, chosen=chosen)
    for i in (0, 17, 71):
        k, v = F.cache_read(cache, pages[i:i + 1], n[i:i + 1], dtype=torch.float32)
        m = int(n[i])
        ref = Attention(q[i].view(1, 1, 3 * kv, d), k[:, :m], v[:, :m])
        # (queries of 32 bits enter in three factors: sums of three times as many products)
        near(whole[i].view(ref.out.shape), ref.out, 3 * ref.out_err, f"request {i}")
        for j in range(kv):
            at = (chosen[i, j].long().unsqueeze(1) * page + torch.arange(page, device="cuda")).flatten()
            at = at[at < m]
            got = some[i, 3 * j:3 * j + 3]
            if len(at) == 0:
                assert not got.any()
                continue
            ref = Attention(q[i, 3 * j:3 * j + 3].view(1, 1, 3, d), k[:, at, j:j + 1], v[:, at, j:j + 1])
            near(got.view(ref.out.shape), ref.out, 3 * ref.out_err, f"request {i}, kv head {j}")


# ------------------------------------------------------------------ together

def test_a_conversation():
    """A prompt written, read back for its own attention, then tokens decoded over all pages and over chosen ones."""
    g = torch.Generator(device="cuda").manual_seed(9)
    b, h, kv, d, page, prompt = 2, 8, 2, 64, 16, 200
    cache = F.PagedCache.empty(64, kv, d, page=page, storage="int8")
    pages = torch.randperm(64, generator=torch.Generator().manual_seed(1))[: b * 16].view(b, 16).to(torch.int32).cuda()
    k, v = (torch.randn((b, prompt, kv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    n = torch.full((b,), prompt, dtype=torch.int32, device="cuda")
    F.cache_write(cache, k.flatten(0, 1), v.flatten(0, 1), pages, n)
    for step in range(8):
        kr, vr = F.cache_read(cache, pages, n, 256)
        q = torch.randn((b, h, d), generator=g, device="cuda").bfloat16()
        lr = torch.stack([torch.zeros_like(n), n - 1], -1).view(b, 1, 2)
        whole, lse = F.attend_paged(q, cache, pages, n, return_lse=True)
        want, lse2 = F.attend(q.unsqueeze(1), kr, vr, lr, return_lse=True)
        # both within their errors of the exact result: weights 2^-8 (attend's short caches: 2^-16), one rounding each
        assert torch.allclose(whole.float(), want[:, 0].float(), rtol=2 ** -7, atol=2 ** -7)
        assert torch.allclose(lse, lse2[..., 0], rtol=1e-5, atol=1e-5)
        chosen = F.select_pages(q, cache, pages, n, 16)
        assert torch.equal(F.attend_paged(q, cache, pages, n, chosen=chosen), whole)
        some = F.select_pages(q, cache, pages, n, 5, first=1)
        check(q.cpu(), cache, pages.cpu(), n.cpu(), chosen=some.cpu())
        n += 1
        F.cache_write(cache, *(torch.randn((b, kv, d), generator=g, device="cuda").bfloat16() for _ in range(2)), pages, n)


def test_the_example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_cache.py")
    spec = importlib.util.spec_from_file_location("attention_cache", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    q, cache, pages, n, chosen, out = example.paged()
    assert n.tolist() == [170, 920, 60]
    ref = Cache(cache)
    assert torch.equal(chosen.cpu(), ref.select(q, pages.cpu(), n.cpu(), 8, 1, 1))
    want, err, _, _ = ref.attend(q.cpu(), pages.cpu(), n.cpu(), chosen.cpu())
    near(out.cpu(), want, err, "out")

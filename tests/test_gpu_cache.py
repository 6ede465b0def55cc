"""Attention over a shared prefix with paged tails, and eviction, against
their definitions."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from tests.attention_ref import Attention, near, select  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def make(kind, b, prefix, most, h, kv, d, page, ranges, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = torch.Generator().manual_seed(seed)
    t = TYPES[kind]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(t)

    width = max(1, -(-most // page))
    n = torch.randint(0, most + 1, (b,), generator=r)
    n[torch.randint(0, b, (1,), generator=r)] = most
    if b > 2:
        n[torch.randint(0, b, (1,), generator=r)] = 0
    pages = torch.randperm(b * width + 2, generator=r)[: b * width].view(b, width)
    lr = None
    if ranges:
        lo = torch.randint(-3, prefix + 3, (b,), generator=r)
        lr = torch.stack([lo, lo + torch.randint(-2, prefix + 5, (b,), generator=r)], -1).to(torch.int32).cuda()
    return dict(q=normal(b, h, d, std=1.5), k=normal(prefix, kv, d), v=normal(prefix, kv, d),
                k_pages=normal(b * width + 2, page, kv, d), v_pages=normal(b * width + 2, page, kv, d),
                pages=pages.to(torch.int32).cuda(), lengths=n.to(torch.int32).cuda()), lr


def check(s, lr, cap=0.0, slopes=None):
    out, lse = F.attend_shared(**s, lr=lr, cap=cap, slopes=slopes, return_lse=True)
    page, tk = s["k_pages"].shape[1], s["k"].shape[0]
    for i in range(s["q"].shape[0]):
        n = int(s["lengths"][i])
        used = s["pages"][i, : -(-n // page)].long()
        lo, hi = (0, tk - 1) if lr is None else (max(0, int(lr[i, 0])), min(tk - 1, int(lr[i, 1])))
        at = torch.cat([torch.arange(lo, hi + 1, device="cuda") if hi >= lo else torch.zeros(0, device="cuda", dtype=torch.long),
                        tk + torch.arange(n, device="cuda")])
        rows = [torch.cat([s[x][lo:hi + 1] if hi >= lo else s[x][:0], s[x + "_pages"][used].flatten(0, 1)[:n]]).unsqueeze(0) for x in ("k", "v")]
        opt = {} if slopes is None else dict(slopes=slopes, at_q=torch.full((1, 1), float(tk + n - 1), device="cuda"), at_k=at.float().unsqueeze(0))
        ref = Attention(s["q"][i].view(1, 1, *s["q"].shape[1:]), *rows, cap=cap, **opt)
        near(out[i].view(ref.out.shape), ref.out, ref.out_err, f"request {i} out")
        near(lse[i].view(ref.lse.shape), ref.lse, ref.lse_err, f"request {i} lse")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", [(1, 1, 0, 1, 1, 32, 1), (1, 40, 5, 4, 4, 64, 16), (5, 333, 70, 8, 2, 128, 16), (9, 1000, 33, 14, 2, 96, 7),
                                   (40, 130, 300, 8, 8, 64, 32), (3, 0, 50, 4, 1, 128, 16), (70, 2500, 20, 4, 4, 32, 16)], ids=str)
def test_shared(kind, shape):
    print(f"[gpu] shared prefix {kind} {shape}", flush=True)
    h = shape[3]
    for n, (cap, bias, ranges) in enumerate(((0.0, False, False), (5.0, True, True), (0.0, True, True), (5.0, False, False))):
        s, lr = make(kind, *shape, ranges and shape[1] > 0, seed=n)
        check(s, lr, cap, torch.exp2(-8.0 * torch.arange(1, h + 1, device="cuda") / h) if bias else None)


def test_shared_rows_outside_may_hold_anything():
    s, lr = make("bf16", 4, 200, 40, 4, 2, 64, 16, False, seed=3)
    lr = torch.tensor([[20, 150], [30, 99], [5, 4], [160, 170]], dtype=torch.int32, device="cuda")
    used = torch.zeros(200, dtype=torch.bool)
    for lo, hi in lr.tolist():
        used[lo:hi + 1] = True
    for x in ("k", "v"):
        s[x][~used.cuda()] = math.nan
        for i, n in enumerate(s["lengths"].tolist()):
            for t in range(n, s["pages"].shape[1] * 16):
                s[x + "_pages"][s["pages"][i, t // 16].item(), t % 16] = math.inf
    # entries past a tail are not read
    for i, n in enumerate(s["lengths"].tolist()):
        s["pages"][i, -(-n // 16):] = 2 ** 30
    check(s, lr)
    check(s, lr, 5.0)


def test_shared_pages_of_two_requests_and_strides():
    s, lr = make("fp16", 2, 100, 48, 4, 2, 64, 16, False, seed=5)
    s["pages"][1] = s["pages"][0]
    s["lengths"][:] = torch.tensor([48, 33])
    check(s, lr)
    out = F.attend_shared(**s)
    t = dict(s, k=s["k"].transpose(0, 1).contiguous().transpose(0, 1), v_pages=s["v_pages"].transpose(1, 2).contiguous().transpose(1, 2))
    assert torch.equal(out, F.attend_shared(**t))
    for _ in range(3):
        assert torch.equal(out, F.attend_shared(**s))


def test_shared_graph_and_stream():
    s, lr = make("bf16", 6, 3000, 100, 8, 2, 128, 16, True, seed=7)
    want = F.attend_shared(**s, lr=lr)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = F.attend_shared(**s, lr=lr, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = F.attend_shared(**s, lr=lr)
    for _ in range(4):
        s["q"].normal_()
        s["lengths"].random_(0, 101)
        want = F.attend_shared(**s, lr=lr)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


# ------------------------------------------------------------------ eviction

def check_evict(k, v, w, at, n, keep, recent):
    b, t, h, d = k.shape
    ko, vo, wo, po, no = F.evict(k, v, w, at, n, keep, recent=recent)
    assert no.tolist() == [min(max(0, min(x, t)), keep) for x in n.tolist()]
    for i in range(b):
        live = max(0, min(int(n[i]), t))
        for j in range(h):
            kept = select(w[i, j].tolist(), live, keep, recent)
            m, rows = len(kept), torch.tensor(kept, device="cuda", dtype=torch.long)
            assert m == min(live, keep)
            assert torch.equal(ko[i, :m, j], k[i, rows, j]) and torch.equal(vo[i, :m, j], v[i, rows, j])
            assert wo[i, j, :m].tolist() == w[i, j, rows].tolist() or torch.isnan(w[i, j, rows]).any()
            assert po[i, j, :m].tolist() == (rows if at is None else at[i, j, rows]).tolist()
            assert not ko[i, m:, j].any() and not vo[i, m:, j].any() and not wo[i, j, m:].any() and bool((po[i, j, m:] == -1).all())


def cache(kind, b, t, h, d, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((b, t, h, d), generator=g, device="cuda").to(TYPES[kind]) for _ in range(2))
    w = torch.exp(6 * torch.rand((b, h, t), generator=g, device="cuda") - 4)
    at = torch.cumsum(torch.randint(1, 4, (b, h, t), generator=g, device="cuda"), -1).to(torch.int32)
    n = torch.randint(0, t + 1, (b,), generator=g, device="cuda").to(torch.int32)
    n[0] = t
    return k, v, w, at, n


@pytest.mark.parametrize("kind,b,t,h,d", [("bf16", 1, 1, 1, 8), ("fp32", 3, 100, 2, 4), ("fp16", 2, 1025, 3, 64), ("bf16", 2, 5000, 2, 128),
                                          ("fp32", 1, 20000, 1, 20), ("bf16", 4, 257, 5, 200)])
def test_evict(kind, b, t, h, d):
    k, v, w, at, n = cache(kind, b, t, h, d)
    for keep, recent in {(1, 0), (1, 1), (t, 0), (t // 2, t // 4), (t - 1, 0), (t // 2, t // 2), (min(t, 10), min(t, 3)), (0, 0)}:
        if recent <= keep:
            check_evict(k, v, w, at, n, keep, recent)
    check_evict(k, v, w, None, n, t // 2, 0)


def test_evict_ties_and_special_weights():
    k, v, w, at, n = cache("fp16", 3, 3000, 2, 16, seed=1)
    w.copy_((w * 4).floor() / 4)                     # many equal
    for keep in (1, 100, 1500, 2999):
        check_evict(k, v, w, at, n, keep, keep // 3)
    w[:] = 0.0
    w[:, :, ::3] = -0.0                              # equal to 0
    check_evict(k, v, w, at, n, 700, 0)
    w[:, :, 1::7], w[:, :, 2::7], w[:, :, 3::7], w[:, :, 4::7] = math.nan, math.inf, -math.inf, 1e-42
    for keep in (200, 1000, 2800):
        check_evict(k, v, w, at, n, keep, 0)


def test_evict_strides_lengths_and_repeats():
    k, v, w, at, n = cache("bf16", 2, 700, 4, 64, seed=2)
    n[:] = torch.tensor([-5, 10 ** 6], device="cuda")
    check_evict(k, v, w, at, n, 300, 10)
    first = F.evict(k, v, w, at, n, 300, recent=10)
    other = F.evict(k.transpose(1, 2).contiguous().transpose(1, 2), v.transpose(0, 1).contiguous().transpose(0, 1), w, at, n, 300, recent=10)
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = F.evict(k, v, w, at, n, 300, recent=10, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other = F.evict(k, v, w, at, n, 300, recent=10)
    for _ in range(3):
        w.uniform_()
        first = F.evict(k, v, w, at, n, 300, recent=10)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_a_shortened_cache_is_attended_like_its_rows():
    k, v, w, at, n = cache("bf16", 2, 400, 2, 64, seed=3)
    k2, v2, w2, at2, n2 = F.evict(k, v, w, at, n, 150, recent=20)
    q = torch.randn((2, 1, 8, 64), device="cuda").to(torch.bfloat16)
    slopes = torch.exp2(-torch.arange(8, device="cuda").float())
    at_q = at.amax((1, 2)).float().view(2, 1)
    lr = torch.stack([torch.zeros_like(n2), n2 - 1], -1).view(2, 1, 2).contiguous()
    out, w3 = F.attend(q, k2, v2, lr, slopes=slopes, at_q=at_q, at_k=at2.float(), weights=w2)
    ref = Attention(q, k2, v2, lr, slopes=slopes, at_q=at_q, at_k=at2.float())
    near(out, ref.out, ref.out_err, "out")
    near(w3, w2.double() + ref.weights, ref.weights_err + 4e-7 * (w2.double() + ref.weights), "weights")


def test_refusals():
    s, lr = make("bf16", 2, 20, 10, 4, 2, 64, 16, False)
    for bad in (dict(q=s["q"].cpu()), dict(k=s["k"].float()), dict(pages=s["pages"].long()), dict(lengths=s["lengths"][:1]),
                dict(v=s["v"][:5]), dict(lr=torch.zeros((1, 2), dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            F.attend_shared(**{**s, **bad})
    with pytest.raises(F.FrogError) as e:
        F.attend_shared(**s, cap=-2.0)
    assert e.value.code == -1
    k, v, w, at, n = cache("bf16", 2, 50, 2, 64)
    for args, kw in (((k, v, w, at, n, 51), {}), ((k, v, w, at, n, 10), dict(recent=11)), ((k, v[:1], w, at, n, 10), {}),
                     ((k, v, w.double(), at, n, 10), {}), ((k, v, w, at.long(), n, 10), {}), ((k.cpu(), v, w, at, n, 10), {})):
        with pytest.raises(ValueError):
            F.evict(*args, **kw)
    with pytest.raises(F.FrogError) as e:
        F.evict(k[..., :20], v[..., :20], w, at, n, 10)
    assert e.value.code == -7

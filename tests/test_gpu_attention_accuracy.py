"""How far 16-bit results are from 64 bits as a whole, against a result that is
rounded once: by the roundings that are chosen, and no further."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import attention as A  # noqa: E402
from tests.attention_ref import Attention, intervals  # noqa: E402


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def rows(dtype, tokens, h=4, kv=2, d=64, seed=0):
    # some 4,000 query rows whatever their length, so that the norms vary by little
    b = max(1, 1024 // tokens)
    g = torch.Generator(device="cuda").manual_seed(seed + tokens)
    x = [(torch.randn(s, generator=g, device="cuda") * std).to(dtype) for s, std in
         (((b, tokens, h, d), 1.5), ((b, tokens, kv, d), 1.0), ((b, tokens, kv, d), 1.0), ((b, tokens, h, d), 1.0))]
    return (*x[:3], intervals("causal", b, tokens, tokens).cuda(), x[3])


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("tokens", [2, 4, 8, 30, 64, 200, 1024, 2500])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_16_bit_results(dtype, tokens, cap):
    # out and dv have one factor rounded to the type (p) besides the result, dq and dk one (dx): errors of the same size,
    # independent of each other, so the square root of 2 of the single rounding's (1.41); 1.5 allows for the sums and the
    # sample.  delta = dout . out, whatever dout . v is beside it, may add nothing to that.
    q, k, v, lr, dout = rows(dtype, tokens)
    ref = Attention(q, k, v, lr, cap=cap, dout=dout)
    x = [t.requires_grad_() for t in (q, k, v)]
    out = F.attend(*x, lr, cap=cap)
    for what, got in zip(("out", "dq", "dk", "dv"), (out.detach(), *torch.autograd.grad(out, x, dout))):
        want = getattr(ref, what)
        ratio = off(got, want) / off(want.to(dtype), want)
        assert ratio < 1.5, (what, ratio)


@pytest.mark.parametrize("tq,tk", [(1, 300), (1, 3000), (5, 2500), (70, 200), (300, 100), (64, 9000), (3, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
def test_what_the_rounding_of_the_output_left(dtype, tq, tk):
    # through the C entry point, in every kind of pass: out as without it, and out + out_low as near as an output in 32 bits
    b, h, kv, d = 2, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(tq + tk)
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((b, tq, h, d), (b, tk, kv, d), (b, tk, kv, d)))
    out, low = torch.empty((2, b, tq, h, d + 8), device="cuda", dtype=dtype)[..., :d]
    out.fill_(float("nan"))
    low.fill_(float("nan"))
    ws = torch.empty(2 ** 26, device="cuda", dtype=torch.uint8)
    a = A.AttendArgs()
    for n, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        setattr(a, n, t.data_ptr() or None)
        setattr(a, n + "_stride", t.stride()[:3])
    a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type, a.scale = b, tq, tk, h, kv, d, A._TYPES[dtype], d ** -0.5
    a.out_low, a.ws, a.ws_bytes = low.data_ptr(), ws.data_ptr(), ws.numel()
    assert F.lib().frog_attend(C.byref(a), torch.cuda.current_stream().cuda_stream) == 0, F.lib().frog_last_error()
    assert torch.equal(out, F.attend(q, k, v))
    if dtype == torch.float32:
        assert bool(low.isnan().all())       # not looked at
        return
    if tk == 0:
        assert not low.any()
        return
    # the reference's own rounding of p stays in the sum, so the sum is compared with the output in steps of the rounding of out
    half = torch.finfo(dtype).eps / 2
    assert bool((low.float().abs() <= out.float().abs() * half * 1.001 + 2.0 ** -24).all()) and bool(low.any())
    both = off(out.double() + low.double(), Attention(q, k, v).out)
    assert both < off(out, Attention(q, k, v).out)
    a.out_low = low.data_ptr() + 2
    assert F.lib().frog_attend_workspace(C.byref(a), 0) == -1


@pytest.mark.parametrize("b,tq,tk,h,kv,d", [(8, 1, 100, 16, 4, 64), (16, 1, 1001, 16, 4, 128), (8, 1, 5000, 32, 8, 96), (4, 5, 3000, 8, 2, 128), (64, 2, 300, 8, 8, 32)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_16_bit_outputs_of_few_rows(dtype, b, tq, tk, h, kv, d):
    # nothing is rounded on the way but the output: an error of 32-bit sums, 2^-15 and less of the rounding's, only
    # moves values that lie as near to a tie
    g = torch.Generator(device="cuda").manual_seed(tk)
    q, k, v = ((torch.randn(s, generator=g, device="cuda") * std).to(dtype) for s, std in (((b, tq, h, d), 1.5), ((b, tk, kv, d), 1.0), ((b, tk, kv, d), 1.0)))
    ref = Attention(q, k, v)
    assert off(F.attend(q, k, v), ref.out) < 1.05 * off(ref.out.to(dtype), ref.out)
    out, w = F.attend(q, k, v, weights=torch.zeros((b, kv, tk), device="cuda"), cap=20.0)
    ref = Attention(q, k, v, cap=20.0)
    assert off(out, ref.out) < 1.05 * off(ref.out.to(dtype), ref.out)


@pytest.mark.parametrize("b,prefix,tail,h,kv,d", [(4, 700, 60, 16, 4, 64), (3, 3000, 200, 8, 2, 128), (6, 3000, 100, 8, 2, 96), (3, 0, 900, 40, 1, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_16_bit_outputs_over_a_shared_prefix(dtype, b, prefix, tail, h, kv, d):
    g = torch.Generator(device="cuda").manual_seed(prefix)
    q, k, v = ((torch.randn(s, generator=g, device="cuda") * std).to(dtype) for s, std in (((b, h, d), 1.5), ((prefix, kv, d), 1.0), ((prefix, kv, d), 1.0)))
    pages = torch.randperm(b * tail, generator=g, device="cuda").to(torch.int32).view(b, tail)
    kp, vp = (torch.randn((b * tail, 1, kv, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    out = F.attend_shared(q, k, v, kp, vp, pages, torch.full((b,), tail, device="cuda", dtype=torch.int32))
    own = [torch.cat([x.expand(b, prefix, kv, d), p[pages.long(), 0]], 1) for x, p in ((k, kp), (v, vp))]
    ref = Attention(q.unsqueeze(1), *own)
    assert off(out.unsqueeze(1), ref.out) < 1.05 * off(ref.out.to(dtype), ref.out)

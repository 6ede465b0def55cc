"""The ways a call is cut that depend on the number of heads a key head serves,
on long prefixes of few requests and on where a single launch ends; pages
without a number; and intervals as the filtered search writes them."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from tests import test_gpu_attention as one  # noqa: E402
from tests import test_gpu_cache as many  # noqa: E402
from tests.attention_ref import Attention, near  # noqa: E402

TYPES = list(many.TYPES)


def slopes(h):
    return torch.exp2(-8.0 * torch.arange(1, h + 1, device="cuda") / h)


# batch, prefix, longest tail, heads, kv heads, d, page
SHARED = [(3, 3000, 100, 8, 2, 128, 16),     # at most 16 query rows a kv head over a long prefix
          (6, 3000, 100, 8, 2, 128, 16),     # 17 to 32
          (1, 2500, 300, 16, 1, 64, 7), (1, 3000, 200, 32, 1, 96, 16), (2, 1100, 0, 16, 2, 32, 16),
          (2, 300, 50, 20, 1, 64, 16),       # groups of 17 to 32 heads, prefix and tails in one launch
          (3, 500, 90, 40, 1, 128, 16),      # above 32: several workgroups a group
          (2, 200, 100, 70, 2, 32, 5), (3, 0, 60, 33, 1, 96, 16),
          (2, 2600, 300, 40, 1, 64, 16),     # the same over a long prefix and long tails
          (5, 1500, 400, 20, 1, 128, 32), (4, 1200, 1300, 48, 1, 32, 16),
          (2, 1000, 24, 4, 2, 64, 8), (2, 1001, 24, 4, 2, 64, 8),
          (4, 400, 112, 16, 4, 128, 16), (4, 420, 112, 16, 4, 128, 16), (4, 0, 700, 8, 2, 128, 16)]   # prefix and tail of 1,024 rows, and one more


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHARED, ids=str)
def test_shared(kind, shape):
    print(f"[gpu] shared prefix {kind} {shape}", flush=True)
    for n, (cap, bias, ranges) in enumerate(((0.0, False, False), (5.0, True, True), (0.0, True, False), (5.0, False, True))):
        s, lr = many.make(kind, *shape, ranges and shape[1] > 0, seed=10 + n)
        many.check(s, lr, cap, slopes(shape[3]) if bias else None)


@pytest.mark.parametrize("prefix,width,h,kv", [(200, 6, 8, 2), (3000, 6, 8, 2), (3000, 90, 40, 1), (0, 90, 4, 2)])
@pytest.mark.parametrize("kind", TYPES)
def test_pages_without_a_number_count_as_no_rows(kind, prefix, width, h, kv):
    page, b = 16, 3
    s, _ = many.make(kind, b, prefix, width * page, h, kv, 64, page, False, seed=3)
    s["lengths"][:] = torch.tensor([width * page, width * page - 5, 2 * page + 1])
    num = s["k_pages"].shape[0]
    gone = {(0, 1): -1, (0, width - 1): num, (1, 0): 2 ** 31 - 1, (1, width // 2): -2 ** 31, (2, 0): -1, (2, 1): num + 7, (2, 2): -9}
    for (i, p), x in gone.items():
        s["pages"][i, p] = x
    sl = slopes(h)
    out, lse = F.attend_shared(**s, slopes=sl, return_lse=True)
    for i in range(b):
        n = int(s["lengths"][i])
        t = torch.tensor([t for t in range(n) if (i, t // page) not in gone], device="cuda", dtype=torch.long)
        at = torch.cat([torch.arange(prefix, device="cuda"), prefix + t])
        pages = s["pages"][i].long()[t // page]
        k, v = (torch.cat([s[x], s[x + "_pages"][pages, t % page]]).unsqueeze(0) for x in ("k", "v"))
        ref = Attention(s["q"][i].view(1, 1, h, 64), k, v, slopes=sl, at_q=torch.full((1, 1), float(prefix + n - 1), device="cuda"), at_k=at.float().unsqueeze(0))
        near(out[i].view(ref.out.shape), ref.out, ref.out_err, f"request {i} out")
        near(lse[i].view(ref.lse.shape), ref.lse, ref.lse_err, f"request {i} lse")


# b, tq, tk, h, kv, d: 17 to 32 query rows a kv head, in one part and in many; a single launch's last key and one more
FEW = [(1, 5, 3000, 8, 2, 128), (2, 1, 2500, 20, 1, 64), (1, 1, 1500, 32, 1, 96), (3, 8, 129, 8, 2, 32), (2, 3, 700, 10, 1, 128),
       (1, 2, 1024, 8, 2, 64), (1, 2, 1025, 8, 2, 64), (1, 33, 300, 1, 1, 64),
       (64, 1, 1000, 4, 4, 64), (2, 1, 600, 8, 2, 128), (1, 3, 500, 4, 1, 128)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", FEW, ids=str)
def test_few_rows(kind, shape):
    print(f"[gpu] few rows {kind} {shape}", flush=True)
    for n, (cap, bias) in enumerate(itertools.product((0.0, 5.0), (False, True))):
        mask = ("causal", "wild", "lengths", "window")[(FEW.index(shape) + n) % 4]
        s, opt, dout = one.make(kind, *shape, mask, bias, seed=100 + n)
        one.check(s, opt, dout, cap, f"{mask} cap {cap} bias {bias}")


def test_intervals_of_the_filtered_search():
    # rank_bounds of attribute ranges are the intervals of attention over the rows in attribute order
    import numpy as np
    n, nq, h, kv, d = 700, 90, 4, 2, 64
    r = np.random.default_rng(5)
    attr = np.sort(r.integers(0, 300, n).astype(np.float64))           # with equal ones
    ix = F.Index.build(r.standard_normal((n, 32)).astype(np.float32), attr).upload(0)
    lo = r.integers(-20, 320, nq).astype(np.float64)
    hi = lo + r.integers(-5, 150, nq)
    lo[3], hi[5] = np.nan, np.nan
    lr = F.rank_bounds(ix, torch.as_tensor(lo, device="cuda"), torch.as_tensor(hi, device="cuda"))
    s, _, dout = one.make("bf16", 1, nq, n, h, kv, d, None, seed=7)
    s["lr"] = lr
    one.check(s, {}, dout, 0.0, "ranks")
    # against the ranges themselves
    seen = torch.as_tensor((attr >= lo[:, None]) & (attr <= hi[:, None]), device="cuda")
    weights = torch.zeros((1, kv, n), device="cuda")
    out, weights = F.attend(s["q"], s["k"], s["v"], lr, weights=weights)
    k, v = (s[x].double().transpose(1, 2).repeat_interleave(h // kv, 1) for x in ("k", "v"))
    z = (s["q"].double().transpose(1, 2) @ k.transpose(2, 3) * d ** -0.5).masked_fill(~seen, -float("inf"))
    p = torch.softmax(z, -1).nan_to_num(0.0)
    ref = Attention(s["q"], s["k"], s["v"], lr.unsqueeze(0))
    near(out, (p @ v).transpose(1, 2), ref.out_err, "out")
    near(weights, p.view(1, kv, -1, n).sum(2), ref.weights_err, "weights")
    one_token = F.attend(s["q"][:, 7:8].contiguous(), s["k"], s["v"], lr[7:8].contiguous())
    near(one_token, (p @ v).transpose(1, 2)[:, 7:8], ref.out_err[:, 7:8], "one token")


@pytest.mark.parametrize("tq", [1, 3, 70, 200])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (5.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("kind", TYPES)
def test_queries_without_keys_may_hold_anything(kind, cap, bias, tq):
    # rows of padding between rows that see keys: their q, dout and attribute, and the attributes of keys nobody sees
    s, opt, dout = one.make(kind, 2, tq, 150, 4, 2, 64, "causal", bias, seed=17)
    pad = torch.arange(tq, device="cuda") % 3 == 1 if tq > 1 else torch.ones(1, device="cuda", dtype=torch.bool)
    s["lr"][..., 0], s["lr"][..., 1] = 20, s["lr"][..., 1].clamp(max=110)
    s["lr"][0, pad] = torch.tensor([70, 60], device="cuda", dtype=torch.int32)
    what = (math.nan, math.inf, -math.inf)
    clean = dict(s, q=s["q"].clone()), {n: t.clone() for n, t in opt.items()}, dout.clone()
    clean[0]["q"][0, pad], clean[2][0, pad] = 0, 0
    for n, x in enumerate(what):
        s["q"][0, pad, n], dout[0, pad, n + 1] = x, x
        if bias:
            opt["at_q"][0, pad] = x
            opt["at_k"][:, :, 3 * n:20:2], opt["at_k"][:, :, 111 + n::3] = x, x
    if bias:
        clean[1]["at_q"][0, pad], clean[1]["at_k"][:, :, :20], clean[1]["at_k"][:, :, 111:] = 0, 0, 0

    ref = Attention(*(clean[0][n] for n in ("q", "k", "v", "lr")), cap=cap, dout=clean[2], **clean[1])
    x = [s[n].detach().requires_grad_() for n in ("q", "k", "v")]
    out, lse, w = F.attend(*x, s["lr"], cap=cap, return_lse=True, weights=torch.zeros((2, 2, 150), device="cuda"), **opt)
    grads = torch.autograd.grad(out, x, dout)
    for what, got in zip(("out", "lse", "weights", "dq", "dk", "dv"), (out, lse, w, *grads)):
        near(got, getattr(ref, what), getattr(ref, what + "_err"), what)
    assert not out[0, pad].any() and not grads[0][0, pad].any() and bool((lse[0, :, pad] == -math.inf).all())

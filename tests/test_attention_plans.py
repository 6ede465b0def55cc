"""Which calls order their tiles by length (a small launch of its own in front
of a pass): the workspace then holds the order."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import attention as A  # noqa: E402


F32, BF16 = 0, 2


def workspace(backward, lr, batch, tokens, heads, kv, d, type_=BF16, keys=None):
    a = A.AttendArgs()
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(a, n, 4096)
        setattr(a, n + "_stride", (0, d * heads, d))
    a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type, a.scale = batch, tokens, keys or tokens, heads, kv, d, type_, 0.125
    a.lr, a.lse = 4096 if lr else None, 4096
    n = F.lib().frog_attend_workspace(C.byref(a), backward)
    assert n >= 0, F.lib().frog_last_error()
    return n


# batch, tokens, heads, kv heads, d, type, and whether rows (forward), keys and rows (gradients) are ordered
@pytest.mark.parametrize("batch,tokens,heads,kv,d,type_,rows,keys,dq", [
    (1, 8192, 16, 4, 128, BF16, True, True, True), (1, 8191, 12, 12, 96, BF16, True, True, True), (1, 32768, 16, 4, 128, BF16, True, True, True),
    (4, 8192, 16, 4, 64, BF16, True, True, True), (1, 4096, 16, 4, 128, BF16, False, False, False), (1, 2048, 32, 8, 128, BF16, False, False, False),
    (1, 8192, 8, 1, 64, BF16, False, False, False), (1, 16384, 8, 1, 64, BF16, True, False, True), (64, 2048, 4, 4, 64, BF16, False, False, False),
    (1024, 2048, 2, 2, 64, BF16, False, False, False), (4096, 2048, 1, 1, 32, BF16, False, False, False), (8, 8192, 8, 2, 64, BF16, False, False, False),
    (1, 4096, 16, 4, 64, F32, True, True, True), (1, 4096, 8, 8, 64, F32, True, True, False), (1, 2048, 8, 8, 64, F32, False, False, False),
    (1, 1500, 32, 4, 128, F32, False, False, False), (16, 2048, 4, 4, 64, F32, True, True, True)])
def test_orders_are_made_where_they_pay(batch, tokens, heads, kv, d, type_, rows, keys, dq):
    order = [workspace(b, True, batch, tokens, heads, kv, d, type_) - workspace(b, False, batch, tokens, heads, kv, d, type_) for b in (0, 1)]
    row_tiles, key_tiles = -(-tokens * (heads // kv) // 128) * batch, -(-tokens // 128) * batch
    size = [-(-4 * n // 256) * 256 for n in (row_tiles, key_tiles)]
    assert order[0] == (size[0] if rows else 0)
    assert order[1] == (size[0] if dq else 0) + (size[1] if keys else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("mask", ["documents", "one", "lengths", "empty", "wild"])
@pytest.mark.parametrize("type_,batch,tq,tk,d", [(BF16, 1, 6500, 6144, 128), (F32, 1, 2600, 2500, 96), (F32, 2, 2100, 2304, 64)])
def test_ordered_passes(mask, type_, batch, tq, tk, d):
    # sizes whose tiles are ordered, each group of heads against the formulas in 64 bits
    from tests.attention_ref import Attention, intervals, near
    h, kv = 14, 7
    for backward in (0, 1):
        assert workspace(backward, True, batch, tq, h, kv, d, type_, tk) > workspace(backward, False, batch, tq, h, kv, d, type_, tk)
    print(f"[gpu] ordered passes {mask} {batch} x {tq} x {tk}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tq)
    q, k, v, dout = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16 if type_ == BF16 else torch.float32)
                     for s in ((batch, tq, h, d), (batch, tk, kv, d), (batch, tk, kv, d), (batch, tq, h, d)))
    lr = intervals("causal" if mask == "one" else mask, batch, tq, tk, 5).cuda()
    if mask == "one":
        # a few rows see every key, the others one
        lr[:, :, 0] = lr[:, :, 1] = lr[:, :, 1].clamp(min=0)
        lr[:, 700:704, 0], lr[:, 700:704, 1] = 0, tk - 1
    x = [t.requires_grad_() for t in (q, k, v)]
    out, lse, w = F.attend(*x, lr, return_lse=True, weights=torch.zeros((batch, kv, tk), device="cuda"))
    grads = torch.autograd.grad(out, x, dout)
    for b in range(batch):
        for i in range(kv):
            hs = slice(i * h // kv, (i + 1) * h // kv)
            ref = Attention(q[b:b + 1, :, hs].detach(), k[b:b + 1, :, i:i + 1].detach(), v[b:b + 1, :, i:i + 1].detach(), lr[b:b + 1], dout=dout[b:b + 1, :, hs])
            got = (out[b:b + 1, :, hs], lse[b:b + 1, hs], w[b:b + 1, i:i + 1], grads[0][b:b + 1, :, hs], grads[1][b:b + 1, :, i:i + 1], grads[2][b:b + 1, :, i:i + 1])
            for what, y in zip(("out", "lse", "weights", "dq", "dk", "dv"), got):
                near(y, getattr(ref, what), getattr(ref, what + "_err"), f"{mask} {what}")


# batch, keys, heads, kv heads, d, type, key weights, and whether one launch takes all (no workspace)
@pytest.mark.parametrize("batch,keys,heads,kv,d,type_,weights,whole", [
    (1, 128, 16, 4, 128, F32, False, True), (1, 256, 16, 4, 128, F32, False, True), (1, 257, 16, 4, 128, F32, False, False),
    (1, 512, 16, 4, 128, BF16, False, True), (1, 1024, 16, 4, 128, BF16, False, True), (1, 1024, 16, 4, 64, BF16, False, True),
    (1, 1025, 16, 4, 32, BF16, False, False), (64, 1024, 16, 4, 128, F32, False, True), (63, 1024, 16, 4, 128, F32, False, False),
    (1, 512, 16, 4, 128, BF16, True, True), (1, 700, 16, 4, 128, F32, True, False), (64, 512, 16, 4, 128, BF16, True, True)])
def test_short_caches_are_cut_where_that_pays(batch, keys, heads, kv, d, type_, weights, whole):
    a = A.AttendArgs()
    for n in ("q", "k", "v", "out"):
        setattr(a, n, 4096)
        setattr(a, n + "_stride", (0, d * heads, d))
    a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type, a.scale = batch, 1, keys, heads, kv, d, type_, 0.125
    scores = 0
    if weights:
        a.w_out = a.lse = 4096
        scores = -(-batch * heads * keys * 4 // 256) * 256
    assert (F.lib().frog_attend_workspace(C.byref(a), 0) == scores) == whole


@pytest.mark.parametrize("batch,prefix,tail,heads,kv,d,type_,whole", [
    (4, 700, 64, 16, 4, 64, BF16, True), (4, 400, 112, 16, 4, 128, BF16, True), (4, 656, 113, 16, 4, 128, BF16, False), (4, 200, 57, 16, 4, 128, F32, False),
    (16, 900, 64, 16, 4, 128, F32, True), (4, 0, 520, 16, 4, 128, F32, False), (64, 0, 1000, 16, 4, 128, BF16, True), (4, 960, 65, 16, 4, 32, BF16, False)])
def test_short_shared_prefixes_are_cut_where_that_pays(batch, prefix, tail, heads, kv, d, type_, whole):
    a = A.SharedArgs()
    for n in ("q", "k", "v", "out"):
        setattr(a, n, 4096)
        setattr(a, n + "_stride", (d * heads, d))
    a.k_pages = a.v_pages = a.pages = a.lengths = 4096
    a.k_pages_stride = a.v_pages_stride = (d * heads, d * heads, d)
    a.batch, a.prefix, a.num_pages, a.pages_per_request, a.page, a.heads, a.kv_heads, a.d, a.type, a.scale = batch, prefix, 4, tail, 1, heads, kv, d, type_, 0.125
    assert (F.lib().frog_attend_shared_workspace(C.byref(a)) == 0) == whole

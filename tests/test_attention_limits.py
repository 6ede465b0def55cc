"""Sizes at which a launch of the attention section ends: calls below them run,
calls above are refused before anything is enqueued, by the workspace query
too."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import attention as A  # noqa: E402


def rows(a, names, strides):
    for n in names:
        setattr(a, n, 4096)
        setattr(a, n + "_stride", strides)


def attend_args(**kw):
    a = A.AttendArgs()
    rows(a, ("q", "k", "v", "out", "dout", "dq", "dk", "dv"), (0, 64, 64))
    a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type, a.scale = 2, 3, 5, 1, 1, 64, 2, 0.125
    a.lse = 4096
    for k, v in kw.items():
        setattr(a, k, v)
    return a


# single tokens: 512 threads a (sequence, kv head); longer: 256 threads 128 rows or keys
SIZES = [(dict(batch=2 ** 23, queries=1, keys=64), dict(batch=2 ** 23 - 1, queries=1, keys=64), 0),
         (dict(batch=2 ** 12, queries=2 ** 19, keys=64), dict(batch=2 ** 12 - 1, queries=2 ** 19, keys=64), 0),
         (dict(batch=2 ** 12, queries=2 ** 19, keys=64), dict(batch=2 ** 12 - 1, queries=2 ** 19, keys=64), 1),
         (dict(batch=2 ** 12, queries=64, keys=2 ** 19), dict(batch=2 ** 12 - 1, queries=64, keys=2 ** 19), 1),
         (dict(batch=2 ** 12, queries=64, keys=2 ** 19, w_out=4096), dict(batch=2 ** 12 - 1, queries=64, keys=2 ** 19, w_out=4096), 0)]


@pytest.mark.parametrize("above,below,backward", SIZES, ids=str)
def test_the_workspace_query_tells_which_sizes_run(above, below, backward):
    L = F.lib()
    fn = L.frog_attend_backward if backward else L.frog_attend
    assert L.frog_attend_workspace(C.byref(attend_args(**above)), backward) == -7 and b"launch" in L.frog_last_error()
    assert fn(C.byref(attend_args(**above)), None) == -7
    assert L.frog_attend_workspace(C.byref(attend_args(**below)), backward) >= 0


def test_shared_prefixes_of_many_requests():
    a = A.SharedArgs()
    rows(a, ("q", "k", "v", "out"), (64, 64))
    rows(a, ("k_pages", "v_pages"), (1024, 64, 64))
    a.pages = a.lengths = 4096
    a.prefix, a.num_pages, a.pages_per_request, a.page, a.heads, a.kv_heads, a.d, a.type, a.scale = 10, 4, 1, 16, 1, 1, 64, 1, 0.125
    for batch, code in ((2 ** 24, -7), (2 ** 24 - 1, 0)):
        a.batch = batch
        assert min(0, F.lib().frog_attend_shared_workspace(C.byref(a))) == code


@pytest.mark.gpu
def test_a_large_batch_of_long_sequences():
    # 64 sequences of 8,192 tokens and 64 heads: 2^25 query rows and keys, which need neither parts nor joins.  The
    # sequences are one sequence repeated, so that each has to come out like it alone.
    print("[gpu] attention of 64 x 8,192 tokens, 64 heads, d = 128", flush=True)
    b, t, h, d = 64, 8192, 64, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    one = [torch.randn((1, t, h, d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16) for _ in range(4)]
    place = torch.arange(t, device="cuda", dtype=torch.int32)
    lr = torch.stack([(place - 20).clamp(min=0), place], -1)
    x = [y.detach().requires_grad_() for y in one[:3]]
    o = F.attend(*x, lr)
    want = [o.detach(), *torch.autograd.grad(o, x, one[3])]
    x = [y.expand(b, t, h, d).detach().requires_grad_() for y in one[:3]]
    o = F.attend(*x, lr)
    assert all(torch.equal(o[i], want[0][0]) for i in range(b))
    got = torch.autograd.grad(o, x, one[3].expand(b, t, h, d))
    for a, w in zip(got, want[1:]):
        assert all(torch.equal(a[i], w[0]) for i in range(b))


@pytest.mark.gpu
def test_evict_of_more_caches_than_a_launch_takes():
    # 2^22 workgroups of 1,024 threads are one more than a launch takes
    b, h, t, d = 2 ** 16 + 1, 64, 2, 8
    print(f"[gpu] eviction from {b * h} caches", flush=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((b, t, h, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.rand((b, h, t), generator=g, device="cuda")
    n = torch.randint(0, t + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    n[-1] = t
    ko, vo, wo, po, no = F.evict(k, v, w, None, n, 1)
    assert torch.equal(no, n.clamp(max=1))
    best = torch.where(n.view(b, 1) == t, (w[..., 1] > w[..., 0]).int(), torch.where(n.view(b, 1) == 1, 0, -1))     # [b, h]
    assert torch.equal(po[..., 0], best)
    take = best.clamp(min=0).long()
    assert torch.equal(wo, torch.where(best.unsqueeze(-1) >= 0, w.gather(2, take.unsqueeze(-1)), 0.0))
    rows_of = take.view(b, 1, h, 1).expand(b, 1, h, d)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got, torch.where(best.view(b, 1, h, 1) >= 0, x.gather(1, rows_of), 0))


@pytest.mark.gpu
def test_evict_of_more_values_than_a_launch_copies():
    # 2^32 pieces of 16 bytes and one row more, of a cache whose slots are one row in memory; k and v out are one buffer
    slots, d = 1025, 2 ** 24
    print(f"[gpu] eviction of {slots} rows of {d} values", flush=True)
    row = torch.randn(d, device="cuda")
    out = torch.full((slots, d), float("nan"), device="cuda")
    w = torch.rand(slots, device="cuda")
    n = torch.full((1,), slots, device="cuda", dtype=torch.int32)
    w_out, at, n_out, ws = torch.empty_like(w), torch.empty(slots, device="cuda", dtype=torch.int32), torch.empty_like(n), torch.empty(slots, device="cuda")
    a = A.EvictArgs()
    a.k = a.v = row.data_ptr()
    a.k_stride = a.v_stride = (0, 0, 0)
    a.weights, a.lengths, a.k_out, a.v_out, a.weights_out = w.data_ptr(), n.data_ptr(), out.data_ptr(), out.data_ptr(), w_out.data_ptr()
    a.positions_out, a.lengths_out, a.ws, a.ws_bytes = at.data_ptr(), n_out.data_ptr(), ws.data_ptr(), 4 * slots
    a.batch, a.slots, a.keep, a.heads, a.d, a.type = 1, slots, slots, 1, d, F.STORAGE_F32
    assert F.lib().frog_evict(C.byref(a), torch.cuda.current_stream().cuda_stream) == 0, F.lib().frog_last_error()
    torch.cuda.synchronize()
    assert int(n_out) == slots and torch.equal(w_out, w) and torch.equal(at, torch.arange(slots, device="cuda", dtype=torch.int32))
    assert all(torch.equal(out[i], row) for i in range(slots))


@pytest.mark.gpu
def test_outputs_of_passes_without_keys_or_queries_above_one_launch():
    # 17 sequences whose outputs lie on one another: 2^32 + 2^28 pieces of 16 bytes are set to 0
    tokens, heads, d = 2 ** 20, 64, 32
    print("[gpu] passes without keys and without queries", flush=True)
    out = torch.full((tokens, heads, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    stream = torch.cuda.current_stream().cuda_stream
    strides = (0, heads * d, d)
    a = attend_args(batch=17, queries=tokens, keys=0, heads=heads, kv_heads=heads, d=d, lse=None, q=out.data_ptr(), q_stride=strides,
                    out=out.data_ptr(), out_stride=strides)
    assert F.lib().frog_attend(C.byref(a), stream) == 0, F.lib().frog_last_error()
    torch.cuda.synchronize()
    assert not out.any()
    # 2^32 weights of keys that no query saw
    w = torch.full((2 ** 32,), float("nan"), device="cuda")
    a = attend_args(batch=1, queries=0, keys=2 ** 26, heads=64, kv_heads=64, d=32, lse=None, k=out.data_ptr(), v=out.data_ptr(), w_out=w.data_ptr())
    assert F.lib().frog_attend(C.byref(a), stream) == 0, F.lib().frog_last_error()
    torch.cuda.synchronize()
    assert bool((w == 0).all())

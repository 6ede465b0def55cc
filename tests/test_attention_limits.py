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

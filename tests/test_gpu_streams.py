"""Workspaces and streams of the attention entry points and of the search."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
import workloads  # noqa: E402
from paper_2608_16491_amd import attention as A  # noqa: E402

PER_THREAD = 2       # the handle hipStreamPerThread: in each thread another stream


def inputs(n, keys):
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((2, 1, 8, 128), (2, keys, 2, 128), (2, keys, 2, 128)))
    return q, k, v, torch.rand((2, 2, keys), generator=g, device="cuda"), torch.full((2,), keys, device="cuda", dtype=torch.int32)


def passes(q, k, v, w, lengths):
    """Calls whose workspace holds parts, scores and slot lists."""
    out, new = F.attend(q, k, v, weights=w)
    return out, new, *F.evict(k, v, w, None, lengths, 1000, recent=10)


def test_threads_on_the_stream_of_each_thread(monkeypatch):
    # sizes that grow from thread to thread and from call to call, results against the default stream's
    print("[gpu] four threads on hipStreamPerThread", flush=True)
    cases = [[inputs(10 * t + i, 3000 + 700 * t + 300 * i) for i in range(3)] for t in range(4)]
    want = [[passes(*x) for x in own] for own in cases]
    torch.cuda.synchronize()
    monkeypatch.setattr(A, "_current", lambda index: PER_THREAD)
    got, start = [None] * 4, threading.Barrier(4)

    def work(t):
        start.wait()
        got[t] = [[passes(*x) for x in cases[t]] for _ in range(8)]

    threads = [threading.Thread(target=work, args=(t,)) for t in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for t in range(4):
        assert got[t] is not None
        for outs in got[t]:
            for a, b in zip(outs, want[t]):
                assert all(torch.equal(x, y) for x, y in zip(a, b)), t


def test_search_on_the_stream_of_each_thread():
    w = workloads.make("c2", n=5000, nq=60)
    ix = F.Index.build(w.X, w.attr).upload(0)
    args = [torch.as_tensor(x, device="cuda") for x in (w.Q, w.lo, w.hi)]
    want = F.search(ix, *args, 10, 32)
    torch.cuda.synchronize()
    got = [F.search(ix, *args, 10, 32, stream=torch.cuda.ExternalStream(PER_THREAD)) for _ in range(3)]
    torch.cuda.synchronize()
    for a in got:
        assert all(torch.equal(x, y) for x, y in zip(a, want))


def test_a_captured_call_takes_the_callers_workspace(monkeypatch):
    # the binding brings one; without it the call is refused, and so is none that needs no workspace
    q, k, v, w, lengths = inputs(1, 3000)
    shared = dict(q=q[:, 0].contiguous(), k=k[0], v=v[0], k_pages=k[:, :64].contiguous(), v_pages=v[:, :64].contiguous(),
                  pages=torch.zeros((2, 1), device="cuda", dtype=torch.int32), lengths=torch.ones(2, device="cuda", dtype=torch.int32))
    calls = (lambda: F.attend(q, k, v), lambda: F.attend(q, k, v, weights=w), lambda: F.attend_shared(**shared),
             lambda: F.evict(k, v, w, None, lengths, 1000))
    want = [f() for f in calls]
    small = F.attend(q, k[:, :100].contiguous(), v[:, :100].contiguous())
    ks, vs = k[:, :100].contiguous(), v[:, :100].contiguous()
    codes = []
    with monkeypatch.context() as m:
        m.setattr(A, "_own_workspace", lambda large: False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for f in calls:
                try:
                    f()
                except F.FrogError as e:
                    codes.append(e.code)
            got = F.attend(q, ks, vs)
        assert codes == [-1] * 4
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, small)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [f() for f in calls]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)))

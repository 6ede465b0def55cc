"""The cache in 8-bit pages in calls large enough for the kernels and rules that
small ones do not meet."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import paged as G  # noqa: E402


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

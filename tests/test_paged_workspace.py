"""What the binding takes an attention call's workspace to be at most, against
the library's own figure."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import paged as G  # noqa: E402
from tests.test_paged_abi import args  # noqa: E402


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (32, 8), (34, 2), (64, 1)])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_no_call_takes_more(kind, heads, kv_heads, page):
    met = False
    for batch in (1, 2, 7, 40, 700):
        for pages in (0, 1, 4, 5, 17, 63, 64, 65, 100, 257, 1000, 4097, 20_000, 300_001):
            for listed in (False, True):
                a = args(G.PagedArgs, heads=heads, type=kind, batch=batch, chosen=4096 if listed else None,
                         num_chosen=pages if listed else 0, pages_per_request=9 if listed else pages,
                         **{"cache.kv_heads": kv_heads, "cache.page": page, "cache.d": 128})
                n = F.lib().frog_attend_paged_workspace(C.byref(a))
                assert 0 <= n <= G._most_workspace(batch, heads, 128, pages * page), (batch, pages, listed)
                met |= n > 2 ** 26
    assert met                                  # (sizes above what a call may leave with the library are among them)

"""The paged-cache section of the C ABI on the host: struct layouts of the
binding against include/frog.h, refusals before any GPU is touched, and the
definition the GPU's results are compared with."""
import ctypes as C
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import paged as G  # noqa: E402
from tests.paged_ref import quantise  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = (("frog_cache_write_t", G.WriteArgs), ("frog_cache_read_t", G.ReadArgs), ("frog_select_pages_t", G.SelectArgs),
         ("frog_attend_paged_t", G.PagedArgs))


def test_struct_layouts_match_the_header(tmp_path):
    lines, want = [], []
    for name, cls in PAIRS:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for f in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f[0]}));')
            want.append(getattr(cls, f[0]).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include "frog.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", f"-I{ROOT}/include", str(src), "-o", exe], check=True)
    assert [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()] == want


def args(cls, **kw):
    a = cls()
    base = {"cache.k": 4096, "cache.v": 4096, "cache.k_exp": 4096, "cache.v_exp": 4096, "cache.bounds": 4096, "cache.num_pages": 9,
            "cache.kv_heads": 2, "cache.page": 16, "cache.d": 64, "cache.storage": 1, "type": 2, "batch": 3, "pages": 4096, "lengths": 4096,
            "pages_per_request": 4, "tokens": 6, "slots": 5, "heads": 4, "chosen": 4096, "keep": 3, "recent": 1, "scale": 0.125}
    for n in ("q", "k", "v", "out"):
        base[n] = 4096
        base[n + "_stride"] = (4096, 256, 64)
    names = {f[0]: f[1] for f in cls._fields_}
    for k, v in {**base, **kw}.items():
        if k in names:
            setattr(a, k, v[:names[k]._length_] if isinstance(v, tuple) else v)
    return a


CACHE = [({"cache.storage": 2}, -1), ({"cache.page": 24}, -1), ({"cache.page": 8}, -1), ({"cache.d": 80}, -7), ({"cache.d": 256}, -7),
         ({"cache.kv_heads": 0}, -1), ({"cache.num_pages": -1}, -1), ({"cache.num_pages": 2 ** 31}, -7), ({"cache.num_pages": 2 ** 30}, -7), ({"type": 3}, -1),
         ({"batch": -1}, -1), ({"pages_per_request": -1}, -1), ({"pages": None}, -1), ({"lengths": None}, -1),
         ({"pages_per_request": 2 ** 27}, -7), ({"batch": 2 ** 31}, -7)]
ROWS = [({"cache.k": None}, -1), ({"cache.v_exp": None}, -1), ({"cache.k": 4100}, -1), ({"cache.k_exp": 4104}, -1)]
CALLS = {
    "frog_cache_write": (G.WriteArgs, CACHE + ROWS + [({"k": None}, -1), ({"v": 4104}, -1), ({"k_stride": (100, 64)}, -1), ({"tokens": 7}, -1),
                                                     ({"tokens": -1}, -1), ({"tokens": 2 ** 31}, -7), ({"cache.bounds": 4100}, -1)]),
    "frog_cache_read": (G.ReadArgs, CACHE + ROWS + [({"k": None}, -1), ({"v_stride": (64, -64, 64)}, -1), ({"slots": -1}, -1), ({"slots": 2 ** 31}, -7)]),
    "frog_select_pages": (G.SelectArgs, CACHE + [({"cache.bounds": None}, -1), ({"cache.bounds": 4104}, -1), ({"q": None}, -1), ({"heads": 3}, -1),
                                                 ({"heads": 0}, -1), ({"first": 3}, -1), ({"first": -1}, -1), ({"recent": -1}, -1), ({"keep": 0}, -1),
                                                 ({"keep": 2 ** 31}, -7), ({"chosen": None}, -1), ({"heads": 2 ** 17}, -7)]),
    "frog_attend_paged": (G.PagedArgs, CACHE + ROWS + [({"q": 4104}, -1), ({"q_stride": (100, 64)}, -1), ({"heads": 5}, -1), ({"out": None}, -1),
                                                       ({"num_chosen": -1}, -1), ({"num_chosen": 2 ** 29}, -7), ({"scale": float("nan")}, -1),
                                                       ({"cap": -1.0}, -1), ({"cap": float("inf")}, -1), ({"out_stride": (4100, 64)}, -1)]),
}


@pytest.mark.parametrize("fn,kw,code", [(fn, kw, code) for fn, (_, bad) in CALLS.items() for kw, code in bad], ids=str)
def test_refusals(fn, kw, code):
    L, a = F.lib(), args(CALLS[fn][0], **kw)
    assert getattr(L, fn)(C.byref(a), None) == code and L.frog_last_error()
    if hasattr(L, fn + "_workspace"):
        assert getattr(L, fn + "_workspace")(C.byref(a)) == code


@pytest.mark.parametrize("fn", CALLS)
def test_no_arguments(fn):
    assert getattr(F.lib(), fn)(None, None) == -1


def test_workspaces():
    L = F.lib()
    # one launch while a request's rows (pages) are few, parts of them else
    assert L.frog_attend_paged_workspace(C.byref(args(G.PagedArgs, chosen=None, pages_per_request=64))) == 0
    assert L.frog_attend_paged_workspace(C.byref(args(G.PagedArgs, chosen=None, pages_per_request=4096))) > 0
    assert L.frog_attend_paged_workspace(C.byref(args(G.PagedArgs, num_chosen=8, pages_per_request=4096))) == 0
    assert L.frog_select_pages_workspace(C.byref(args(G.SelectArgs, pages_per_request=100))) == 0
    assert L.frog_select_pages_workspace(C.byref(args(G.SelectArgs, pages_per_request=10_000))) == 3 * 2 * 10_000 * 4
    # a workspace too small, or off its boundary
    a = args(G.PagedArgs, chosen=None, pages_per_request=4096, ws=4096, ws_bytes=16)
    assert L.frog_attend_paged(C.byref(a), None) == -1 and b"workspace" in L.frog_last_error()
    a = args(G.PagedArgs, chosen=None, pages_per_request=4096, ws=4100, ws_bytes=2 ** 40)
    assert L.frog_attend_paged(C.byref(a), None) == -1


@pytest.mark.parametrize("heads", [2, 8, 34, 66, 512])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_workspaces_of_every_cut(heads, kind):
    # no rows at all, one row, many: parts times (output, maximum and sum) of every query row, or none
    for batch in (1, 300, 5000):
        for pages in (0, 1, 5, 64, 65, 1000, 2 ** 20):
            for chosen in (None, 4096):
                for num in (0, 1, 100, 2 ** 20):
                    a = args(G.PagedArgs, heads=heads, type=kind, batch=batch, pages_per_request=pages, chosen=chosen, num_chosen=num)
                    n = F.lib().frog_attend_paged_workspace(C.byref(a))
                    assert n >= 0 and n % (batch * heads * (64 + 2) * 4) == 0
                    rows = (num if chosen else pages) * 16
                    assert n == 0 if rows <= 128 else n <= batch * heads * 66 * 4 * max(1, rows // 128 + 1)


def test_sizes_above_a_launch_are_refused():
    # before anything is enqueued, by the workspace query too where there is one
    L = F.lib()
    assert L.frog_cache_read(C.byref(args(G.ReadArgs, batch=2 ** 20, slots=2 ** 17)), None) == -7 and b"workgroups" in L.frog_last_error()
    assert L.frog_cache_write(C.byref(args(G.WriteArgs, **{"cache.kv_heads": 65535, "batch": 2 ** 16, "tokens": 2 ** 16, "cache.num_pages": 1})), None) == -7
    big = args(G.PagedArgs, batch=2 ** 20, pages_per_request=2 ** 22, chosen=None)
    assert L.frog_attend_paged_workspace(C.byref(big)) == -7 and L.frog_attend_paged(C.byref(big), None) == -7
    big = args(G.SelectArgs, batch=2 ** 22, pages_per_request=2 ** 24)
    assert L.frog_select_pages_workspace(C.byref(big)) == -7 and L.frog_select_pages(C.byref(big), None) == -7


def test_a_cache_keeps_its_tensors():
    # (their sizes are what the kernels go by)
    for name in ("k", "v", "k_exp", "v_exp", "bounds", "shape", "device"):
        assert isinstance(getattr(F.PagedCache, name), property) and getattr(F.PagedCache, name).fset is None
    with pytest.raises(AttributeError):
        F.no_such_name


def test_the_binding_refuses_what_is_on_no_gpu():
    k = torch.zeros(2, 1, 16, 32, dtype=torch.int8)
    e = torch.zeros(2, 1, 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        F.PagedCache(k, k, e, e)
    with pytest.raises(ValueError, match="storage"):
        F.PagedCache.empty(2, 1, 32, storage="int4", device="cpu")


def test_the_definition():
    # e4m3 codes as torch's own conversion rounds them; magnitudes, powers
    x = torch.randn(64, 32, generator=torch.Generator().manual_seed(0)).double() * 3
    codes, byte = quantise(x, "e4m3")
    y = x * torch.exp2(127.0 - byte.double()).unsqueeze(-1)
    assert torch.equal(codes, y.float().to(torch.float8_e4m3fn).double())
    assert (codes.abs().amax(-1) <= 448).all() and (codes.abs().amax(-1) >= 224).all()
    codes, byte = quantise(x, "int8")
    assert (codes.abs().amax(-1) <= 127).all() and (codes.abs().amax(-1) >= 63).all()
    assert ((codes * torch.exp2(byte.double() - 127).unsqueeze(-1) - x).abs() <= 0.5 * torch.exp2(byte.double() - 127).unsqueeze(-1)).all()
    codes, byte = quantise(torch.tensor([[448.0, 1.0], [448.5, 1.0], [0.0, 0.0], [float("inf"), 1.0]]).double(), "e4m3")
    assert byte.tolist() == [127, 128, 27, 255] and codes[0].tolist() == [448.0, 1.0] and codes[3].tolist() == [0.0, 0.0]

"""The attention section of the C ABI on the host: struct layouts of the
binding against include/frog.h, and refusals before any GPU is touched."""
import ctypes as C
import os
import subprocess

import pytest

pytest.importorskip("torch")

import paper_2608_16491_amd as F  # noqa: E402
from paper_2608_16491_amd import attention as A  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = (("frog_attend_t", A.AttendArgs), ("frog_attend_shared_t", A.SharedArgs), ("frog_evict_t", A.EvictArgs))


def test_struct_layouts_match_the_header(tmp_path):
    lines = []
    for name, cls in PAIRS:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include "frog.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", f"-I{ROOT}/include", str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, cls in PAIRS:
        want.append(C.sizeof(cls))
        want += [getattr(cls, f[0]).offset for f in cls._fields_]
    assert got == want


def rows(a, names, strides):
    for n in names:
        setattr(a, n, 4096)
        setattr(a, n + "_stride", strides)


def attend_args(**kw):
    a = A.AttendArgs()
    rows(a, ("q", "k", "v", "out", "dout", "dq", "dk", "dv"), (4096, 256, 64))
    a.batch, a.queries, a.keys, a.heads, a.kv_heads, a.d, a.type, a.scale = 2, 3, 5, 4, 2, 64, 2, 0.125
    a.lse = 4096
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD = [(dict(q=None), -1), (dict(q=4100), -1), (dict(k_stride=(4096, 100, 64)), -1), (dict(v_stride=(-4096, 256, 64)), -1),
       (dict(type=7), -1), (dict(heads=3), -1), (dict(kv_heads=0), -1), (dict(d=40), -7), (dict(d=256), -7), (dict(batch=-1), -1),
       (dict(scale=float("inf")), -1), (dict(cap=-1.0), -1), (dict(cap=float("nan")), -1), (dict(slopes=4096), -1),
       (dict(at_k=4096), -1), (dict(w_in=4096), -1), (dict(lr=4100), -1), (dict(keys=2 ** 31), -7), (dict(queries=2 ** 30), -7),
       (dict(batch=2 ** 30), -7), (dict(out=None), -1)]


@pytest.mark.parametrize("kw,code", BAD, ids=lambda x: str(x))
def test_attend_refuses(kw, code):
    L = F.lib()
    a = attend_args(**kw)
    assert L.frog_attend(C.byref(a), None) == code and L.frog_last_error()
    assert L.frog_attend_workspace(C.byref(a), 0) == code
    assert L.frog_attend_backward(C.byref(a), None) == code


def test_backward_refuses():
    L = F.lib()
    for kw in (dict(lse=None), dict(dq=None), dict(dk=4104), dict(dout=None), dict(w_out=4096)):
        assert L.frog_attend_backward(C.byref(attend_args(**kw)), None) == -1
    assert L.frog_attend(None, None) == -1 and L.frog_attend_backward(None, None) == -1
    # a workspace that is too small, or starts between its boundaries
    assert L.frog_attend_backward(C.byref(attend_args(ws=4096, ws_bytes=4)), None) == -1
    assert L.frog_attend_backward(C.byref(attend_args(ws=4097, ws_bytes=2 ** 30)), None) == -1


def test_the_stride_of_one_row_is_not_looked_at():
    a = attend_args(batch=1, q_stride=(3, 256, 64))
    assert F.lib().frog_attend_workspace(C.byref(a), 0) >= 0


def test_nothing_to_do_is_no_error():
    L = F.lib()
    a = attend_args(batch=0, q=None, k=None, v=None, out=None, dq=None, dk=None, dv=None, dout=None, lse=None)
    assert L.frog_attend_workspace(C.byref(a), 0) >= 0 and L.frog_attend_workspace(C.byref(a), 1) >= 0


def shared_args(**kw):
    a = A.SharedArgs()
    rows(a, ("q", "k", "v", "out"), (256, 64))
    rows(a, ("k_pages", "v_pages"), (4096, 128, 64))
    a.pages = a.lengths = 4096
    a.batch, a.prefix, a.num_pages, a.pages_per_request, a.page = 2, 10, 4, 2, 16
    a.heads, a.kv_heads, a.d, a.type, a.scale = 4, 2, 64, 1, 0.125
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(q=None), -1), (dict(k=8), -1), (dict(page=0), -1), (dict(pages=None), -1), (dict(lengths=None), -1),
                                     (dict(k_pages=None), -1), (dict(d=16), -7), (dict(prefix=-1), -1), (dict(lr=4100), -1),
                                     (dict(prefix=2 ** 31), -7), (dict(pages_per_request=2 ** 28), -7), (dict(heads=5), -1)],
                         ids=lambda x: str(x))
def test_shared_refuses(kw, code):
    a = shared_args(**kw)
    assert F.lib().frog_attend_shared(C.byref(a), None) == code and F.lib().frog_last_error()
    assert F.lib().frog_attend_shared_workspace(C.byref(a)) == code


def evict_args(**kw):
    a = A.EvictArgs()
    rows(a, ("k", "v"), (4096, 128, 64))
    for n in ("weights", "positions", "lengths", "k_out", "v_out", "weights_out", "positions_out", "lengths_out"):
        setattr(a, n, 4096)
    a.batch, a.slots, a.keep, a.recent, a.heads, a.d, a.type = 2, 32, 16, 4, 2, 64, 1
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(k=None), -1), (dict(keep=33), -1), (dict(recent=17), -1), (dict(recent=-1), -1), (dict(d=12), -7),
                                     (dict(weights=None), -1), (dict(lengths=None), -1), (dict(v_out=8), -1), (dict(heads=0), -1),
                                     (dict(slots=2 ** 31), -7), (dict(type=3), -1), (dict(lengths_out=None), -1)], ids=lambda x: str(x))
def test_evict_refuses(kw, code):
    a = evict_args(**kw)
    assert F.lib().frog_evict(C.byref(a), None) == code and F.lib().frog_last_error()
    assert F.lib().frog_evict_workspace(C.byref(a)) == code


def test_names_are_reached_from_the_package():
    assert all(callable(getattr(F, n)) for n in ("attend", "attend_shared", "evict"))
    with pytest.raises(AttributeError):
        F.no_such_name


@pytest.mark.parametrize("cap", [1e-39, 3e38])
def test_caps_whose_quotient_or_multiple_overflows_are_refused(cap):
    assert F.lib().frog_attend(C.byref(attend_args(cap=cap)), None) == -1
    assert F.lib().frog_attend_shared(C.byref(shared_args(cap=cap)), None) == -1

"""Parts of the attention kernels that also run on the host, under the address
sanitizer there."""
import os
import subprocess

import pytest

from paper_2608_16491_amd import _build

PIECES = """
#include <cstdio>
#include <cstdlib>
#include "attend_tile.h"
using namespace frog;
template <typename T, int C>
int check() {
    T* p = (T*)aligned_alloc(32, 32);
    for (int i = 0; i < C; ++i) p[i] = (T)(float)(i + 1);
    const vec<T, C> x = load_piece<T, C>(p);
    int bad = 0;
    for (int i = 0; i < C; ++i) bad += (float)x[i] != (float)(i + 1);
    free(p);
    return bad;
}
template <typename T>
int checks() { return check<T, 2>() + check<T, 4>() + check<T, 6>() + check<T, 8>(); }
int main() { return checks<float>() + checks<f16_t>() + checks<bf16_t>(); }
"""


@pytest.fixture()
def run(tmp_path):
    def f(text):
        src, exe = tmp_path / "host.hip", str(tmp_path / "host")
        src.write_text(text)
        # (nothing optimised away, the checks on the host's side of the code alone)
        subprocess.run([_build.HIPCC, "-O0", "-g", "-std=c++17", "--offload-host-only", "-Wno-psabi", f"-I{_build.INCLUDE}", f"-I{_build.CSRC}",
                        "-Xarch_host", "-fsanitize=address", str(src), "-o", exe], check=True)
        done = subprocess.run([exe], capture_output=True, text=True, env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
        assert done.returncode == 0, done.stderr[:2000]
    return f


def test_pieces_of_value_rows_stay_within_what_was_read(run):
    run(PIECES)

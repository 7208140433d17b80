"""Whether what a call writes lies in what it reads (lpp_overlap.h), tried on the host against every byte (no GPU)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06352_amd", "csrc")
SOURCE = """
#include "lpp_overlap.h"
extern "C" int32_t ranges(uint64_t a, uint64_t na, uint64_t b, uint64_t nb) { return ranges_meet((void*)a, na, (void*)b, nb); }
extern "C" int32_t rows(uint64_t data, int64_t item, int64_t row, int64_t head, int64_t B, int64_t M, int64_t heads, int64_t width, uint64_t out,
                        int64_t n) {
  return rows_meet((void*)data, item, row, head, B, M, heads, width, (void*)out, n);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "t.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "t.cpp"), "-o", str(d / "t.so")], check=True)
    L = C.CDLL(str(d / "t.so"))
    L.ranges.argtypes, L.rows.argtypes = [C.c_uint64] * 4, [C.c_uint64] + [C.c_int64] * 7 + [C.c_uint64, C.c_int64]
    return L


def test_ranges(lib):
    for a, na, b, nb, meet in ((100, 10, 110, 5, 0), (100, 10, 109, 5, 1), (110, 5, 100, 10, 0), (105, 1, 100, 10, 1), (100, 10, 100, 10, 1),
                               (100, 0, 95, 10, 0), (0, 1000, 100, 10, 0), (100, 10, 0, 1000, 0)):
        assert lib.ranges(a, na, b, nb) == meet


def test_rows_against_every_byte(lib):
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(20000):
        B, M, heads, width = (int(x) for x in rng.integers(1, 5, 4))
        item, row, head = (int(x) for x in rng.integers(0, [60, 25, 12]))
        data = 1000
        out, n = int(rng.integers(900, 1300)), int(rng.integers(1, 40))
        starts = data + (np.arange(B)[:, None, None] * item + np.arange(M)[:, None] * row + np.arange(heads) * head).ravel()
        want = bool(np.any((starts < out + n) & (starts + width > out)))
        assert lib.rows(data, item, row, head, B, M, heads, width, out, n) == want, (data, item, row, head, B, M, heads, width, out, n)
        seen[want] += 1
    assert min(seen) > 2000

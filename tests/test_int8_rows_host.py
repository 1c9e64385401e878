"""Rows to 8 bits and back at the top of their range: the walk of a launch with fewer workgroups than rows (csrc/moe_rows.h),
replayed on the host, and what is refused beyond."""
import ctypes as C
import os
import subprocess

import pytest

from test_abi_host import L  # noqa: F401
from test_int8_host import BF16, F32, INVALID, at  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2402_07033_amd", "csrc")
WALK = r"""
#include "moe_rows.h"
extern "C" int walk(int first, int step, int T, long long* taken, int* last) {
    long long n = 0;
    bool inside = true;
    struct Left {};
    try {
        each_row(first, step, T, [&](int t) {
            if (t < 0 || t >= T) inside = false;
            if (!inside || n > 1 << 17) throw Left{};
            n++;
            *last = t;
        });
    } catch (Left) {}
    *taken = n;
    return inside;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "w.cpp").write_text(WALK)
    # (-fwrapv: a counter that wraps shows as one, whatever the compiler makes of it)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "w.so"), str(d / "w.cpp")],
                   check=True)
    return C.CDLL(str(d / "w.so")).walk


# the grids of rows to codes and of codes to rows
@pytest.mark.parametrize("step", [1 << 20, 65535])
@pytest.mark.parametrize("T", [1, 65535, 65536, (1 << 20) + 37, 2047 << 20, (2047 << 20) + 1, (1 << 31) - 65535, (1 << 31) - 1])
def test_every_row_is_taken_once(walk, step, T):
    rows = 0
    for first in sorted({0, 1, 36, 37, step // 2, step - 2, step - 1}):
        if first >= min(T, step):
            continue  # no such workgroup
        n, last = C.c_longlong(), C.c_int(-1)
        assert walk(first, step, T, C.byref(n), C.byref(last)) == 1
        assert n.value == (T - first + step - 1) // step and last.value == first + (n.value - 1) * step
        rows += n.value
    assert rows > 0


def test_too_many_values_are_refused(L, at):  # noqa: F811
    w, q, s = (C.c_void_p(p) for p in (1 << 40, 1 << 44, 1 << 45))   # far enough apart for any size
    for T, K in ((1 << 23, 1 << 17), ((1 << 31) - 1, 528), ((1 << 31) - 1, 1 << 17)):
        for t in (F32, BF16):
            assert L.moe_int8_quantize_rows(w, t, T, K, q, s, None) == INVALID
            assert L.moe_int8_dequantize_rows(q, s, T, K, w, t, None) == INVALID

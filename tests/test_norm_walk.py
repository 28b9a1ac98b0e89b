"""The norms' walk over rows, compiled for the host from the header that the kernels use."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# A kernel's loop: rows are asked for `ahead` steps ahead of the one that is worked on.  Rows worked on; -1: a row that does not exist is asked for or worked on, -2: no end.
LOOP = r"""
#include "norm_walk.h"
using namespace vardrop;
extern "C" long long rows(long long first, long long n, long long step, int behind, int ahead) {
    const RowSteps walk{static_cast<RowIndex>(n), static_cast<RowIndex>(step)};
    RowIndex i = static_cast<RowIndex>(first), next = i;
    const long long most = n / step + behind + 2;
    auto ask = [&] {
        const bool bad = walk.there(next) && !(static_cast<long long>(next) >= 0 && static_cast<long long>(next) < n);
        next += walk.step;
        return bad;
    };
    for (int s = 0; s < ahead; ++s) if (ask()) return -1;
    long long done = 0;
    for (long long turns = 0; walk.goes_on(i, static_cast<RowIndex>(behind)); i += walk.step) {
        if (ask()) return -1;
        if (walk.there(i)) {
            if (static_cast<long long>(i) < 0 || static_cast<long long>(i) >= n) return -1;
            ++done;
        }
        if (++turns > most) return -2;
    }
    return done;
}
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("walk")
    (d / "walk.cpp").write_text(LOOP)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", f"-I{ROOT}/paper_2501_14183_b200/csrc", "-o", str(d / "walk.so"), str(d / "walk.cpp")])
    f = C.CDLL(str(d / "walk.so")).rows
    f.restype, f.argtypes = C.c_longlong, [C.c_longlong] * 3 + [C.c_int] * 2
    return f


@pytest.mark.parametrize("n", [1, 2, 31, 32, 9471, 9472, 9473, 100000, 2 ** 31 - 28417, 2 ** 31 - 28400, 2 ** 31 - 9473, 2 ** 31 - 9472, 2 ** 31 - 2, 2 ** 31 - 1])
def test_every_row_once_and_none_behind_the_last(rows, n):
    """Up to the 2^31 - 1 rows that a call may have; 9472 groups go side by side where rows are narrow, 32 in the run of a CTA."""
    for step in (1, 32, 9472):
        if n / step > 1e7:
            continue
        for first in {0, 1, 3, min(step, n) // 2, min(step, n) - 1, step - 1}:
            for behind in (0, 1, 3):
                got = rows(first, n, step, behind, 2)
                assert got == max(0, -(-(n - first) // step)), (n, step, first, behind)

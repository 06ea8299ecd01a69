"""The rows that the attention operators take from two ends in an array on the device, whatever those hold: the function that the
kernels call, compiled for the CPU."""
from __future__ import annotations

import itertools
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LEAST, MOST = -2 ** 31, 2 ** 31 - 1

PROGRAM = """
#include <cstdio>
#include "gqsa_attention.hpp"
static_assert(gqsa::rows_between(5, -2147483647 - 1, 100).count == 0);        // (a constant expression with an overflow does not compile)
static_assert(gqsa::rows_between(2147483647, -2147483647 - 1, 1 << 25).count == 0);
int main()
{
    int first, end;
    long long n;
    while (std::scanf("%d %d %lld", &first, &end, &n) == 3) {
        const gqsa::Rows r = gqsa::rows_between(first, end, n);
        std::printf("%d %d\\n", r.start, r.count);
    }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++ here")
def test_rows_between_any_two_ends(tmp_path):
    (tmp_path / "rows.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2412_17560_amd", "csrc"),
                    "-o", str(tmp_path / "rows"), str(tmp_path / "rows.cpp")], check=True)
    numbers = [LEAST, LEAST + 1, LEAST + 5, -(2 ** 30), -100, -1, 0, 1, 5, 99, 100, 101, 2 ** 25 - 1, 2 ** 25, 2 ** 30, MOST - 1, MOST]
    cases = list(itertools.product(numbers, numbers, [0, 1, 100, 2 ** 25]))
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    out = subprocess.run([str(tmp_path / "rows")], input=text, check=True, capture_output=True, text=True).stdout.split("\n")
    for (first, end, n), line in zip(cases, out, strict=False):
        start, count = map(int, line.split())
        wanted = set(range(max(first, 0), min(end, n))) if n <= 100 else None
        assert 0 <= start <= n and 0 <= count <= n - start, (first, end, n)
        if wanted is not None:
            assert set(range(start, start + count)) == wanted, (first, end, n)
        else:
            assert count == max(min(end, n) - max(first, 0), 0) and (count == 0 or start == max(first, 0)), (first, end, n)

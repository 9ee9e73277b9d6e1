"""Quotients that the kernels of branch_attention form without a division (csrc/kd_branch.h), run on the host."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_15364_amd", "csrc")

PROGRAM = r"""
#include "kd_branch.h"
#include <cstdio>
int main()
{
    long bad = 0;
    auto check = [&](long n, const kd::Divisor &by, long d) {
        if (n >= 0 && n <= 0x7fffffffL && by.divide((int)n) != (int)(n / d) && bad++ < 5) printf("%ld / %ld: %d\n", n, d, by.divide((int)n));
    };
    auto all = [&](long d) {
        kd::Divisor by;
        by.set((unsigned)d);
        for (long n = 0; n < 2000; ++n) check(n, by, d);
        for (long q = 1; q * d <= 0x80000000L; q += 1 + q / 9)
            for (long e = -2; e <= 2; ++e) check(q * d + e, by, d);
        for (long n = 0x40000000L; n <= 0x7fffffffL; n += 0x100001L) check(n, by, d);
        for (long n = 0x7fffffffL - 100; n <= 0x7fffffffL; ++n) check(n, by, d);
    };
    for (long d = 1; d < 3000; ++d) all(d);
    for (int s = 10; s < 31; ++s)
        for (long e = -3; e <= 3; ++e) all((1L << s) + e);
    for (long d = 1001; d < 0x7fffffffL; d += d / 5) all(d);
    printf("%ld\n", bad);
    return bad != 0;
}
"""


def test_division_by_numbers_the_host_knows(tmp_path):
    if not shutil.which("hipcc"):
        pytest.skip("needs hipcc")
    src, exe = tmp_path / "counts.hip", tmp_path / "counts"
    src.write_text(PROGRAM)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-ffp-contract=off", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", f"-I{CSRC}", str(src), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout

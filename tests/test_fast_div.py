"""The division by a product that the rotary and cache kernels find rows and pages with: its quotients on the host, over the divisors in use and the ends of its
range, and that a structure which holds one is built from an empty list without a warning (the kernels' arguments are)."""
import os
import subprocess

import pytest

from paper_2609_33916_b200 import build as mbuild

SOURCE = r"""
#include "rotate.cuh"
#include <cstdio>
struct Args { int a; moa::FastDiv by; };
static unsigned long long state = 88172645463325252ull;
static unsigned next() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (unsigned)(state >> 33); }
static int check(unsigned d)
{
    const moa::FastDiv by(d);
    const unsigned most = 0x7fffffffu, last = most / d * d;
    const unsigned ends[] = {0u, 1u, d - 1u, d, d + 1u, 2u * d - 1u, last, last - 1u, last + 1u, most, most - 1u};
    for (unsigned x : ends)
        if (x <= most && by.div(x) != x / d) return 1;
    for (int i = 0; i < 200; ++i) {
        const unsigned x = next(), up = x / d * d;
        if (by.div(x) != x / d || by.div(up) != up / d || (up && by.div(up - 1u) != (up - 1u) / d)) return 1;
    }
    return 0;
}
int main()
{
    Args a{};
    if (a.by.div(12345u) != 12345u) return 2;
    for (unsigned d = 1; d <= 70000; ++d)
        if (check(d)) { std::printf("%u\n", d); return 1; }
    for (int i = 0; i < 20000; ++i) {
        const unsigned d = next();
        if (d && check(d)) { std::printf("%u\n", d); return 1; }
    }
    return check(0x7fffffffu) || check(0x40000000u) || check(0x40000001u);
}
"""


def test_quotients_and_empty_lists(tmp_path):
    nvcc = mbuild._nvcc()
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    src, exe = tmp_path / "div.cu", tmp_path / "div"
    src.write_text(SOURCE)
    flags = [f for f in mbuild.NVCC_FLAGS if f != "-lineinfo"]
    r = subprocess.run([nvcc, *flags, "-Werror", "all-warnings", "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)

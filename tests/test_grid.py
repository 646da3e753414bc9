"""How workgroups are laid into a launch, compiled by the host compiler from the header that the library uses."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_01381_amd", "csrc")


def test_every_launch_has_fewer_threads_than_32_bits_count(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text("""
#include <stdio.h>
#include <initializer_list>
#include "grid.hpp"
using namespace adaqp;
#define CHECK(x) do { if (!(x)) { printf("%lld workgroups of %d, line %d: %s\\n", (long long)n, threads, __LINE__, #x); return 1; } } while (0)
int main() {
    for (int threads : {64, 256, 512, 1024})
        for (int bit = 0; bit <= 31; ++bit)
            for (int64_t off = -9; off <= 9; ++off) {
                const int64_t n = ((int64_t)1 << bit) + off;
                if (n < 1 || n > kMostWorkgroups) continue;
                const GridSize g = grid_size(n, threads);
                CHECK(g.x >= 1 && g.y >= 1 && g.y <= 65535);
                CHECK((int64_t)g.x * threads < ((int64_t)1 << 32));
                CHECK((int64_t)g.x * g.y >= n && (int64_t)g.x * (g.y - 1) < n);
                CHECK((int64_t)g.x * g.y < ((int64_t)1 << 32));
                CHECK(g.y == 1 ? g.x == n : g.x % 8 == 0);
            }
    return 0;
}
""")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout

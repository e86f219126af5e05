"""The bisection that picks alternatives' segments, compiled for the host from the kernel's own header: it ends, and
finds the k-th largest key, for ranges up to all unsigned numbers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <vector>
#include "tok_select.h"

static uint64_t state = 1;
static unsigned next() {                             // any generator will do
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return (unsigned)(state >> 32);
}

int main() {
    const int sizes[] = {1, 2, 33, 513, 600, 1023};
    int cases = 0;
    for (int n : sizes)
        for (int kind = 0; kind < 5; ++kind) {
            std::vector<unsigned> key(n);
            for (unsigned& x : key)
                x = kind == 0 ? next() : kind == 1 ? 0x80000000u + next() % 7 : kind == 2 ? 0xffffffffu - next() % 3 : kind == 3 ? next() % 4 : 0x007fffffu;
            std::vector<unsigned> sorted = key;
            std::sort(sorted.rbegin(), sorted.rend());
            for (int k : {1, 2, 20, 32})
                for (unsigned top : {0xffffffffu, sorted[0]}) {
                    if (k > n) continue;
                    const unsigned bounds[] = {0u, sorted[n - 1], sorted[k - 1]};
                    for (unsigned lo : bounds) {
                        int steps = 0;
                        const unsigned t = pb::highest_reached(lo, top, k, [&](unsigned at) {
                            if (++steps > 32) {
                                printf("no end: n=%d k=%d lo=%u hi=%u\n", n, k, lo, top);
                                exit(1);
                            }
                            int c = 0;
                            for (unsigned x : key) c += x >= at;
                            return c;
                        });
                        const int reached = (int)std::count_if(key.begin(), key.end(), [&](unsigned x) { return x >= t; });
                        if (t != sorted[k - 1] && reached != k) {
                            printf("wrong: n=%d k=%d lo=%u hi=%u t=%u\n", n, k, lo, top, t);
                            return 1;
                        }
                        ++cases;
                    }
                }
        }
    printf("%d\n", cases);
    return cases > 500 ? 0 : 1;
}
"""


def test_bisection_ends_and_finds_the_kth_largest(tmp_path):
    compiler = shutil.which("g++") or shutil.which("c++")
    if compiler is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "select.cpp", tmp_path / "select"
    src.write_text("#include <cstdlib>\n" + PROGRAM)
    subprocess.run([compiler, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2003_11666_b200", "csrc"), str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout

"""What the launches remember of the GPU's answers is told apart by kernel, device, threads and shared memory (host code alone)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1905_05686_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "occupancy_cache.cuh"
static void one(int) {}
static void two(int) {}                    // the same type
int main()
{
    lrbi::OccupancyCache cache;
    int asked = 0;
    auto get = [&](void (*f)(int), int device, int threads, size_t smem, int answer) {
        return cache.get(reinterpret_cast<const void *>(f), device, threads, smem, [&] { ++asked; return answer; });
    };
    for (int i = 0; i < 3; ++i) {          // alternating: each is asked for once
        if (get(one, 0, 512, 4096, 2) != 2 || get(two, 0, 512, 4096, 3) != 3 || get(one, 1, 512, 4096, 4) != 4) return 1;
        if (get(one, 0, 256, 4096, 5) != 5 || get(one, 0, 512, 8192, 6) != 6 || get(one, 0, 512, (size_t)1 << 32, 7) != 7) return 2;
    }
    if (asked != 6) return 3;
    if (get(two, 1, 512, 1, 0) != 1 || get(two, 1, 512, 1, 2) != 2) return 4;      // a failure is not kept
    return 0;
}
"""


def test_answers_are_told_apart(tmp_path):
    source, program = tmp_path / "t.cpp", tmp_path / "t"
    source.write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-pthread", "-I", CSRC, str(source), "-o", str(program)], check=True)
    assert subprocess.run([str(program)]).returncode == 0

"""Whether strided arrays share memory (csrc/overlap.h, compiled for the host), against sets of their bytes."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2510_15312_b200", "csrc")

PROGRAM = r"""
#include "overlap.h"
#include <cstdio>
#include <random>
#include <set>
using namespace sdv;
static std::mt19937 rng(3);
static int pick(int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); }
static std::set<long long> bytes(const Area& a) {
    std::set<long long> s;
    for (long long i = 0; i < a.dim[0].n; ++i)
        for (long long j = 0; j < a.dim[1].n; ++j)
            for (long long k = 0; k < a.dim[2].n; ++k)
                for (long long x = 0; x < a.run; ++x) s.insert((long long)(intptr_t)a.p + i * a.dim[0].step + j * a.dim[1].step + k * a.dim[2].step + x);
    return s;
}
static Area some(int style) {
    Area a = area((const void*)(intptr_t)(100000 + pick(0, 400)), pick(1, 9));
    long long step = a.run + pick(0, 3) * (style & 1);
    for (int d = 2; d >= 0; --d) {
        a.dim[d].n = pick(1, 4);
        a.dim[d].step = style < 2 ? step : style == 2 ? pick(-40, 40) : 24 >> d;   // nested, anything, the same ones in both
        step = step * a.dim[d].n + pick(0, 5) * (style & 1);
    }
    return a;
}
int main() {
    Overlap meet;
    int yes = 0, no = 0;
    for (int t = 0; t < 16000; ++t) {
        const Area a = some(t % 4), b = some(t / 4 % 4);
        bool want = false;
        const std::set<long long> sa = bytes(a);
        for (long long x : bytes(b)) want |= sa.count(x) > 0;
        if (meet(a, b) != want || meet(b, a) != want) return std::printf("%d: %d\n", t, (int)want), 1;
        (want ? yes : no)++;
    }
    if (yes < 2000 || no < 2000) return 2;
    // q, k and v side by side, heads outside and rows outside; a row further on
    const void* p = (const void*)(intptr_t)0x7f0000000000ll;
    const auto at = [&](long long off) { return (const void*)((const char*)p + off); };
    const Area q = area(p, 256, 9000, 8192, 24, 256), k = area(at(24 * 256), 256, 9000, 8192, 8, 256), later = area(at(8192), 256, 9000, 8192, 24, 256);
    if (meet(q, k) || !meet(q, later) || !meet(q, q)) return 3;
    const Area h0 = area(p, 128, 1000000, 256, 8, 256000000), h1 = area(at(128), 128, 1000000, 256, 8, 256000000);   // two tensors interleaved by element runs
    if (meet(h0, h1) || !meet(h0, area(at(127), 128, 1000000, 256, 8, 256000000))) return 4;
    if (meet(area(nullptr, 4), q) || meet(area(p, 0), q) || meet(area(p, 4, 0, 8), q)) return 5;
    // at the ends of the address space and of the counts
    if (!meet(area((const void*)~0ull, 1), area((const void*)~0ull, 1)) || meet(area((const void*)~0ull, 1), area(p, 8, 3, 8))) return 6;
    if (!meet(area(p, 8, 4, 1ll << 62), area(p, 8)) || meet(area(p, 8, 4, 1ll << 62), area(at(8), 8))) return 8;
    if (!meet(area(p, 4, 0x7fffffff, 1ll << 16, 0x7fffffff, 4), area(at((0x7ffffffell << 16) + 4), 4))) return 7;
    return 0;
}
"""


def test_overlap_of_strided_arrays(tmp_path):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], timeout=300, capture_output=True, text=True)
    assert out.returncode == 0, (out.returncode, out.stdout + out.stderr[-2000:])

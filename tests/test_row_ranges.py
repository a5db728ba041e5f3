"""Which row ranges can share memory (csrc/row_ranges.h), compiled as plain C++ and held against the bytes themselves: never "no" where a byte is
shared, and exact where both tensors have one stride or a single row."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "row_ranges.h"
#include <stdio.h>
#include <set>
using namespace dirotq;

int main() {
    const long long base = 1 << 20;
    long said_yes = 0, said_no = 0;
    for (int rows_a = 1; rows_a <= 4; rows_a += rows_a)
        for (int rows_b = 1; rows_b <= 3; ++rows_b)
            for (int wa = 1; wa <= 6; wa += 2)
                for (int sa = wa; sa <= wa + 7; ++sa) {
                    std::set<long long> bytes;
                    for (int r = 0; r < rows_a; ++r)
                        for (int i = 0; i < wa; ++i) bytes.insert(base + r * sa + i);
                    for (int wb = 1; wb <= 7; wb += 3)
                        for (int sb = wb; sb <= 13; ++sb)
                            for (long long b0 = base - 45; b0 <= base + 45; ++b0) {
                                bool shared = false;
                                for (int r = 0; r < rows_b && !shared; ++r)
                                    for (int i = 0; i < wb && !shared; ++i) shared = bytes.count(b0 + r * sb + i) != 0;
                                const bool said = rows_overlap(reinterpret_cast<const void*>(base), rows_a, wa, sa, reinterpret_cast<const void*>(b0), rows_b, wb, sb);
                                (said ? said_yes : said_no)++;
                                if (shared && !said) { printf("missed: %d x %d / %d, %d x %d / %d at %lld\n", rows_a, wa, sa, rows_b, wb, sb, b0 - base); return 1; }
                                if (said && !shared && rows_a == 1 && rows_b == 1) { printf("single rows: %d, %d at %lld\n", wa, wb, b0 - base); return 1; }
                            }
                }
    // rows of one wide tensor: columns apart are apart, columns that touch are not
    auto at = [](long long v) { return reinterpret_cast<const void*>(base + v); };
    if (rows_overlap(at(0), 8, 64, 256, at(64), 8, 128, 256) || rows_overlap(at(128), 8, 64, 256, at(0), 8, 128, 256)) { printf("columns apart\n"); return 1; }
    if (!rows_overlap(at(0), 8, 66, 256, at(64), 8, 128, 256) || !rows_overlap(at(128), 8, 64, 256, at(0), 8, 130, 256)) { printf("columns that touch\n"); return 1; }
    // more than 32 bits apart and wide
    if (rows_overlap(at(0), 1 << 20, 1 << 12, 1ll << 14, at((1ll << 34)), 4, 64, 64)) { printf("far\n"); return 1; }
    if (!rows_overlap(at(0), 1 << 20, 1 << 12, 1ll << 14, at((1ll << 34) - (1 << 14)), 4, 64, 64)) { printf("far, touching\n"); return 1; }
    return said_yes && said_no ? 0 : 1;
}
"""


def test_against_the_bytes(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_16732_b200", "csrc"), str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr

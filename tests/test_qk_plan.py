"""What the kernels take from a description of queries and keys (csrc/qk_plan.h), compiled as plain C++: where nothing is rotated no pointer of the
rotation's reaches a kernel, whatever the description still holds from another call."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "qk_plan.h"
#include <initializer_list>
#include <stdio.h>
#include <string.h>
using namespace dirotq;

int main() {
    dirotq_qk_t qk;
    memset(&qk, 0, sizeof qk);
    const int32_t* const stale = reinterpret_cast<const int32_t*>(0x1001);  // (neither aligned nor mapped; never read here)
    for (const int32_t* p : {stale, static_cast<const int32_t*>(nullptr)}) {
        qk.positions = p;
        qk.rope = DIROTQ_ROPE_NONE;
        if (qk_positions(qk) != nullptr) { printf("positions without a rotation\n"); return 1; }
        for (int rope : {int(DIROTQ_ROPE_PAIRS), int(DIROTQ_ROPE_HALVES)}) {
            qk.rope = rope;
            if (qk_positions(qk) != p) { printf("positions of a rotation lost\n"); return 1; }
        }
    }
    return 0;
}
"""


def test_positions(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_16732_b200", "csrc"), str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


def test_every_kernel_takes_positions_from_there():
    """No launcher passes the description's pointer on by itself."""
    csrc = os.path.join(ROOT, "paper_2605_16732_b200", "csrc")
    for name in sorted(os.listdir(csrc)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(csrc, name)) as f:
                for line in f:
                    assert "p.positions = qk.positions" not in line and "qk.positions :" not in line, name

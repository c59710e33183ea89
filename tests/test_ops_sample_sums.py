"""The whole numbers that sampling adds weights up in, without a GPU: the longest row that the call takes, all of its weights
the highest."""
from __future__ import annotations

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sums_of_the_longest_row_fit(tmp_path):
    src = tmp_path / "sum.cpp"
    src.write_text("""
#include "ops_forms.h"
#include "simgpu_ops.h"
int main() {
    uint64_t sum = 0;
    for (int i = 0; i < SIM_SAMPLE_MAX_V; i++) {
        const uint64_t more = sum + (uint64_t)(1. * simops::kWeightUnit + .5);
        if (more <= sum) return 1;
        sum = more;
    }
    return (double)sum == simops::kWeightUnit * SIM_SAMPLE_MAX_V ? 0 : 2;
}
""")
    exe = str(tmp_path / "sum")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2606_10440_amd", "csrc"),
                    "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    assert subprocess.run([exe]).returncode == 0

"""The comparison of what a call reads and writes, by itself: none of its arrays goes unlooked at."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_12422_gb300", "csrc")
MAIN = """#include <cstdio>
#include <cstdint>
#include "kv_checks.h"
int main() {
    for (int n = 0; n <= 20; ++n)
        for (int over = 0; over < 2; ++over) {  // the last one over the first
            pbd::checks::Ranges mem;
            for (int i = 0; i < n; ++i)
                mem.add("x", reinterpret_cast<void *>((uintptr_t)(over && i == n - 1 ? 1 : i + 1) << 20), 4, true);
            mem.add("nothing", nullptr, 4, true);
            printf("%d", mem.clash() != nullptr);
        }
}
"""


def test_every_array_is_compared(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("nvcc unavailable")
    (tmp_path / "main.cu").write_text(MAIN)
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"),
                    str(tmp_path / "main.cu"), "-o", str(tmp_path / "main")], check=True, capture_output=True)
    got = subprocess.run([str(tmp_path / "main")], check=True, capture_output=True, text=True).stdout
    for n in range(21):
        apart, over = got[2 * n] == "1", got[2 * n + 1] == "1"
        assert apart == (n > 16) and over == (n > 1), n  # (more than there is room for is refused)

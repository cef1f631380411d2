"""After how long waits of the attention kernels on packed rows give up: beyond the longest work that one of them waits for."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_12422_gb300", "csrc")
PROMPTS = [1, 128, 512, 16384, 1 << 20, 90_000_000, (1 << 30) - 1, 1 << 30]
TREES = [(5.0, 152), (1e6, 152), (2147483646.0, 152), (2147483646.0, 1)]
MAIN = """#include <cstdio>
#include "packed_ops.h"
int main() {
    const int T[] = {%s};
    for (int t : T) printf("%%u\\n", pbd::prompt_patience(t));
    const double tree[][2] = {%s};
    for (auto &x : tree) printf("%%u\\n", pbd::tree_patience(x[0], (int)x[1]));
}
""" % (",".join(map(str, PROMPTS)), ",".join("{%.1f, %d}" % x for x in TREES))


@pytest.fixture(scope="module")
def limits(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("nvcc unavailable")
    d = tmp_path_factory.mktemp("waits")
    (d / "main.cu").write_text(MAIN)
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(d / "main.cu"), "-o",
                    str(d / "main")], check=True, capture_output=True)
    # (2^20 ns each)
    return [int(x) * 2 ** 20 * 1e-6 for x in subprocess.run([str(d / "main")], check=True, capture_output=True, text=True).stdout.split()]


def test_a_wait_outlasts_what_it_waits_for(limits):
    """An item of a prompt has a block of keys for each 128 of its tokens, and two tiles of rows a block take 1.5 us at heads of 128 (4 us are
    allowed here; the waits in question last two items at most).  A CTA's stretch of a batch of trees has its share of the list's places;
    a block copied row by row, the slowest form, takes 5 to 10 us."""
    for T, ms in zip(PROMPTS, limits):
        assert ms >= 1000 and ms > 2 * (T / 128) * 4e-3, T
    for (places, workers), ms in zip(TREES, limits[len(PROMPTS):]):
        assert ms >= 1000 and ms > places / workers * 10e-3


def test_a_usual_wait_gives_up_after_a_second(limits):
    for T, ms in zip(PROMPTS, limits):
        if T <= 1 << 20:
            assert ms <= 1300, T
    assert 1000 <= limits[len(PROMPTS)] < 1002

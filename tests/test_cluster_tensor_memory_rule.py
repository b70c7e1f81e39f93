"""CTAs of a cluster wait for one another while they hold tensor memory, of which an SM has 512 columns: whatever of them can share an SM has to
fit, or clusters of two streams could wait for each other without an end.  Shared memory sees to that (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_14090_b200", "csrc")

PROGRAM = r"""
#include "common.cuh"
#include <stdio.h>
int main() {
  const int limits[2] = {232448, 101376};
  for (int limit : limits)
    for (int cols = 32; cols <= 512; cols *= 2)
      for (int bytes = 0; bytes <= limit; bytes += 1111)
        printf("%d %d %d %zu\n", limit, cols, bytes, aiq::cluster_smem(bytes, cols, limit));
}
"""


def test_shared_memory_is_at_least_the_share_of_the_columns(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("nvcc not found")
    (tmp_path / "rule.cu").write_text(PROGRAM)
    subprocess.run([nvcc, "-std=c++17", "-I", CSRC, "-o", str(tmp_path / "rule"), str(tmp_path / "rule.cu")], check=True, capture_output=True)
    lines = subprocess.run([str(tmp_path / "rule")], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    assert len(lines) > 1000
    for limit, cols, used, asked in (map(int, line.split()) for line in lines):
        assert used <= asked <= limit
        # CTAs whose shares of the SM's shared memory add up to one at most have columns that add up to 512 at most
        assert (asked + 1024) * 512 >= cols * (limit + 1024)


def test_every_cluster_with_tensor_memory_asks_for_it():
    launches = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")) or name == "common.cuh":
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        if "tmem_alloc(" not in text or "launch_chained_cluster(" not in text:
            continue
        for m in re.finditer(r"launch_chained_cluster\(", text):
            launches += 1
            head = text[m.end():m.end() + 400]
            assert re.search(r"dim3\([\w:]+\), smem, s,", head), f"{name}: a launch whose shared memory is not `smem`"
            assert re.search(r"const size_t smem = p\.cluster > 1 \? cluster_smem\(", text[:m.start()]), f"{name}: shared memory by no rule"
    assert launches == 3

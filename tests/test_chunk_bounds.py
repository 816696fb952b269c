"""What the chunk kernels make of row boundaries and lengths that lie on the device and may say anything: compiled from the kernels'
own header and run on the host."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
NVCC = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"

SRC = r"""
#include <climits>
#include <cstdio>
#include "chunk.cuh"
int main() {
  const int edge[] = {INT_MIN, INT_MIN + 1, INT_MIN + 5, -1000, -1, 0, 1, 5, 6, 7, 20, 1000, INT_MAX - 1, INT_MAX};
  const int totals[] = {0, 1, 6, 1 << 30};
  long long bad = 0;
  for (int total : totals)
    for (int first : edge)
      for (int end : edge) {
        const int cu[2] = {first, end}, lens[1] = {first};
        const ug::ChunkBatch B = {cu, lens, nullptr, 1, total, 3, 10};
        int row0 = -1;
        const long long n = B.rows(0, row0);
        auto held = [&](long long x) { return x < 0 ? 0 : x > total ? total : x; };
        const long long want0 = held(first), want = held(end) > want0 ? held(end) - want0 : 0;
        const long long room = 3 * 64, L = first < 0 ? 0 : first > room ? room : first;
        if (row0 != want0 || n != want || B.len(0) != L) {
          ++bad;
          std::printf("rows [%d, %d) of %d: %lld from %d on\n", first, end, total, n, row0);
        }
      }
  return bad != 0;
}
"""


@pytest.mark.skipif(not Path(NVCC).exists(), reason="needs nvcc")
def test_boundaries_and_lengths_stay_inside(tmp_path):
    src = tmp_path / "bounds.cu"
    src.write_text(SRC)
    exe = tmp_path / "bounds"
    subprocess.check_call([NVCC, "-O2", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", str(ROOT / "include"),
                           "-I", str(ROOT / "paper_2509_15763_b200" / "csrc"), str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr

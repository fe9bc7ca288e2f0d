"""Block norms off the 16-byte grid copy the 16-byte blocks that a row touches.  Only rows far
enough from both ends of their array take the copies without bounds: every block of theirs
lies inside the array, whatever the width, distance, address and number of rows.  The rule,
compiled for the host from its header."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2608_07814_gb300", "csrc")
NVCC = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"

PROGRAM = r"""
#include <cstdio>
#include "lx_rows.cuh"
int main() {
  long whole = 0;
  for (uint32_t es = 2; es <= 4; es += 2)
    for (uint32_t H = 1; H <= 24; ++H)
      for (uint32_t ld = H; ld <= H + 9; ++ld)
        for (uint32_t T = 1; T <= 20; ++T)
          for (uint64_t base = 4096; base < 4096 + 16; base += es) {
            const uint32_t ldb = T > 1 ? ld * es : 0, ends = lx::rows::end_rows(ldb);
            const uint64_t last = base + (uint64_t)(T - 1) * ld * es + H * es;  // the array's end
            for (uint32_t t = 0; t < T; ++t) {
              const uint64_t row = base + (uint64_t)t * ldb, first = row & ~15ull, end = (row + H * es + 15) & ~15ull;
              if (!(t >= ends && t + ends < T)) continue;
              ++whole;
              if (first < base || end > last) {
                printf("es %u H %u ld %u T %u base %d row %u: %d before, %d behind\n", es, H, ld, T,
                       (int)(base - 4096), t, (int)(base - first), (int)(end - last));
                return 1;
              }
            }
          }
  printf("%ld\n", whole);
  return 0;
}
"""


@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
def test_whole_blocks_lie_inside_the_array(tmp_path):
    src, exe = tmp_path / "reads.cu", tmp_path / "reads"
    src.write_text(PROGRAM)
    subprocess.run([NVCC, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "--expt-relaxed-constexpr",
                    "-I", CSRC, "-o", str(exe), str(src)], check=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout
    assert int(p.stdout) > 100000


def test_the_copies_take_that_rule():
    """Not the first and the last row alone, as rows narrower than 14 bytes would need more."""
    src = open(os.path.join(CSRC, "lx_resnorm.cu")).read()
    assert "t >= A.ends && t + A.ends < (unsigned)A.T" in src
    assert "std::max(A.ends, end_rows(A.ldb[k]))" in src

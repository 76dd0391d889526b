"""Where the product of eight-bit rows in tiles of 256 reads its scales in the LDS: the kernel's own places (csrc/mx8_rules.h),
compiled for the CPU and walked over every stage."""
import subprocess

from linear_paths import CSRC

# mx8_gemm_tile256's walk over its stages: what of the scales in the LDS each lane group reads, for rows of up to 200 blocks
PLACES = r"""
#include <cstdio>
#include "mx8_rules.h"
using namespace afno;
int main() {
  long long reads = 0;
  for (int blocks = 1; blocks <= 200; ++blocks) {
    const int S = blocks / 4, left = blocks % 4;
    for (int stage = 0; stage < S + (left > 0); ++stage) {
      const int there = stage < S ? 4 : left, first = stage & ~3, buffer = 16 * kScaleRows256 * (first >> 2 & 1);
      const int from = first ? next_scales256(first - 4, blocks) : 0;
      if (from < 0 || (blocks >= 16 && from + 16 > blocks)) printf("%d blocks, stage %d: loads from block %d\n", blocks, stage, from);
      for (int gq = 0; gq < 4; ++gq, ++reads) {
        // within the 16 bytes of a row: of the last row no byte behind the array, and the row's own block where there is one
        const int at = scales_at256(first, stage & 3, blocks) + gq - scale_back256(gq, there) - buffer;
        if (at < 0 || at >= 16 || (gq < there && from + at != 4 * stage + gq))
          printf("%d blocks, stage %d, lane group %d: byte %d of a row's 16\n", blocks, stage, gq, at);
      }
    }
  }
  printf("%lld reads\n", reads);
}
"""


def test_scales_are_read_where_they_are(tmp_path):
    (tmp_path / "places.cpp").write_text(PLACES)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I" + CSRC, str(tmp_path / "places.cpp"), "-o", str(tmp_path / "places")], check=True)
    out = subprocess.run([str(tmp_path / "places")], capture_output=True, text=True, check=True).stdout
    assert out == "20400 reads\n", out

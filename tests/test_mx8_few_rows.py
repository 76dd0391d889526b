"""The product of up to sixteen eight-bit rows: each wave of a workgroup takes one stage of k, and the rule that sends calls there
(csrc/mx8_rules.h, compiled for the CPU) admits no more of them, and calls with as many."""
import subprocess

import pytest

from linear_paths import CSRC

torch = pytest.importorskip("torch")

import test_gpu_mx8 as tm  # noqa: E402

DRIVER = r"""
#include <cstdio>
#include "mx8_rules.h"
int main() {
  int most = 0;
  for (int ld = 32; ld <= 1 << 20; ld += 32)
    if (afno::mx8_few_rows(1, ld)) most = ld;
  printf("%d %d", most, 128 * afno::kFewRowsWaves);
}
"""


def test_no_stage_without_a_call(tmp_path):
    (tmp_path / "rows.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-I" + CSRC, str(tmp_path / "rows.cpp"), "-o", str(tmp_path / "rows")], check=True)
    most, room = subprocess.run([str(tmp_path / "rows")], capture_output=True, text=True, check=True).stdout.split()
    assert most == room


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [1, 32, 33, 96, 127, 128, 129, 250, 1024, 1900, 1921, 2016, 2017, 2047, 2048, 2049])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17])
def test_few_rows(M, K, dtype):
    """No stage, part of one, all of them, and the first sizes behind the rule."""
    tm.check_linear(M, K, 70, dtype, "gelu", 0.1, True, True, backward=False, seed=M + K)

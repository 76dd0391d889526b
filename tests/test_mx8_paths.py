"""Every kernel that a product of eight-bit rows can take has a case: the library's rules (csrc/mx8_rules.h), compiled for
the CPU, say which kernels the sizes in use reach and which the cases run; the cases run on the GPU against the float64
oracle, elementwise, with the bounds of test_gpu_mx8.py.  The workspace of splits holds their sums at every size."""
import itertools
import os
import subprocess

import pytest

from linear_paths import CSRC

torch = pytest.importorskip("torch")

import test_gpu_mx8 as tm  # noqa: E402

DRIVER = r"""
#include <cstdio>
#include "mx8_rules.h"
using namespace afno;
int main() {
  long long M, K, N;
  int es;
  while (scanf("%d %lld %lld %lld", &es, &M, &K, &N) == 4) {
    const int64_t ld = ceil_div(K, 32) * 32;
    if (mx8_few_rows(M, ld)) { printf("rows 1\n"); continue; }
    const Cut c = cut_mx8(M, N, ld, es);
    printf("%d %d", c.tile, c.splits);
    if (c.kper % 128 || c.kper * c.splits < ld || c.kper * (c.splits - 1) >= ld) printf(" CUT");
    if (part_of(M, N, c) > mx8_part_bytes(M, N, ld, es)) printf(" OVERRUN");
    if (c.splits > 1 && (c.tile != 64)) printf(" UNSPLIT KERNEL");
    printf("\n");
  }
}
"""

# dtype, M, K, N, activation, p, residual, odd addresses
PATHS = [
    ("bf16", 1, 1000, 4100, "gelu", 0.1, True, False),      # rows
    ("bf16", 16, 2048, 65, "none", 0.0, True, True),
    ("fp32", 3, 1984, 130, "gelu", 0.1, True, True),
    ("fp32", 16, 33, 1000, "relu", 0.0, False, False),
    ("bf16", 17, 4096, 520, "gelu", 0.1, True, False),      # 64, split in four
    ("bf16", 5, 2080, 100, "gelu", 0.1, True, True),        # in three stages and two, the last not whole
    ("fp32", 60, 3000, 77, "gelu", 0.1, True, False),
    ("bf16", 16, 10000, 33, "relu", 0.1, True, False),
    ("bf16", 700, 130, 700, "gelu", 0.0, False, True),      # 64, whole
    ("fp32", 5000, 1100, 300, "gelu", 0.1, True, True),
    ("bf16", 5000, 500, 600, "gelu", 0.1, True, True),      # 128
    ("bf16", 5000, 1100, 600, "relu", 0.0, True, False),
    ("fp32", 5000, 500, 600, "gelu", 0.1, True, True),
    ("fp32", 5000, 1100, 600, "relu", 0.0, True, False),
    ("fp32", 10300, 70, 1030, "gelu", 0.1, False, False),
    ("fp32", 6000, 384, 600, "none", 0.0, False, True),
    # 256: stages of 128 k's by fours, what is left of them, and of a stage; up to 16 blocks of scales and more
    ("bf16", 10300, 512, 1030, "gelu", 0.1, False, False),
    ("bf16", 10300, 520, 1030, "none", 0.1, True, False),
    ("bf16", 10300, 770, 1040, "gelu", 0.0, False, True),
    ("bf16", 10300, 900, 1030, "relu", 0.1, True, False),
    ("bf16", 10300, 1024, 1025, "gelu", 0.1, False, False),
    ("bf16", 10300, 1730, 1030, "gelu", 0.1, True, False),
    ("bf16", 10300, 100, 1030, "gelu", 0.0, True, True),
    ("bf16", 10300, 256, 1056, "none", 0.0, False, False),
    ("bf16", 10300, 384, 1030, "gelu", 0.1, False, False),
]
ROWS = (1, 2, 3, 16, 17, 64, 65, 100, 129, 200, 300, 513, 1000, 1030, 2048, 2100, 4104, 5000, 8192, 8200, 10368, 16384, 16500,
        33000, 64800)
WIDTHS = (1, 2, 7, 8, 16, 33, 64, 65, 100, 128, 130, 200, 264, 333, 512, 520, 1000, 1024, 1029, 2048, 2056, 4096, 4099, 8200, 16384,
          100000)


@pytest.fixture(scope="module")
def kinds(tmp_path_factory):
    d = tmp_path_factory.mktemp("mx8_paths")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I" + CSRC, str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def walk(calls):
        lines = "".join("{} {} {} {}\n".format(*c) for c in calls)
        out = subprocess.run([str(d / "driver")], input=lines, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
        assert len(out) == len(calls)
        for c, line in zip(calls, out):
            assert len(line.split()) == 2, (c, line)
        return {(c[0], line.split()[0], int(line.split()[1]) > 1) for c, line in zip(calls, out)}

    return walk


def test_every_reachable_kernel_has_a_case(kinds):
    size = {"fp32": 4, "bf16": 2}
    reached = kinds([(es, M, K, N) for es, M, K, N in itertools.product((2, 4), ROWS, WIDTHS, WIDTHS)])
    cases = kinds([(size[c[0]], *c[1:4]) for c in PATHS])
    assert reached == cases
    assert {(2, "256", False), (2, "128", False), (4, "64", True), (4, "128", False)} <= reached and os.path.isdir(CSRC)


@pytest.mark.gpu
@pytest.mark.parametrize("case", PATHS, ids=lambda c: "{}_{}x{}x{}_{}{}".format(*c[:5], "_odd" if c[7] else ""))
def test_path(case):
    dtype, M, K, N, act, p, residual, odd = case
    tm.check_linear(M, K, N, dtype, act, p, True, residual, backward=False, odd=odd, seed=K)

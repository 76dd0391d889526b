"""Which kernel each product of a linear call takes, by the library's own rules (csrc/linear_rules.h)
compiled for the CPU: shared by the test that every reachable one has a case and by those cases."""
from __future__ import annotations

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2208_05419_amd", "csrc")

DRIVER = r"""
#include <cstdio>
#include "linear_rules.h"
using namespace afno;

static void show(const char* layout, const Product& p, int es, const Layout& l) {
  const Path r = product_path(p, es);
  if (r.rows) printf("%s rows%d 1", layout, p.M >= 3 ? 4 : (int)p.M);
  else printf("%s %s%d %d", layout, r.units ? "tile" : "reg", r.cut.tile, r.cut.splits);
  // the splits' sums fit behind everything else
  const size_t part = r.rows ? 0 : part_of(p.M, p.N, r.cut);
  if (l.part + part > l.bytes) printf(" OVERRUN");
  // whole units: what the direct-to-LDS kernels may read lies within the operand's rows
  if (!r.rows && r.units) {
    const int64_t ue = 16 / es, ka = p.ar ? 0 : ceil_div(p.K, ue) * ue, kb = p.br ? 0 : ceil_div(p.K, ue) * ue;
    if (ka > p.lda || kb > p.ldb || (p.ar && p.ma > p.lda) || (p.br && p.nb > p.ldb) || (p.ar && p.M > p.ma) || (p.br && p.N > p.nb))
      printf(" BEYOND");
    const int64_t stage = 128 / es;
    if (r.cut.kper % stage || r.cut.kper * r.cut.splits < p.K || r.cut.kper * (r.cut.splits - 1) >= p.K) printf(" CUT");
  }
  printf("\n");
}

// lines of es M K N x16 w16 g16 factor (an activation or dropout)
int main() {
  long long M, K, N;
  int es, x16, w16, g16, factor;
  while (scanf("%d %lld %lld %lld %d %d %d %d", &es, &M, &K, &N, &x16, &w16, &g16, &factor) == 8) {
    LinearSizes s = {M, K, N, es, x16 != 0, w16 != 0, true, false, false, false, false};
    const Layout f = forward_layout(s);
    show("forward", forward_product(s, f), es, f);
    s.g16 = g16 != 0;
    s.dx = s.dw = s.db = true;
    s.factor = factor != 0;
    const Layout b = backward_layout(s);
    show("dx", dx_product(s, b), es, b);
    show("dw", dw_product(s, b), es, b);
    // a query with the same sizes and every array misplaced is room enough for any of them
    LinearSizes q = s;
    q.x16 = q.w16 = q.g16 = false;
    q.factor = true;
    const Layout fq = forward_layout(q), bq = backward_layout(q);
    printf("%s\n", fq.bytes >= f.bytes && bq.bytes >= b.bytes ? "room" : "SHORT");
  }
}
"""


def build(directory: str) -> str:
    src, exe = os.path.join(directory, "linear_paths.cpp"), os.path.join(directory, "linear_paths")
    with open(src, "w") as f:
        f.write(DRIVER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + CSRC,
                    src, "-o", exe], check=True)
    return exe


def walk(exe: str, calls):
    """For each call (es, M, K, N, x16, w16, g16, factor) its products' (layout, kernel, splits)."""
    text = "\n".join(" ".join(str(int(v)) for v in c) for c in calls) + "\n"
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
    got = []
    for i in range(len(calls)):
        lines = out[4 * i:4 * i + 4]
        assert lines[3] == "room", (calls[i], lines)
        three = [line.split() for line in lines[:3]]
        assert all(len(t) == 3 for t in three), (calls[i], lines)
        got.append([(t[0], t[1], int(t[2])) for t in three])
    return got

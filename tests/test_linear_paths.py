"""Every kernel that a product of a linear call can take has a case: the library's rules (csrc/linear_rules.h), compiled
for the CPU, say which kernels the sizes in use reach and which the cases run; the cases run on the GPU
against the float64 oracle, elementwise, with the bounds of test_gpu_train.py."""
import itertools

import pytest

import linear_paths

torch = pytest.importorskip("torch")

import test_gpu_train as tg  # noqa: E402

PATHS = [
    # dtype, M, K, N, activation, p, residual, odd addresses: sizes that no tile divides, in each direction
    ("bf16", 4200, 1032, 4104, "gelu", 0.1, True, False),    # 256 tiles: whole forward, split over k in both gradients
    ("bf16", 520, 10248, 2056, "gelu", 0.1, True, False),    # split forward, dw whole; dx in 128 tiles
    ("bf16", 136, 2056, 2056, "gelu", 0.1, True, False),     # split 64 tiles forward and dx; dw in 128 tiles, whole
    ("bf16", 200, 4096, 264, "gelu", 0.25, True, False),     # split 64 tiles of few rows, joined with every epilogue
    ("bf16", 4104, 1032, 1032, "relu", 0.1, False, False),   # 128 tiles, whole, forward and dx
    ("bf16", 136, 200, 8200, "gelu", 0.0, False, False),     # long sums: split 128 tiles in dx,
    ("bf16", 136, 8200, 200, "gelu", 0.1, True, False),      # forward,
    ("bf16", 10368, 200, 136, "none", 0.0, False, False),    # and dw
    ("bf16", 300, 9, 269, "none", 0.0, True, True),          # no units and not worth a copy: 64 tiles, split in dx and dw
    ("bf16", 2100, 9, 77, "gelu", 0.1, True, True),
    ("bf16", 77, 515, 3, "relu", 0.1, True, True),
    ("bf16", 16500, 9, 131, "gelu", 0.1, True, False),       # 128 tiles, whole, forward,
    ("bf16", 16500, 131, 1, "none", 0.0, False, False),      # dx,
    ("bf16", 1, 1001, 4099, "none", 0.0, True, False),       # and dw
    ("fp32", 16500, 131, 133, "gelu", 0.1, True, False),     # no units: 128 tiles whole, split in dw
    ("fp32", 131, 2051, 2053, "gelu", 0.1, True, False),     # split, dw whole
    ("fp32", 40, 8200, 264, "gelu", 0.1, True, False),       # split 64 tiles forward, 128 tiles in dw
    ("fp32", 200, 4096, 264, "gelu", 0.25, True, False),
    ("fp32", 136, 200, 8200, "gelu", 0.0, False, False),     # long sums: split 128 tiles in dx,
    ("fp32", 136, 8200, 200, "gelu", 0.1, True, False),      # forward,
    ("fp32", 10368, 200, 136, "none", 0.0, False, False),    # and dw
    ("fp32", 8200, 1032, 1544, "gelu", 0.1, True, False),    # 128 tiles forward and dx; dw split for two workgroups a CU
]

# the sizes to walk over: those of the tests and a logarithmic sweep to 64,800 rows and 16,384 channels, each with
# its neighbours that no unit or tile divides
ROWS = (1, 2, 3, 16, 17, 64, 65, 100, 129, 200, 300, 513, 1000, 1030, 2048, 2100, 4104, 5000, 8192, 8200, 10368, 16384, 16500,
        33000, 64800)
WIDTHS = (1, 2, 3, 7, 8, 9, 16, 33, 64, 65, 72, 100, 128, 130, 131, 200, 264, 333, 512, 520, 1000, 1024, 1029, 2048, 2056, 4096,
          4099, 8192, 8200, 16384)


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    return linear_paths.build(str(tmp_path_factory.mktemp("linear_paths")))


def _kinds(driver, calls):
    """(element size, layout, kernel, whether k is split) that the calls' products take."""
    return {(c[0], layout, kernel, splits > 1)
            for c, products in zip(calls, linear_paths.walk(driver, calls)) for layout, kernel, splits in products}


def test_every_reachable_kernel_has_a_case(driver):
    """(walk() also checks at every size that the splits' sums fit into the workspace behind everything else, that the
    query's answer is room enough at any address, and that no operand is read behind its rows.)"""
    reachable = _kinds(driver, [(es, M, K, N, a, a, a, f) for es, M, K, N, a, f in
                                itertools.product((2, 4), ROWS, WIDTHS, WIDTHS, (0, 1), (0, 1))])
    calls = [({"bf16": 2, "fp32": 4}[c[0]], *c[1:4], *[not c[7]] * 3, c[4] != "none" or c[5] > 0) for c in PATHS]
    for c in tg.LINEAR:
        calls += [(es, *c[:3], 1, 1, 1, c[3] != "none" or c[4] > 0) for es in (2, 4)]
    missing = reachable - _kinds(driver, calls)
    assert not missing, sorted(missing)
    # the bf16 products' three large tiles and both kinds of split are among them, so the walk sees what it should
    assert {(2, d, "tile256", s) for d in ("forward", "dx", "dw") for s in (False, True)} <= reachable
    assert len(reachable) >= 56


def test_mixed_addresses(driver):
    """Arrays that are aligned one by one: room and bounds hold for each of the eight combinations."""
    linear_paths.walk(driver, list(itertools.product((2, 4), (1, 17, 300, 4104), (9, 64, 333, 2056), (8, 77, 512, 2050),
                                                     (0, 1), (0, 1), (0, 1), (0, 1))))


def test_largest_sizes(driver):
    """At the limits of a call (2^25 rows, 2^20 channels, 2^34 values) no size wraps."""
    calls = [(es, M, K, N, a, a, a, 1) for es in (2, 4) for a in (0, 1) for M, K, N in
             ((2 ** 25, 1, 1), (2 ** 25, 512, 512), (2 ** 25, 511, 3), (2 ** 14, 2 ** 20, 1), (1, 2 ** 20, 2 ** 14),
              (2 ** 14, 2 ** 20, 2 ** 14), (2 ** 14 - 1, 2 ** 14 + 1, 2 ** 20 - 1), (17, 2 ** 14, 2 ** 20))]
    assert len(linear_paths.walk(driver, calls)) == len(calls)


@pytest.mark.gpu
@pytest.mark.parametrize("case", PATHS, ids=lambda c: "{}_{}x{}x{}_{}_p{}{}".format(*c[:6], "_odd" if c[7] else ""))
def test_against_the_oracle(case):
    dtype, M, K, N, act, p, residual, odd = case
    tg.check_linear(M, K, N, dtype, act, p, residual=residual, odd=odd, seed=M + N)

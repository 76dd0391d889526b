"""The host code of the linear products, LayerNorm and dropout under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): refusals, calls without work, and the workspace queries at and just above every
limit.  Nothing here passes the checks that stand before the first HIP call, so the library is built with
its host code alone (ten seconds) and run in a child process with the sanitizer's runtime preloaded."""
import glob
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2208_05419_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _runtime():
    found = glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    return found[0] if found else None


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    if shutil.which(HIPCC) is None or _runtime() is None:
        pytest.skip("hipcc or its sanitizer runtime missing")
    d = tmp_path_factory.mktemp("sanitized")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]

    def run(*cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return r.stdout

    objs = []
    for name in ("afno_kernels.hip", "afno_api.cpp"):
        objs.append(str(d / (name + ".o")))
        run(HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fPIC", *san,
            "-Xarch_host", "-fno-omit-frame-pointer", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
            "-c", "-x", "hip", os.path.join(CSRC, name), "-o", objs[-1])
    # an empty bundle of device code in the place of each unit's
    wanted = [line.split()[-1] for o in objs for line in run("nm", "-u", o).splitlines() if "__hip_fatbin_" in line]
    empty = d / "empty.c"
    empty.write_text("".join(f'const char {w}[32] = "__CLANG_OFFLOAD_BUNDLE__";\n' for w in wanted))
    run("gcc", "-fPIC", "-c", str(empty), "-o", str(d / "empty.o"))
    lib = str(d / "libafno_host_asan.so")
    run(HIPCC, "--offload-arch=gfx950", "-shared", *san, "-Xarch_host", "-shared-libsan", *objs, str(d / "empty.o"), "-o", lib)
    return lib


def test_train_entry_points_under_asan_ubsan(library):
    script = f"""
    import itertools
    import paper_2208_05419_amd as afno
    from paper_2208_05419_amd import afno as binding
    binding.LIB_PATH = {library!r}
    import tests.test_train_refusals as t
    INV, UNS, ALI = t.INV, t.UNS, t.ALI

    # the refusals of the ordinary build, and every argument that is NULL, negative or huge by itself
    for mark in t.test_refused.pytestmark:
        for call, want, kw in mark.args[1]:
            assert call(**kw) == want, (call.__name__, kw)
            assert afno.afno_last_error()
    t.test_nothing_to_do_needs_no_gpu()
    t.test_workspace_sizes()
    t.test_workspace_sizes_of_the_widest_rows()
    big = 2 ** 63 - 1
    for call, sizes in ((t.linear, "MKN"), (t.linear_bwd, "MKN"), (t.norm, "MC"), (t.norm_bwd, "MC"), (t.drop, "n")):
        for s, v in itertools.product(sizes, (big, -big - 1, 2 ** 62, 2 ** 35)):
            for dtype in (0, 1):
                assert call(**{{s: v, "dtype": dtype}}) in (INV, UNS), (call.__name__, s, v)
        if call not in (t.drop, t.norm, t.norm_bwd):
            assert call(act=2 ** 31 - 1) == INV and call(act=-2 ** 31) == INV
        assert call(dtype=2 ** 31 - 1) == INV

    # the queries at the limits, and one beyond each
    rows, cols, values = 2 ** 25, 2 ** 20, 2 ** 34
    for dtype, aligned in itertools.product((0, 1), (0, 1)):
        for q in (afno.afno_linear_forward_workspace, afno.afno_linear_backward_workspace):
            for M, K, N in ((rows, 512, 512), (rows, 511, 1), (rows, 1, 1), (2 ** 14, cols, 1), (2 ** 14, cols, 2 ** 14),
                            (2 ** 14 - 1, cols - 1, 2 ** 14 - 1), (1, 2 ** 14, cols), (1, 1, 1), (17, 333, 77)):
                n = q(M, K, N, dtype, aligned)
                assert n >= 0, (q.__name__, M, K, N)
                # dz alone, where it is copied or made
                if q is afno.afno_linear_backward_workspace:
                    assert n >= M * N * (2 if dtype else 4)
            for M, K, N in ((rows + 1, 8, 8), (8, cols + 1, 8), (8, 8, cols + 1), (rows, 513, 8), (rows, 8, 513),
                            (8, cols, 2 ** 14 + 1), (big, 8, 8), (8, big, 8), (8, 8, big)):
                assert q(M, K, N, dtype, aligned) == UNS, (q.__name__, M, K, N)
            assert q(-1, 8, 8, dtype, aligned) == INV and q(8, -big, 8, dtype, aligned) == INV
        q = afno.afno_layer_norm_backward_workspace
        for M, C in ((rows, 512), (rows, 1), (values // cols, cols), (1, cols), (1, 1), (8, 8193), (8, 8192)):
            assert q(M, C, dtype) >= 2 * C * 4, (M, C)
        for M, C in ((rows + 1, 1), (1, cols + 1), (rows, 513), (values // cols + 1, cols), (big, 1), (1, big)):
            assert q(M, C, dtype) == UNS, (M, C)

    # a workspace one byte short, at every size of it
    for M, K, N in ((2100, 72, 2104), (300, 77, 333), (16, 64, 32)):
        need = afno.afno_linear_backward_workspace(M, K, N, t.BF16, 1)
        far = [0x100000000 * (i + 1) for i in range(9)]
        kw = dict(M=M, K=K, N=N, g=far[0], x=far[1], w=far[2], pre=far[3], dx=far[4], dw=far[5], db=far[6], counter=far[7],
                  ws=far[8])
        assert need > 0 and t.linear_bwd(**kw, have=need - 1) == INV
        assert str(need) in afno.afno_last_error()
    print("CHILD OK")
    """
    env = dict(os.environ, LD_PRELOAD=_runtime(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(script)], capture_output=True, text=True, env=env,
                       cwd=os.path.dirname(library), timeout=600)
    report = "AddressSanitizer" in r.stderr or "runtime error:" in r.stderr
    assert r.returncode == 0 and not report and "CHILD OK" in r.stdout, (r.returncode, r.stdout[-2000:], r.stderr[-4000:])

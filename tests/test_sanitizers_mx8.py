"""The host code of the operators in eight bits and the root-mean-square norm under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only), as test_sanitizers_train.py does it: refusals, calls without work, and the
workspace queries at and just above every limit."""
import os
import subprocess
import sys
import textwrap

from test_sanitizers_train import ROOT, _runtime, library  # noqa: F401


def test_mx8_entry_points_under_asan_ubsan(library):  # noqa: F811
    script = f"""
    import itertools
    import paper_2208_05419_amd as afno
    from paper_2208_05419_amd import afno as binding
    binding.LIB_PATH = {library!r}
    import tests.test_mx8_refusals as t
    INV, UNS, ALI = t.INV, t.UNS, t.ALI

    for call, want, kw in t.REFUSED:
        assert call(**kw) == want, (call.__name__, kw)
        assert afno.afno_last_error()
    t.test_nothing_to_do_needs_no_gpu()
    t.test_workspace_sizes()
    big = 2 ** 63 - 1
    for call, sizes in ((t.pack, "MC"), (t.unpack, "MC"), (t.norm, "MC"), (t.norm_bwd, "MC"), (t.linear, "MKN"), (t.linear_bwd, "MKN")):
        for s, v in itertools.product(sizes, (big, -big - 1, 2 ** 62, 2 ** 35)):
            for dtype in (0, 1):
                assert call(**{{s: v, "dtype": dtype}}) in (INV, UNS), (call.__name__, s, v)
        assert call(dtype=2 ** 31 - 1) == INV

    rows, cols, values = 2 ** 25, 2 ** 20, 2 ** 34
    fwd = lambda M, K, N, dtype, aligned: afno.afno_mx8_linear_forward_workspace(M, K, N, dtype)
    bwd = afno.afno_mx8_linear_backward_workspace
    for dtype, aligned in itertools.product((0, 1), (0, 1)):
        for q in (fwd, bwd):
            for M, K, N in ((rows, 512, 512), (rows, 511, 1), (rows, 1, 1), (2 ** 14, cols, 1), (2 ** 14, cols, 2 ** 14),
                            (2 ** 14 - 1, cols - 1, 2 ** 14 - 1), (1, 2 ** 14, cols), (1, 1, 1), (17, 333, 77)):
                n = q(M, K, N, dtype, aligned)
                assert n >= 0 and (q is fwd or n >= M * (N + K) * (2 if dtype else 4)), (M, K, N)
            for M, K, N in ((rows + 1, 8, 8), (8, cols + 1, 8), (8, 8, cols + 1), (rows, 513, 8), (rows, 8, 513),
                            (8, cols, 2 ** 14 + 1), (big, 8, 8), (8, big, 8), (8, 8, big)):
                assert q(M, K, N, dtype, aligned) == UNS, (M, K, N)
            assert q(-1, 8, 8, dtype, aligned) == INV and q(8, -big, 8, dtype, aligned) == INV
        q = afno.afno_rms_norm_backward_workspace
        for M, C in ((rows, 512), (rows, 1), (values // cols, cols), (1, cols), (1, 1), (8, 8193), (8, 8192)):
            assert q(M, C, dtype) >= C * 4, (M, C)
        for M, C in ((rows + 1, 1), (1, cols + 1), (rows, 513), (values // cols + 1, cols), (big, 1), (1, big)):
            assert q(M, C, dtype) == UNS, (M, C)
    print("CHILD OK")
    """
    env = dict(os.environ, LD_PRELOAD=_runtime(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(script)], capture_output=True, text=True, env=env,
                       cwd=os.path.dirname(library), timeout=600)
    report = "AddressSanitizer" in r.stderr or "runtime error:" in r.stderr
    assert r.returncode == 0 and not report and "CHILD OK" in r.stdout, (r.returncode, r.stdout[-2000:], r.stderr[-4000:])

"""The root-mean-square norm of rows whose squares float32 does not hold, down to its smallest number, with an eps that is 0 or as
small: result, eight bits and gradients against the float64 oracle, elementwise, with the bounds of test_gpu_mx8.py, which
count relative errors alone."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
import test_gpu_mx8 as tm
import test_gpu_train as tg
from gpu_util import say, to_f64
from oracle import mx8 as om

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

#: sizes of rows: ordinary ones, on either side of where the kernels change over, squares that are subnormal or 0, subnormal rows
SIZES = [1.0, 2.0 ** -49, 2.0 ** -51, 1e-18, 3e-20, 1e-23, 1e-30, 1e-38]
SUBNORMAL = {"fp32": 1e-42, "bf16": 1e-39}


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140, 2.0 ** -102, 2.0 ** -98])
@pytest.mark.parametrize("C", [1, 7, 333, 1024, 2048, 2049, 5000, 9001])
def test_small_rows(C, eps, dtype):
    say(f"[small rows] C={C} eps={eps} {dtype}")
    r = np.random.default_rng(C)
    sizes, h = [*SIZES, SUBNORMAL[dtype]], tg.HALF[dtype]
    M = 3 * len(sizes)
    size = np.resize(sizes, (M, 1))
    away = r.uniform(0.5, 2.0, (M, C)) * r.choice([-1.0, 1.0], (M, C))  # no row is 0: that of eps 0 has its own test
    x, xd = tg.store(size * away, dtype)
    ga, gad = tg.store(1 + 0.1 * r.standard_normal(C), dtype)
    # gradients that the smallest rows leave within float32: 1 / 1e-42 times 1e-10
    g, gd = tg.store(np.where(size < 1e-30, 1e-10, 1.0) * r.standard_normal((M, C)), dtype)
    out8, out = afno.mx8_empty((M, C), "cuda"), torch.empty_like(xd)
    afno.rms_norm_forward(xd, gad, eps=eps, out=out, out8=out8)
    d = afno.rms_norm_backward(gd, xd, gad, eps=eps)
    torch.cuda.synchronize()
    ref, e = om.rms_norm(x, ga, eps), tg.k(C) * tg.U
    # beside the relative errors what float32 flushes or rounds below its normal numbers (rows that a larger eps divides)
    least = 2.0 ** -126
    tg.close("out", out, ref, (e + h * 1.01) * np.abs(ref) + least)
    tm.close8("out8", out8, ref, e * np.abs(ref) + least)
    rms = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dx, dga = om.rms_norm_backward(g, x, ga, eps)
    a, hh = np.abs(g * ga), np.abs(x * rms)
    tg.close("dx", d["dx"], dx, rms * (2 * e * a + 5 * e * hh * (a * hh).mean(-1, keepdims=True)) + h * np.abs(dx) * 1.01)
    tg.close("dgamma", d["dgamma"], dga, (np.abs(g) * (hh * (e + tg.k(M) * tg.U) + least)).sum(0) + least)


@pytest.mark.parametrize("C", [64, 9001])
def test_rows_keep_to_themselves(C):
    """A small row, a row of zeros and an ordinary one side by side have the bits that they have alone."""
    x = torch.randn(9, C, device="cuda")
    x[::3] *= 1e-25
    x[4] = 0.0
    g, ga = torch.randn(9, C, device="cuda"), torch.ones(C, device="cuda")
    out, d = afno.rms_norm_forward(x, ga, eps=0.0), afno.rms_norm_backward(g, x, ga, eps=0.0)["dx"]
    assert torch.isnan(out[4]).all() and torch.isnan(d[4]).all()
    for i in (0, 1, 3, 5, 8):
        assert torch.isfinite(out[i]).all() and torch.isfinite(d[i]).all()
        assert torch.equal(out[i], afno.rms_norm_forward(x[i:i + 1], ga, eps=0.0)[0])
        assert torch.equal(d[i], afno.rms_norm_backward(g[i:i + 1], x[i:i + 1], ga, eps=0.0)["dx"][0])
    assert np.allclose((to_f64(out[::3]) ** 2).mean(-1), 1.0, rtol=1e-5)

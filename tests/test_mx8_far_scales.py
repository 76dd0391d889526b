"""Products of eight-bit rows whose blocks have scales at either end of the format, each beside its opposite, so that the
products are alike in size; on every kernel, against float64, with the bounds of test_gpu_mx8.py."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
import test_gpu_mx8 as tm
import test_gpu_train as tg

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N", [(1, 70), (16, 96), (300, 128), (5000, 600), (10300, 1030)])
@pytest.mark.parametrize("K", [256, 608])
def test_far_scales(M, N, K, dtype):
    r = np.random.default_rng(M + K)
    powers = r.permutation(np.resize([126, -109, 60, -43, 8], K // 32))
    some = lambda n, p: r.uniform(0.55, 1.9, (n, K)) * r.choice([-1.0, 1.0], (n, K)) * 2.0 ** np.repeat(p, 32)  # noqa: E731
    x, xd = tm.packed(some(M, powers))
    w, wd = tm.packed(some(N, 17 - powers))
    scales = xd.scales.view(torch.uint8)
    assert scales.min() <= 11 and scales.max() >= 245  # 1.9 2^-109 is 243 2^-116, 1.75 2^-109 448 2^-117; 1.75 2^126 448 2^118
    out = afno.mx8_linear_forward(xd, wd, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16)
    torch.cuda.synchronize()
    ref = x @ w.T
    tol = tg.k(K) * tg.U * (np.abs(x) @ np.abs(w).T) + tm.dropped(x, w.T, dtype)
    tg.close("out", out, ref, tol + 1.01 * tg.HALF[dtype] * np.abs(ref))

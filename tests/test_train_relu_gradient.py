"""ReLU's gradient selects: a unit whose value before the activation is not above zero passes on 0
whatever reaches it, an infinity or a NaN among them, in the oracle and on the GPU."""
import numpy as np
import pytest

from oracle import train as ot

BAD = (np.inf, -np.inf, np.nan)
OFF = (-2.0, 0.0, -0.0, -np.inf, np.nan)  # values before the activation that let nothing through


def _case(M, N, seed=3):
    """g, pre, and what reaches z: every bad gradient at every value that lets nothing through, spread over
    the rows and columns of an ordinary case."""
    r = np.random.default_rng(seed)
    g, pre = r.integers(-4, 5, (M, N)).astype(float), r.integers(1, 5, (M, N)) * r.choice([-1.0, 1.0], (M, N))
    want = np.where(pre > 0, g, 0.0)
    places = r.permutation(M * N)[:len(BAD) * len(OFF)]
    for at, (b, z) in zip(places, [(b, z) for b in BAD for z in OFF]):
        g.flat[at], pre.flat[at], want.flat[at] = b, z, 0.0
    return g, pre, want


def test_oracle():
    r = np.random.default_rng(0)
    g, pre, want = _case(9, 11)
    x, w = r.standard_normal((9, 5)), r.standard_normal((5, 11))
    for p in (0.0, 0.3):
        dx, dw, db, dz = ot.linear_backward(g, x, w, pre, "relu", p=p, seed=4)
        kept = ot.drop(want, p, 4)
        assert (dz == kept).all()
        assert np.isfinite(dx).all() and np.isfinite(dw).all() and (db == kept.sum(0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(7, 5, 9), (70, 64, 72), (33, 24, 1030)])
def test_gpu(M, K, N, dtype):
    """Small whole numbers in g, x and w: every sum is exact in single precision and in the stored type but for
    its one rounding, so the results are compared bit for bit with the rounded exact ones."""
    import paper_2208_05419_amd as afno
    from gpu_util import to_dev, to_f64
    from paper_2208_05419_amd import synth
    torch = pytest.importorskip("torch")
    put = lambda a: to_dev(synth.quantize(a, dtype), dtype)  # noqa: E731
    r = np.random.default_rng(M)
    x, w = (r.integers(-1, 2, s).astype(float) for s in ((M, K), (K, N)))
    g, pre, want = _case(M, N)
    d = afno.linear_backward(put(g), put(x), put(w), pre=put(pre), activation="relu")
    torch.cuda.synchronize()
    for name, ref in (("dx", want @ w.T), ("dw", x.T @ want), ("db", want.sum(0))):
        ref = synth.widen(synth.quantize(ref, dtype), dtype)
        assert (to_f64(d[name]) == ref).all(), name
    # an infinity at a unit that is on goes through
    on = put(np.full((M, N), 1.0))
    g[:] = 1.0
    g[M // 2, N // 2] = np.inf
    d = afno.linear_backward(put(g), put(x), put(w), pre=on, activation="relu")
    assert float(d["db"][N // 2]) == np.inf and torch.isfinite(d["db"][:N // 2]).all()

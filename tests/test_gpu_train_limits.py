"""The linear products, LayerNorm and dropout at the ends of their ranges: the widest rows, the most rows, the
largest probability, and calls that leave optional outputs out.  Bounds as in test_gpu_train.py."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
import test_gpu_train as tg
from gpu_util import say, to_f64
from oracle import train as ot

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

WIDEST, MOST = 2 ** 20, 2 ** 25


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, WIDEST, 5), (9, WIDEST, 24), (40, WIDEST - 3, 2), (2, 3, WIDEST), (9, 16, WIDEST), (5, 7, WIDEST - 3)])
def test_widest_linear(M, K, N, dtype):
    tg.check_linear(M, K, N, dtype, "gelu", 0.1, residual=True, seed=N % 1000)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_widest_norm(dtype):
    tg.check_norm(2, WIDEST, True, dtype, tg.store)


def _rows(t, at):
    return to_f64(t[torch.tensor(at, device="cuda")])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_most_rows(dtype):
    """2^25 rows: outputs in the first, middle and last of them, the sums over all of them against float64 on the GPU."""
    dt, h = (torch.float32 if dtype == "fp32" else torch.bfloat16), tg.HALF[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    K, N = 8, 12
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dt)  # noqa: E731
    x, w, g = normal(MOST, K), normal(K, N), normal(MOST, N)
    at = [0, 1, MOST // 2 - 1, MOST // 2, MOST - 65, MOST - 2, MOST - 1]
    out = afno.linear_forward(x, w)
    d = afno.linear_backward(g, x, w)
    torch.cuda.synchronize()
    say("[most rows] products ran")
    x64, w64, g64 = _rows(x, at), to_f64(w), _rows(g, at)
    ref = x64 @ w64
    tg.close("out", _rows(out, at), ref, tg.k(K) * tg.U * (np.abs(x64) @ np.abs(w64)) + h * np.abs(ref) * 1.01)
    ref = g64 @ w64.T
    tg.close("dx", _rows(d["dx"], at), ref, tg.k(N) * tg.U * (np.abs(g64) @ np.abs(w64).T) + h * np.abs(ref) * 1.01)

    def total(a, b):  # a^T b and |a|^T |b| over all rows, a chunk at a time in float64
        s, m = 0.0, 0.0
        for i in range(0, MOST, 2 ** 22):
            p, q = a[i:i + 2 ** 22].double(), b[i:i + 2 ** 22].double()
            s, m = s + p.t().contiguous() @ q, m + p.abs().t().contiguous() @ q.abs()
        return s.cpu().numpy(), m.cpu().numpy()

    s, m = total(x, g)
    tg.close("dw", d["dw"], s, tg.k(MOST) * tg.U * m + h * np.abs(s) * 1.01)
    one = torch.ones(MOST, 1, dtype=dt, device="cuda")
    s, m = total(one, g)
    tg.close("db", d["db"], s[0], tg.k(MOST) * tg.U * m[0] + h * np.abs(s[0]) * 1.01)
    del out, d
    ga = normal(N)
    y = afno.layer_norm_forward(g, ga, ga)
    n = afno.layer_norm_backward(y, g, ga)
    torch.cuda.synchronize()
    say("[most rows] norm ran")
    v, ga64, up = g64, to_f64(ga), _rows(y, at)
    rstd = 1 / np.sqrt(v.var(-1, keepdims=True) + 1e-6)
    e, hh = tg.norm_slack(v, rstd, N), np.abs((v - v.mean(-1, keepdims=True)) * rstd)
    ref = ot.layer_norm(v, ga64, ga64, 1e-6)
    tg.close("norm", up, ref, e * (1 + hh) * np.abs(ga64) + 4 * tg.U * (np.abs(ga64) + np.abs(ref)) + h * np.abs(ref) * 1.01)
    ref = ot.layer_norm_backward(up, v, ga64, 1e-6)[0]
    tg.close("norm dx", _rows(n["dx"], at), ref, tg.norm_dx_slack(np.abs(up * ga64), hh, rstd, e) + h * np.abs(ref) * 1.01)
    s, m = total(one, y)
    tg.close("dbeta", n["dbeta"], s[0], tg.k(MOST) * tg.U * m[0])


def test_one_row_too_many_is_refused():
    x = torch.empty(MOST + 1, 1, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(afno.AfnoError):
        afno.linear_forward(x, w)
    with pytest.raises(afno.AfnoError):
        afno.linear_backward(x, x, w)
    with pytest.raises(afno.AfnoError):
        afno.layer_norm_forward(x, w[0], w[0])
    with pytest.raises(afno.AfnoError):
        afno.layer_norm_backward(x, x, w[0])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_largest_probability(dtype):
    """One number in 65,536 is kept, and scaled by 65,536; p of half a step keeps everything unscaled."""
    n = 1 << 20
    x = torch.ones(n, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda")
    p = 65535 / 65536
    keep = ot.keep(n, p, 5)
    assert 0 < keep.sum() < 64
    assert (to_f64(afno.dropout_forward(x, p, 5)) == keep * 65536.0).all()
    assert torch.equal(afno.dropout_forward(x, 2.0 ** -17, 5), x)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_optional_outputs_left_out(dtype):
    """The same bits without pre and without sum_out, and with the caller's out."""
    r = np.random.default_rng(0)
    for M, K, N in ((1, 64, 40), (300, 72, 264), (77, 33, 19)):
        (_, x), (_, w), (_, b) = (tg.store(r.standard_normal(s), dtype) for s in ((M, K), (K, N), N))
        pre, out = (torch.empty(M, N, dtype=x.dtype, device="cuda") for _ in range(2))
        a = afno.linear_forward(x, w, b, activation="gelu", p=0.1, seed=1, pre=pre)
        assert torch.equal(afno.linear_forward(x, w, b, activation="gelu", p=0.1, seed=1), a)
        assert afno.linear_forward(x, w, b, activation="gelu", p=0.1, seed=1, out=out) is out and torch.equal(out, a)
    for C in (40, 333, 2056, 9001):
        (_, x), (_, res), (_, ga) = (tg.store(r.standard_normal(s), dtype) for s in ((9, C), (9, C), C))
        s = torch.empty_like(x)
        a = afno.layer_norm_forward(x, ga, ga, residual=res, sum_out=s)
        assert torch.equal(afno.layer_norm_forward(x, ga, ga, residual=res), a)
        assert torch.equal(afno.layer_norm_forward(s, ga, ga), a)

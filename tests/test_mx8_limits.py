"""The operators in eight bits and the root-mean-square norm where their range ends, and their workspaces where they hold
something: the widest rows, the most rows, offsets beyond 32 bits, exactly the bytes that the queries name between
fences and full of NaN, the library's own workspace, and captured calls without one.  Bounds as in test_gpu_mx8.py."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
import test_gpu_mx8 as tm
import test_gpu_train as tg
from gpu_util import say, to_f64
from oracle import mx8 as om
from oracle import train as ot
from test_train_workspaces import Fenced

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

WIDEST, MOST = 2 ** 20, 2 ** 25
CODE = {"fp32": 0, "bf16": 1}
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, WIDEST, 5), (9, WIDEST, 24), (40, WIDEST - 3, 2), (2, 3, WIDEST), (17, 16, WIDEST - 3)])
def test_widest_linear(M, K, N, dtype):
    tm.check_linear(M, K, N, dtype, "gelu", 0.1, residual=True, seed=N % 1000)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_widest_pack(dtype):
    x, xd = tg.store(np.random.default_rng(0).standard_normal((2, WIDEST)), dtype)
    t = afno.mx8_pack(xd)
    q, s = om.pack(x)
    got = tm.raw(t)
    assert (got[0] == q).all() and (got[1] == s).all()
    assert (to_f64(afno.mx8_unpack(t)) == om.unpack(q, s, WIDEST)).all()


def _rows8(t, at):
    """Those rows of an Mx8, as float64."""
    i = torch.tensor(at, device="cuda")
    q, s = t.values.view(torch.uint8)[i].cpu().numpy(), t.scales.view(torch.uint8)[i].cpu().numpy()
    return om.unpack(q, s, t.channels)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_most_rows(dtype):
    """2^25 rows: results in the first, middle and last of them, sums over all of them against float64 on the GPU."""
    h = tg.HALF[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    K, N = 8, 12
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(DT[dtype])  # noqa: E731
    x, w, g, ga = normal(MOST, K), normal(K, N), normal(MOST, N), normal(K)
    at = [0, 1, MOST // 2 - 1, MOST // 2, MOST - 65, MOST - 2, MOST - 1]
    rows = lambda t: to_f64(t[torch.tensor(at, device="cuda")])  # noqa: E731
    x8 = afno.mx8_pack(x)
    x64 = _rows8(x8, at)
    assert (x64 == om.unpack(*om.pack(rows(x)), K)).all()
    assert (rows(afno.mx8_unpack(x8)) == x64).all()
    w8 = afno.mx8_pack(w.t().contiguous())
    wt = tm.value8(w8).T
    out8 = afno.mx8_empty((MOST, N), "cuda")
    out = afno.mx8_linear_forward(x8, w8, dtype=DT[dtype], out=torch.empty(MOST, N, dtype=DT[dtype], device="cuda"), out8=out8)
    d = afno.mx8_linear_backward(g, x8, w, pre8=None)
    torch.cuda.synchronize()
    say("[most rows] products ran")
    ref = x64 @ wt
    tol = tg.k(K) * tg.U * (np.abs(x64) @ np.abs(wt)) + tm.dropped(x64, wt, dtype)
    tg.close("out", rows(out), ref, tol + h * np.abs(ref) * 1.01)
    tg.close("out8", _rows8(out8, at), ref, tol + 1.0001 * om.half_step(np.abs(ref) + tol))
    g64, w64 = rows(g), to_f64(w)
    tg.close("dx", rows(d["dx"]), g64 @ w64.T, tg.k(N) * tg.U * (np.abs(g64) @ np.abs(w64).T) + h * np.abs(g64 @ w64.T) * 1.01)
    xs = afno.mx8_unpack(x8, dtype=torch.float32)
    s = sum(xs[i:i + 2 ** 22].double().t().contiguous() @ g[i:i + 2 ** 22].double() for i in range(0, MOST, 2 ** 22)).cpu().numpy()
    m = sum(xs[i:i + 2 ** 22].double().abs().t().contiguous() @ g[i:i + 2 ** 22].double().abs() for i in range(0, MOST, 2 ** 22)).cpu().numpy()
    tg.close("dw", d["dw"], s, tg.k(MOST) * tg.U * m + h * np.abs(s) * 1.01)
    del out, out8, d, xs
    n8 = afno.mx8_empty((MOST, K), "cuda")
    y = afno.rms_norm_forward(x, ga, out=torch.empty_like(x), out8=n8)
    b = afno.rms_norm_backward(x, x, ga)
    torch.cuda.synchronize()
    say("[most rows] norm ran")
    v, ga64, e = rows(x), to_f64(ga), tg.k(K) * tg.U
    ref = om.rms_norm(v, ga64, 1e-6)
    tg.close("norm", rows(y), ref, (e + h * 1.01) * np.abs(ref))
    tg.close("norm8", _rows8(n8, at), ref, e * np.abs(ref) + 1.0001 * om.half_step(np.abs(ref) * (1 + e)))
    ref, _ = om.rms_norm_backward(v, v, ga64, 1e-6)
    r = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-6)
    a, hh = np.abs(v * ga64), np.abs(v * r)
    tg.close("norm dx", rows(b["dx"]), ref, r * (2 * e * a + 5 * e * hh * (a * hh).mean(-1, keepdims=True)) + h * np.abs(ref) * 1.01)


def test_one_row_too_many_is_refused():
    x = torch.empty(MOST + 1, 1, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    w8, x8 = afno.mx8_pack(one), afno.mx8_empty((MOST + 1, 1), "cuda")
    for call in (lambda: afno.mx8_pack(x), lambda: afno.mx8_unpack(x8), lambda: afno.rms_norm_forward(x, one[0]),
                 lambda: afno.rms_norm_backward(x, x, one[0]), lambda: afno.mx8_linear_forward(x8, w8),
                 lambda: afno.mx8_linear_backward(x, x8, one)):
        with pytest.raises(afno.AfnoError):
            call()


def test_offsets_beyond_32_bits():
    """Over 2^31 values, checked in their last rows."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    M, K, N, last = 1_050_000, 40, 2056, 300
    x8 = afno.mx8_pack(torch.randn(M, K, generator=gen, device="cuda").bfloat16())
    w8 = afno.mx8_pack(torch.randn(N, K, generator=gen, device="cuda").bfloat16())
    out8, pre8 = (afno.mx8_empty((M, N), "cuda") for _ in range(2))
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    afno.mx8_linear_forward(x8, w8, activation="gelu", p=0.3, seed=tg.SEED, offset=tg.OFFSET, out=out, out8=out8, pre8=pre8)
    at = list(range(M - last, M))
    x, w = _rows8(x8, at), tm.value8(w8).T
    z = x @ w
    ez = tg.k(K) * tg.U * (np.abs(x) @ np.abs(w)) + tm.dropped(x, w, "bf16")
    tg.close("pre8", _rows8(pre8, at), z, ez + 1.0001 * om.half_step(np.abs(z) + ez))
    keep = tg.keep_from((M - last) * N, last * N, 0.3).reshape(last, N)
    y = ot.act(z, "gelu")
    ref = np.where(keep, y * tg.scale_of(0.3), 0.0)
    tol = keep * tg.scale_of(0.3) * (1.13 * ez + 1.4e-5 * np.abs(y) + 1.2e-18)
    tg.close("out", out[-last:], ref, tol + 2.0 ** -8 * 1.01 * np.abs(ref))
    tg.close("out8", _rows8(out8, at), ref, tol + 1.0001 * om.half_step(np.abs(ref) + tol))
    d = afno.mx8_linear_backward(out, x8, tm.store(w, "bf16")[1], pre8=pre8, activation="gelu", need_dw=False)
    g, wb = to_f64(out[-last:]), tm.store(w, "bf16")[0]
    _, _, _, dz = ot.linear_backward(g, x, wb, _rows8(pre8, at), "gelu")
    bound = tg.k(N) * tg.U * (np.abs(dz) @ np.abs(wb).T) + (3e-7 * np.abs(g)) @ np.abs(wb).T + 6 * 2.0 ** -8 * np.sqrt((dz * dz) @ (wb * wb).T)
    tg.close("dx", d["dx"][-last:], dz @ wb.T, bound + 2.0 ** -8 * 1.01 * np.abs(dz @ wb.T))
    del d, pre8
    assert (to_f64(afno.mx8_unpack(out8)[-last:]) == _rows8(out8, at)).all()
    again = afno.mx8_pack(out)
    assert (_rows8(again, at) == om.unpack(*om.pack(g), N)).all()
    del again
    ga = torch.ones(N, dtype=torch.bfloat16, device="cuda")
    afno.rms_norm_forward(out, ga, out8=out8)
    ref, e = om.rms_norm(g, 1.0, 1e-6), tg.k(N) * tg.U
    tg.close("norm8", _rows8(out8, at), ref, e * np.abs(ref) + 1.0001 * om.half_step(np.abs(ref) * (1 + e)))


# dtype, M, K, N, aligned arrays
WORKSPACES = [("bf16", 40, 4100, 77, True), ("fp32", 40, 4100, 77, True), ("bf16", 2100, 77, 2099, True), ("bf16", 2100, 72, 2104, False),
              ("fp32", 2100, 72, 520, True), ("fp32", 131, 2051, 2053, True), ("bf16", 300, 9, 269, False), ("bf16", 4200, 1032, 4104, True)]


@pytest.mark.parametrize("case", WORKSPACES, ids=lambda c: "{}_{}x{}x{}{}".format(*c[:4], "" if c[4] else "_odd"))
def test_linear_in_exactly_its_bytes(case):
    dtype, M, K, N, aligned = case
    code, r = CODE[dtype], np.random.default_rng(0)
    put = (lambda a: tg.store(a, dtype)[1]) if aligned else (lambda a: tg.misplaced(a, dtype)[1])
    x8, w8, pre8 = (tm.packed(r.standard_normal(s))[1] for s in ((M, K), (N, K), (M, N)))
    g, w = put(r.standard_normal((M, N))), put(r.standard_normal((K, N)))
    want = [afno.mx8_linear_forward(x8, w8, dtype=DT[dtype])]
    want += list(afno.mx8_linear_backward(g, x8, w, pre8=pre8, activation="gelu").values())
    st = torch.cuda.current_stream().cuda_stream
    p8 = lambda t: (t.values.data_ptr(), t.scales.data_ptr())  # noqa: E731
    out, (dx, dw, db) = torch.empty(M, N, dtype=DT[dtype], device="cuda"), (torch.empty_like(t) for t in want[1:])
    for fenced in (True, False):  # exactly the bytes, then the library's own workspace
        [t.zero_() for t in (out, dx, dw, db)]
        need = afno.afno_mx8_linear_forward_workspace(M, K, N, code)
        f = Fenced(need) if need and fenced else None
        assert afno.afno_mx8_linear_forward(*p8(x8), *p8(w8), None, None, M, K, N, 0, 0.0, 0, 0, None, code, out.data_ptr(), None, None,
                                            None, None, f and f.ptr, need if f else 0, st) == afno.AFNO_OK
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and (f is None or f.whole())
        need = afno.afno_mx8_linear_backward_workspace(M, K, N, code, int(aligned))
        f = Fenced(need) if fenced else None
        assert afno.afno_mx8_linear_backward(g.data_ptr(), *p8(x8), w.data_ptr(), *p8(pre8), M, K, N, 2, 0.0, 0, 0, None, code, dx.data_ptr(),
                                             dw.data_ptr(), db.data_ptr(), f and f.ptr, need if f else 0, st) == afno.AFNO_OK
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want[1:])) and (f is None or f.whole())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,C", [(1500, 333), (900, 2056), (300, 9001)])
def test_norm_in_exactly_its_bytes(M, C, dtype):
    r = np.random.default_rng(1)
    g, x = (tg.store(r.standard_normal((M, C)), dtype)[1] for _ in range(2))
    ga = tg.store(r.standard_normal(C), dtype)[1]
    want = afno.rms_norm_backward(g, x, ga)
    need = afno.afno_rms_norm_backward_workspace(M, C, CODE[dtype])
    dx, dga, f = torch.empty_like(g), torch.empty(C, device="cuda"), Fenced(need)
    for ws in (f.ptr, None):
        dga.zero_()
        assert afno.afno_rms_norm_backward(g.data_ptr(), x.data_ptr(), ga.data_ptr(), None, M, C, 1e-6, CODE[dtype], dx.data_ptr(),
                                           dga.data_ptr(), ws, need if ws else 0, torch.cuda.current_stream().cuda_stream) == afno.AFNO_OK
        torch.cuda.synchronize()
        assert torch.equal(dx, want["dx"]) and torch.equal(dga, want["dgamma"]) and f.whole()


def test_captured_calls_bring_their_workspace():
    """Without one they are refused and record nothing; the calls that need none are taken, as often as there are."""
    r = np.random.default_rng(2)
    x8, w8 = (tm.packed(r.standard_normal(s))[1] for s in ((40, 4100), (77, 4100)))
    x = torch.randn(40, 96, device="cuda")
    out, n8, y = torch.empty(40, 77, dtype=torch.bfloat16, device="cuda"), afno.mx8_empty((40, 96), "cuda"), torch.empty_like(x)
    p8 = lambda t: (t.values.data_ptr(), t.scales.data_ptr())  # noqa: E731
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        for _ in range(3):
            afno.rms_norm_forward(x, x[0], out8=n8)
            afno.mx8_unpack(n8, out=y)
        assert afno.afno_mx8_linear_forward(*p8(x8), *p8(w8), None, None, 40, 4100, 77, 0, 0.0, 0, 0, None, 1, out.data_ptr(), None, None, None,
                                            None, None, 0, s.cuda_stream) == afno.AFNO_ERR_UNSUPPORTED
    assert "captured" in afno.afno_last_error()
    want = afno.mx8_unpack(afno.rms_norm_forward(x, x[0].clone(), out8=afno.mx8_empty((40, 96), "cuda")), dtype=torch.float32)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_packed_rows_of_a_larger_tensor():
    """Whole rows of an Mx8 are one: a slice goes in and comes out in place."""
    r = np.random.default_rng(4)
    x, x8 = tm.packed(r.standard_normal((70, 333)))
    part = afno.Mx8(x8.values[13:50], x8.scales[13:50], 333)
    assert (to_f64(afno.mx8_unpack(part)) == x[13:50]).all()
    _, w8 = tm.packed(r.standard_normal((40, 333)))
    assert torch.equal(afno.mx8_linear_forward(part, w8), afno.mx8_linear_forward(x8, w8)[13:50])
    grid = afno.Mx8(x8.values.reshape(7, 10, 352), x8.scales.reshape(7, 10, 11), 333)
    assert torch.equal(afno.mx8_linear_forward(grid, w8), afno.mx8_linear_forward(x8, w8).reshape(7, 10, 40))


def test_norm_of_a_sum_past_float32_and_of_zeros_without_eps():
    """A row whose sum of squares float32 does not hold gives zeros and passes gsum on; 0 / 0 is NaN; other rows as alone."""
    x = torch.randn(4, 64, device="cuda")
    x[1], x[2] = 1e19, 0.0  # 64e38 and 0
    ga, g = torch.ones(64, device="cuda"), torch.randn(4, 64, device="cuda")
    out, out8 = torch.empty_like(x), afno.mx8_empty((4, 64), "cuda")
    afno.rms_norm_forward(x, ga, eps=0.0, out=out, out8=out8)
    dx = afno.rms_norm_backward(g, x, ga, eps=0.0, gsum=g)["dx"]
    got8 = afno.mx8_unpack(out8, dtype=torch.float32)
    assert not out[1].any() and not got8[1].any() and torch.equal(dx[1], g[1])
    assert torch.isnan(out[2]).all() and torch.isnan(got8[2]).all() and torch.isnan(dx[2]).all()
    for i in (0, 3):
        assert torch.equal(out[i], afno.rms_norm_forward(x[i:i + 1], ga, eps=0.0)[0])
        assert torch.equal(dx[i], afno.rms_norm_backward(g[i:i + 1], x[i:i + 1], ga, eps=0.0, gsum=g[i:i + 1])["dx"][0])

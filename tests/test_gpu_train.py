"""The linear products, LayerNorm and dropout on the GPU against the float64 oracle (oracle/train.py) on
the same stored inputs, elementwise.

Bounds, with u = 2^-24 and h = eps / 2 of the storage type (one rounding): a sum of n products in
single precision is off by at most k(n) u times the sum of their magnitudes, k(n) = 4 sqrt(n) + 16
(rounding errors that add up like random ones, four standard deviations, and a few for the epilogue;
the worst case is n u).  GELU is within 7e-7 of its size (7e-6 below -3, where it is under 4e-3) and has
slopes up to 1.13; its slope is within 3e-7.  A sum of rounded factors (dz in bf16) is off by at most
6 h times the root of the sum of its squared terms: the roundings are independent, of standard
deviation at most h / sqrt(3) of a term, and a single one is at most h."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
from gpu_util import say, to_dev, to_f64
from oracle import block as oblock
from oracle import train as ot
from paper_2208_05419_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
SEED, OFFSET = 0x0123456789ABCDEF, 5 << 33


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    afno.load_library()


def k(n):
    return 4.0 * np.sqrt(n) + 16.0


def store(a, dtype):
    """The stored values of float64 numbers (float64) and their device tensor."""
    st = synth.quantize(a, dtype)
    return synth.widen(st, dtype), to_dev(st, dtype)


def close(name, got, ref, tol):
    err = np.abs((to_f64(got) if not isinstance(got, np.ndarray) else got) - ref)
    worst = float(np.max(err / np.maximum(tol, 1e-300))) if err.size else 0.0
    say(f"  {name}: {worst:.3f} of the bound")
    assert np.isfinite(err).all() and (err <= tol).all(), (name, worst)


def rng_args(p, counter=None):
    """Arguments of the call and of the oracle."""
    if not p:
        return {}, {}
    c = None if counter is None else torch.tensor([counter], dtype=torch.int64, device="cuda")
    return (dict(p=p, seed=SEED, offset=OFFSET, counter=c),
            dict(p=p, seed=SEED, offset=OFFSET, counter=counter or 0))


def scale_of(p):
    return 65536.0 / (65536 - ot.threshold(p))


def check_linear(M, K, N, dtype, act, p=0.0, bias=True, residual=False, pre=True, backward=True, odd=False, seed=0):
    say(f"[linear] {M}x{K}x{N} {dtype} {act} p={p} bias={bias} residual={residual} odd={odd}")
    r = np.random.default_rng(seed)
    put = (lambda a: misplaced(a, dtype)) if odd else (lambda a: store(a, dtype))
    x, xd = put(r.standard_normal((M, K)))
    w, wd = put(r.standard_normal((K, N)) / np.sqrt(K))
    b, bd = put(r.standard_normal(N)) if bias else (None, None)
    res, resd = put(r.standard_normal((M, N))) if residual else (None, None)
    call, want = rng_args(p, 77)
    ref, z = ot.linear(x, w, b, act, res, **want)
    pred = torch.empty(M, N, dtype=xd.dtype, device="cuda") if pre else None
    out = afno.linear_forward(xd, wd, bd, activation=act, residual=resd, pre=pred, **call)
    torch.cuda.synchronize()
    h = HALF[dtype]
    ez = k(K) * U * (np.abs(x) @ np.abs(w) + (0.0 if b is None else np.abs(b)))
    if pre:
        close("pre", pred, z, ez + h * np.abs(z))
    y = ot.act(z, act)
    ey = 1.13 * ez + np.where(z < -3, 7e-6, 7e-7) * np.abs(y) * (act == "gelu") + 1e-37
    keep = ot.keep(M * N, p, SEED, OFFSET, 77).reshape(M, N)
    tol = keep * scale_of(p) * (ey + 2 * U * np.abs(y)) + U * (0 if res is None else np.abs(res)) + h * np.abs(ref)
    close("out", out, ref, tol * 1.01)
    if not backward:
        return
    g, gd = put(r.standard_normal((M, N)))
    zs, zd = put(z)
    d = afno.linear_backward(gd, xd, wd, pre=zd, activation=act, bias=bias, **call)
    torch.cuda.synchronize()
    dx, dw, db, dz = ot.linear_backward(g, x, w, zs, act, **want)
    slope = 3e-7 * np.abs(ot.drop(g, **want)) * (act == "gelu") + 2 * U * np.abs(dz)  # dz before its rounding
    hz = h if dtype == "bf16" and (act != "none" or p) else 0.0

    def product(a, c, ec, n):  # a c, c off by ec and rounded to hz of itself
        return k(n) * U * (np.abs(a) @ np.abs(c)) + np.abs(a) @ ec + 6 * hz * np.sqrt((a * a) @ (c * c))

    close("dx", d["dx"], dx, product(w, dz.T, slope.T, N).T + h * np.abs(dx) * 1.01)
    close("dw", d["dw"], dw, product(x.T, dz, slope, M) + h * np.abs(dw) * 1.01)
    if bias:
        close("db", d["db"], db, (k(M) * U * np.abs(dz) + slope).sum(0) + h * np.abs(db) * 1.01)
    else:
        assert d["db"] is None


def misplaced(a, dtype):
    """As store(), in memory that starts one element behind a 16-byte boundary."""
    v, t = store(a, dtype)
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.reshape(-1)
    o = flat[1:].reshape(t.shape)
    assert o.data_ptr() % 16 == t.element_size()
    return v, o


LINEAR = [
    # M, K, N, activation, p, bias, residual
    (1, 1, 1, "none", 0.0, True, True),
    (1, 8, 8, "gelu", 0.0, False, False),
    (1, 64, 256, "gelu", 0.1, True, False),          # a single token
    (2, 1024, 96, "none", 0.0, True, True),           # two tokens, one long sum
    (3, 7, 5, "relu", 0.5, True, True),
    (17, 33, 9, "gelu", 0.25, True, False),
    (31, 40, 24, "gelu", 0.1, False, True),
    (64, 64, 64, "none", 0.0, False, False),
    (65, 72, 136, "relu", 0.0, True, False),          # one row more than a tile
    (127, 129, 131, "gelu", 0.9, True, True),
    (300, 333, 77, "gelu", 0.1, True, False),
    (513, 264, 520, "gelu", 0.1, True, True),
    (1000, 96, 384, "gelu", 0.0, True, False),
    (2049, 512, 256, "none", 0.1, True, True),
    (5000, 256, 640, "gelu", 0.1, True, False),
    (8008, 200, 1032, "gelu", 0.1, True, True),       # many ragged tiles of 256, k behind the last whole stage
    (4104, 2056, 264, "relu", 0.25, True, False),     # few of them, split over k
    (8200, 40, 1024, "none", 0.0, False, True),       # less than one stage of k
    (4111, 333, 205, "gelu", 0.1, True, True),        # rows that are no 16-byte units, copied to some that are
    (2050, 1029, 516, "relu", 0.0, True, False),
    (10, 513, 4099, "gelu", 0.1, True, False),        # few rows
    (16, 1040, 520, "none", 0.0, True, True),
    (16500, 264, 1544, "gelu", 0.3, False, False),    # over the tiles of all CUs
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "{}x{}x{}_{}_p{}".format(*c[:5]))
def test_linear(case, dtype):
    M, K, N, act, p, bias, residual = case
    check_linear(M, K, N, dtype, act, p, bias, residual, seed=M)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("case", [(1, 64, 128, "gelu", 0.2), (130, 256, 264, "relu", 0.0), (600, 128, 512, "gelu", 0.1),
                                  (5000, 136, 264, "gelu", 0.1)])
def test_linear_at_odd_addresses(case, dtype):
    check_linear(*case[:3], dtype, case[3], case[4], residual=True, odd=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_without_rows(dtype):
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x, w = torch.empty(0, 12, dtype=dt, device="cuda"), torch.ones(12, 20, dtype=dt, device="cuda")
    assert afno.linear_forward(x, w).shape == (0, 20)
    d = afno.linear_backward(torch.empty(0, 20, dtype=dt, device="cuda"), x, w)
    torch.cuda.synchronize()
    assert d["dx"].shape == (0, 12) and not d["dw"].any() and not d["db"].any() and d["dw"].shape == (12, 20)
    d = afno.layer_norm_backward(x, x, w[:, 0].contiguous())
    torch.cuda.synchronize()
    assert not d["dgamma"].any() and not d["dbeta"].any()
    assert afno.layer_norm_forward(x, w[:, 0].contiguous(), w[:, 1].contiguous()).shape == (0, 12)
    assert afno.dropout_forward(x, 0.5, 1).shape == (0, 12)


@pytest.mark.parametrize("M,K,N", [(70, 64, 128), (300, 512, 256), (9, 40, 33)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_keeps_its_bounds_and_rows_apart(M, K, N, dtype):
    """Nothing is written beside out, pre and the gradients, and a NaN or infinity stays in its row."""
    r = np.random.default_rng(1)
    (_, x), (_, w), (_, g) = store(r.standard_normal((M, K)), dtype), store(r.standard_normal((K, N)), dtype), store(
        r.standard_normal((M, N)), dtype)

    def fenced(rows, cols):
        f = torch.full((rows * cols + 64,), 7.0, dtype=x.dtype, device="cuda")
        return f, f[32:32 + rows * cols].reshape(rows, cols)

    fo, out = fenced(M, N)
    fp, pre = fenced(M, N)
    afno.linear_forward(x, w, activation="gelu", out=out, pre=pre)
    for f in (fo, fp):
        assert (f[:32] == 7).all() and (f[-32:] == 7).all()
    x[M // 2, K // 3] = float("nan")
    x[0, 0] = float("inf")
    got = afno.linear_forward(x, w, activation="none")
    same = torch.ones(M, dtype=torch.bool)
    same[0] = same[M // 2] = False
    clean = afno.linear_forward(x[same.to("cuda")].contiguous(), w, activation="none")
    assert torch.isnan(got[M // 2]).all() and not torch.isfinite(got[0]).any()
    assert torch.isfinite(got[same.to("cuda")]).all() and torch.isfinite(clean).all()
    g[M // 2, 1] = float("nan")
    d = afno.linear_backward(g, torch.zeros_like(x), w, bias=True)
    torch.cuda.synchronize()
    assert torch.isnan(d["dx"][M // 2]).all() and torch.isfinite(d["dx"][same.to("cuda")][1:]).all()
    assert torch.isnan(d["db"][1]) and torch.isfinite(d["db"][2:]).all() and torch.isfinite(d["dw"][:, 2:]).all()


def test_linear_partial_gradients():
    r = np.random.default_rng(2)
    (_, x), (_, w), (_, g) = store(r.standard_normal((90, 64)), "bf16"), store(r.standard_normal((64, 72)), "bf16"), store(
        r.standard_normal((90, 72)), "bf16")
    full = afno.linear_backward(g, x, w)
    for kw in (dict(bias=False), dict(need_dx=False), dict(need_dw=False), dict(bias=False, need_dw=False)):
        d = afno.linear_backward(g, x, w, **kw)
        torch.cuda.synchronize()
        assert (d["db"] is None) == (kw.get("bias") is False) and (d["dx"] is None) == (kw.get("need_dx") is False)
        for n, v in d.items():
            assert v is None or torch.equal(v.view(torch.int16), full[n].view(torch.int16)), n


def test_gelu_slope_over_its_range():
    """GELU' read through a product with the unit matrix, over -20 .. 20 and at the infinities and NaN."""
    z = np.concatenate([np.linspace(-20, 20, 4000), [0.0, -0.0, np.inf, -np.inf, np.nan] + [0.0] * 91])
    zs, zd = store(z.reshape(64, 64), "fp32")
    ones, eye = torch.ones(64, 64, device="cuda"), torch.eye(64, device="cuda")
    # the unit matrix' zeros times a NaN would spread it over its row: it is checked by itself
    d = afno.linear_backward(torch.ones(64, 64, device="cuda"), ones, eye, pre=torch.nan_to_num(zd, 0.0, 40.0, -40.0),
                             activation="gelu", bias=False, need_dw=False)
    torch.cuda.synchronize()
    ref = ot.act_slope(np.nan_to_num(zs, nan=0.0, posinf=40.0, neginf=-40.0), "gelu")
    close("slope", d["dx"], ref, np.full(ref.shape, 3e-7))
    one = torch.ones(1, 1, device="cuda")
    for v, want in ((np.inf, 1.0), (-np.inf, 0.0), (np.nan, np.nan)):
        d = afno.linear_backward(one, one, one, pre=one * v, activation="gelu")
        np.testing.assert_equal(float(d["dx"]), want)


# ---------------------------------------------------------------- LayerNorm

NORM = [(1, 1), (1, 8), (3, 2), (7, 64), (130, 333), (65, 768), (33, 1024), (9, 2048), (1000, 96), (5, 2049), (70, 5000),
        (2, 8192), (4100, 24), (3, 9001), (1500, 3000)]


def norm_slack(v, rstd, C):
    """How far (v - mean) rstd may be off, relative to 1 + its size: v is exact, its mean off by k(C) u of the
    largest value, the variance likewise twice."""
    return 2 * k(C) * U * (1.0 + np.abs(v).max(-1, keepdims=True) * rstd)


def norm_dx_slack(a, hh, rstd, e):
    """How far dx may be off for a = |g gamma|, h = |(v - mean) rstd| and e of norm_slack: each of its terms by e
    of itself, and h by e (1 + h) wherever it stands."""
    m = lambda t: t.mean(-1, keepdims=True)  # noqa: E731
    return 2 * rstd * (e * (a + m(a) + hh * m(a * hh)) + e * (1 + hh) * m(a * hh) + hh * m(a * e * (1 + hh)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,C", NORM)
def test_layer_norm(M, C, residual, dtype):
    check_norm(M, C, residual, dtype, store)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,C", [(6, 64), (40, 1024), (3, 4096)])
def test_layer_norm_at_odd_addresses(M, C, dtype):
    check_norm(M, C, True, dtype, misplaced)


def check_norm(M, C, residual, dtype, put, mean=0.5):
    say(f"[norm] {M}x{C} {dtype} residual={residual}")
    r = np.random.default_rng(M + C)
    h, eps = HALF[dtype], 1e-6
    x, xd = put(mean + r.standard_normal((M, C)) * r.uniform(0.5, 2.0, C), dtype)
    res, resd = put(r.standard_normal((M, C)), dtype) if residual else (0.0, None)
    ga, gad = put(1 + 0.1 * r.standard_normal(C), dtype)
    be, bed = put(0.1 * r.standard_normal(C), dtype)
    s = torch.empty_like(xd)
    out = afno.layer_norm_forward(xd, gad, bed, residual=resd, sum_out=s, eps=eps)
    torch.cuda.synchronize()
    close("sum", s, x + res, h * np.abs(x + res) * 1.01)
    v = to_f64(s)  # the norm is of the stored sum
    assert residual or (v == x).all()
    rstd = 1 / np.sqrt(v.var(-1, keepdims=True) + eps)
    ref = ot.layer_norm(v, ga, be, eps)
    hh = np.abs((v - v.mean(-1, keepdims=True)) * rstd)
    e = norm_slack(v, rstd, C)
    close("out", out, ref, e * (1 + hh) * np.abs(ga) + 4 * U * (np.abs(be) + np.abs(ref)) + h * np.abs(ref) * 1.01)
    g, gd = put(r.standard_normal((M, C)), dtype)
    d = afno.layer_norm_backward(gd, s, gad, eps=eps, gsum=resd)
    torch.cuda.synchronize()
    dx, dga, dbe = ot.layer_norm_backward(g, v, ga, eps, res)
    a = np.abs(g * ga)
    close("dx", d["dx"], dx, norm_dx_slack(a, hh, rstd, e) + 2 * U * np.abs(res) + h * np.abs(dx) * 1.01)
    close("dgamma", d["dgamma"], dga, (np.abs(g) * e * (1 + hh) + k(M) * U * np.abs(g) * hh).sum(0))
    close("dbeta", d["dbeta"], dbe, k(M) * U * np.abs(g).sum(0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_layer_norm_of_very_wide_rows(dtype):
    check_norm(3, 2 ** 17 + 5, True, dtype, store)


def test_layer_norm_of_a_large_mean():
    """Rows whose mean is 4,096 times their spread: the squares are taken about the mean."""
    check_norm(50, 512, False, "fp32", store, mean=4096.0)


def test_layer_norm_of_equal_channels():
    """No variance: eps alone divides, and out is beta."""
    x = torch.full((5, 96), 3.0, device="cuda")
    be = torch.linspace(-1, 1, 96, device="cuda")
    assert torch.equal(afno.layer_norm_forward(x, torch.ones(96, device="cuda"), be), be.expand(5, 96))


# ---------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,p,residual", [(1, 0.5, True), (7, 0.3, False), (8, 0.5, True), (9, 0.1, True), (2048, 0.1, False),
                                          (2055, 0.9, True), (100003, 0.25, True), (1 << 20, 0.1, False), (4096, 0.0, True)])
def test_dropout(n, p, residual, dtype):
    say(f"[dropout] {n} p={p} {dtype}")
    r = np.random.default_rng(n)
    for put in (lambda a: store(a, dtype), lambda a: misplaced(a, dtype)):
        x, xd = put(r.standard_normal(n))
        res, resd = put(r.standard_normal(n)) if residual else (0.0, None)
        call = dict(offset=OFFSET, counter=torch.tensor([3], dtype=torch.int64, device="cuda"))
        out = afno.dropout_forward(xd, p, SEED, residual=resd, **call)
        back = afno.dropout_backward(xd, p, SEED, **call)
        torch.cuda.synchronize()
        dropped = ot.drop(x, p, SEED, OFFSET, 3)
        close("out", out, dropped + res, 2 * U * np.abs(dropped) + HALF[dtype] * np.abs(dropped + res) * 1.01)
        close("dx", back, dropped, (U + HALF[dtype] * 1.01) * np.abs(dropped))
        if p:
            assert (to_f64(back)[~ot.keep(n, p, SEED, OFFSET, 3)] == 0).all()


def test_dropout_drops_infinities_and_nan():
    x = torch.full((4096,), float("nan"), device="cuda")
    got = torch.isnan(afno.dropout_forward(x, 0.5, SEED)).cpu().numpy()
    assert (got == ot.keep(4096, 0.5, SEED)).all()


def test_dropout_numbers_beyond_32_bits():
    """seed, offset and counter are 64-bit numbers, and their sum wraps."""
    x = torch.ones(4096, device="cuda")
    c = torch.tensor([-1], dtype=torch.int64, device="cuda")  # 2^64 - 1
    for seed, offset in ((2 ** 64 - 1, 2 ** 64 - 1), (2 ** 63, 2 ** 40 + 1)):
        got = afno.dropout_forward(x, 0.5, seed, offset=offset, counter=c).cpu().numpy() > 0
        assert (got == ot.keep(4096, 0.5, seed, offset, 2 ** 64 - 1)).all()


def test_one_mask_everywhere():
    """The product's epilogue, its gradient and dropout of a tensor draw the same mask, whatever the type and tiling."""
    for M, N in ((1, 40), (70, 33), (640, 512)):
        want = ot.keep(M * N, 0.4, 11, 6).reshape(M, N)
        for dt in (torch.float32, torch.bfloat16):
            x, w, b = (torch.zeros(s, dtype=dt, device="cuda") for s in ((M, 16), (16, N), (N,)))
            out = afno.linear_forward(x, w, b + 1, p=0.4, seed=11, offset=6)
            alone = afno.dropout_forward(torch.ones(M, N, dtype=dt, device="cuda"), 0.4, 11, offset=6)
            db = afno.linear_backward(torch.ones(M, N, dtype=dt, device="cuda"), x, w, p=0.4, seed=11, offset=6)["db"]
            torch.cuda.synchronize()
            assert ((out > 0).cpu().numpy() == want).all() and torch.equal(out, alone)
            s = want.sum(0) * scale_of(0.4)
            assert (np.abs(to_f64(db) - s) <= (2.0 ** -8 if dt == torch.bfloat16 else k(M) * U) * s * 1.01).all()


# ---------------------------------------------------------------- beyond 32 bits

def test_offsets_beyond_32_bits():
    """Tensors of over 2^31 values, checked in their last rows (the first are those of any other test)."""
    bf = torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    n = 2 ** 31 + 12345
    x = torch.empty(n, dtype=bf, device="cuda")
    x.fill_(1.0)
    x[-4096:] = torch.randn(4096, generator=gen, device="cuda").to(bf)
    tail = afno.dropout_forward(x, 0.3, SEED, offset=OFFSET)[-4096:]
    want = np.where(keep_from(n - 4096, 4096, 0.3), to_f64(x[-4096:]) * scale_of(0.3), 0.0)
    close("dropout", tail, want, 2.0 ** -8 * 1.01 * np.abs(want))
    del x
    M, K, N = 1_050_000, 16, 2056
    x = torch.randn(M, K, generator=gen, device="cuda").to(bf)
    w = torch.randn(K, N, generator=gen, device="cuda").to(bf)
    out = afno.linear_forward(x, w)
    ref = to_f64(x[-300:]) @ to_f64(w)
    close("linear", out[-300:], ref, k(K) * U * (np.abs(to_f64(x[-300:])) @ np.abs(to_f64(w))) + 2.0 ** -8 * np.abs(ref) * 1.01)
    d = afno.linear_backward(out, x, w, need_dw=False, bias=False)
    g = to_f64(out[-300:])
    close("dx", d["dx"][-300:], g @ to_f64(w).T, k(N) * U * (np.abs(g) @ np.abs(to_f64(w)).T) + 2.0 ** -8 * np.abs(g @ to_f64(w).T) * 1.01)
    ga, be = torch.ones(N, dtype=bf, device="cuda"), torch.zeros(N, dtype=bf, device="cuda")
    y = afno.layer_norm_forward(out, ga, be)
    ref = ot.layer_norm(g, 1.0, 0.0, 1e-6)
    rstd = 1 / g.std(-1, keepdims=True)
    close("norm", y[-300:], ref, norm_slack(g, rstd, N) * (1 + np.abs(ref)) + 2.0 ** -8 * np.abs(ref) * 1.01)
    del y
    up = torch.zeros_like(out)
    up[-300:] = torch.randn(300, N, generator=gen, device="cuda").to(bf)
    dx = afno.layer_norm_backward(up, out, ga)["dx"]
    u64 = to_f64(up[-300:])
    ref = ot.layer_norm_backward(u64, g, 1.0, 1e-6)[0]
    hh = np.abs(ot.layer_norm(g, 1.0, 0.0, 1e-6))
    close("norm dx", dx[-300:], ref, norm_dx_slack(np.abs(u64), hh, rstd, norm_slack(g, rstd, N)) + 2.0 ** -8 * np.abs(ref) * 1.01)


def keep_from(first, n, p):
    """ot.keep of the n elements from `first` on."""
    i = np.arange(first // 8, (first + n) // 8 + 1, dtype=np.uint64)
    full = lambda v: np.full(i.shape, v, dtype=np.uint64)  # noqa: E731
    words = ot.philox4x32((i & ot.LOW, i >> ot.HALF, full(OFFSET & 0xFFFFFFFF), full(OFFSET >> 32)),
                          (SEED & 0xFFFFFFFF, SEED >> 32), 7)
    numbers = np.stack([v for w in words for v in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    return numbers.reshape(-1)[first % 8:first % 8 + n] >= ot.threshold(p)


# ---------------------------------------------------------------- together, streams, graphs

def mlp_step(v, p, r, gout, buf, stream=None):
    """The channel MLP half of a block in training: u + x -> LN -> C x 4C, GELU, drop -> 4C x C, drop, residual;
    and its gradients for gout."""
    C, H4 = v["x"].shape[-1], p["wa"].shape[1]
    afno.layer_norm_forward(v["u"], p["g"], p["b"], residual=v["x"], out=buf["w"], sum_out=buf["v"], stream=stream)
    afno.linear_forward(buf["w"], p["wa"], p["ba"], activation="gelu", out=buf["h"], pre=buf["pre"], **r[0], stream=stream)
    out = afno.linear_forward(buf["h"], p["wb"], p["bb"], residual=buf["v"], out=buf["out"], **r[1], stream=stream)
    d2 = afno.linear_backward(gout, buf["h"], p["wb"], **r[1], stream=stream)
    d1 = afno.linear_backward(d2["dx"], buf["w"], p["wa"], pre=buf["pre"], activation="gelu", **r[0], stream=stream)
    d0 = afno.layer_norm_backward(d1["dx"], buf["v"], p["g"], gsum=gout, stream=stream)
    return [out, d0["dx"], d0["dgamma"], d0["dbeta"], d1["dw"], d1["db"], d2["dw"], d2["db"]]


def mlp_setup(M, C, dtype, seed=0):
    r = np.random.default_rng(seed)
    n = lambda s, sd=1.0, mean=0.0: store(mean + sd * r.standard_normal(s), dtype)  # noqa: E731
    v = {"x": n((M, C)), "u": n((M, C))}
    p = {"g": n(C, 0.1, 1.0), "b": n(C, 0.1), "wa": n((C, 4 * C), C ** -0.5), "ba": n(4 * C, 0.1),
         "wb": n((4 * C, C), (4 * C) ** -0.5), "bb": n(C, 0.1)}
    g = n((M, C))
    buf = {k_: torch.empty(M, c, dtype=g[1].dtype, device="cuda") for k_, c in
           (("v", C), ("w", C), ("pre", 4 * C), ("h", 4 * C), ("out", C))}
    return v, p, g, buf


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-5), ("bf16", 2e-2)])
@pytest.mark.parametrize("M,C", [(60, 64), (500, 256)])
def test_channel_mlp_in_training(M, C, dtype, tol):
    """All operators together against the float64 chain, by the relative 2-norm: fp32 k(4 C) u at most and bf16
    five roundings of 2^-8 in a row."""
    v, p, g, buf = mlp_setup(M, C, dtype)
    step = torch.tensor([41], dtype=torch.int64, device="cuda")
    r = [dict(p=0.1, seed=SEED, offset=i << 40, counter=step) for i in (1, 2)]
    o = [dict(p=0.1, seed=SEED, offset=i << 40, counter=41) for i in (1, 2)]
    dev = lambda d: {k_: t[1] for k_, t in d.items()}  # noqa: E731
    got = mlp_step(dev(v), dev(p), r, g[1], buf)
    torch.cuda.synchronize()
    w = {k_: t[0] for k_, t in {**v, **p}.items()}
    s = w["x"] + w["u"]
    n = ot.layer_norm(s, w["g"], w["b"], 1e-6)
    h, pre = ot.linear(n, w["wa"], w["ba"], "gelu", **o[0])
    out, _ = ot.linear(h, w["wb"], w["bb"], residual=s, **o[1])
    dh, dwb, dbb, _ = ot.linear_backward(g[0], h, w["wb"], **o[1])
    dn, dwa, dba, _ = ot.linear_backward(dh, n, w["wa"], pre, "gelu", **o[0])
    dv, dga, dbe = ot.layer_norm_backward(dn, s, w["g"], 1e-6, g[0])
    for name, a, b in zip(("out", "dv", "dgamma", "dbeta", "dwa", "dba", "dwb", "dbb"), got,
                          (out, dv, dga, dbe, dwa, dba, dwb, dbb)):
        e = np.linalg.norm(to_f64(a) - b) / np.linalg.norm(b)
        say(f"  {name} {e:.2e}")
        assert e <= tol, name


def test_block_from_its_operators():
    """LayerNorm, the filter, LayerNorm and the two products give what the block's oracle gives."""
    wl = synth.Workload("block", 2, 12, 20, 128, 4, "bf16", 0.01, 1.0)
    x_st, p_st = synth.make_x(wl, seed=6), synth.make_block_params(wl, seed=6, mlp_std=0.05)
    x, p = to_dev(x_st, "bf16"), {k_: to_dev(v, "bf16") for k_, v in p_st.items()}
    t = afno.layer_norm_forward(x, p["ln1_g"], p["ln1_b"])
    u = afno.filter_forward(t, p["w1"], p["b1"], p["w2"], p["b2"], 4, 0.01, 1.0)
    v = torch.empty_like(x)
    w = afno.layer_norm_forward(u, p["ln2_g"], p["ln2_b"], residual=x, sum_out=v)
    out = afno.linear_forward(afno.linear_forward(w, p["wa"], p["ba"], activation="gelu"), p["wb"], p["bb"], residual=v)
    torch.cuda.synchronize()
    wide = {k_: synth.widen(a, "bf16") for k_, a in p_st.items()}
    ref = oblock.block_forward(synth.widen(x_st, "bf16"), *(wide[k_] for k_ in afno.BLOCK_PARAMS), 4, 0.01, 1.0)
    assert np.max(np.abs(to_f64(out) - ref)) <= 2e-2 * np.max(np.abs(ref))


def bits(ts):
    return [t.view(torch.int16 if t.element_size() == 2 else torch.int32).clone() for t in ts]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_repeated_calls_other_streams_and_graphs(dtype):
    """The same bits again, on another stream, and from a graph replayed between eager calls; the counter
    on the device draws another mask in a replay."""
    v, p, g, buf = mlp_setup(300, 64, dtype, seed=5)
    dev = lambda d: {k_: t[1] for k_, t in d.items()}  # noqa: E731
    v, p, g = dev(v), dev(p), g[1]
    step = torch.tensor([1], dtype=torch.int64, device="cuda")
    r = [dict(p=0.2, seed=SEED, offset=i << 40, counter=step) for i in (1, 2)]
    eager = {}
    for s in (1, 2, 3):
        step.fill_(s)
        eager[s] = bits(mlp_step(v, p, r, g, buf))
    step.fill_(2)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = mlp_step(v, p, r, g, buf, stream=other)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bits(got), eager[2]))
    assert not torch.equal(eager[1][0], eager[2][0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = mlp_step(v, p, r, g, buf)
    for s in (3, 1, 2, 1):
        step.fill_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits(held), eager[s])), s
        mlp_step(v, p, r, g, {k_: torch.empty_like(t) for k_, t in buf.items()})
        torch.cuda.synchronize()


def test_two_threads():
    """Two host threads at once, each on its own stream, give what they give one after the other."""
    import threading
    sets = []
    for i in range(2):
        v, p, g, buf = mlp_setup(200 + 50 * i, 64, "bf16", seed=i)
        dev = lambda d: {k_: t[1] for k_, t in d.items()}  # noqa: E731
        r = [dict(p=0.1, seed=i, offset=j) for j in (1, 2)]
        sets.append([dev(v), dev(p), r, g[1], buf])
    want = [bits(mlp_step(*s)) for s in sets]
    torch.cuda.synchronize()
    ok = [False, False]

    def work(i):
        st = torch.cuda.Stream()
        for _ in range(20):
            got = mlp_step(*sets[i], stream=st)
            st.synchronize()
            with torch.cuda.stream(st):
                same = all(torch.equal(a, b) for a, b in zip(bits(got), want[i]))
            if not same:
                return
        ok[i] = True

    ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert ok == [True, True]


def test_workspaces_through_the_c_abi():
    """The library's own workspace (NULL), one with exactly the bytes it asks for between fences, and the refusal to
    allocate for a captured call."""
    M, K, N = 130, 512, 96
    r = np.random.default_rng(0)
    (_, x), (_, w), (_, g) = (store(r.standard_normal(s), "bf16") for s in ((M, K), (K, N), (M, N)))
    want = afno.linear_backward(g, x, w, p=0.1, seed=3)
    need = afno.afno_linear_backward_workspace(M, K, N, afno.AFNO_DTYPE_BF16, 1)
    outs = [torch.empty_like(t) for t in (want["dx"], want["dw"], want["db"])]
    st = torch.cuda.current_stream().cuda_stream

    def call(ws, have, handle=st):
        return afno.afno_linear_backward(g.data_ptr(), x.data_ptr(), w.data_ptr(), None, M, K, N, 0, 0.1, 3, 0, None,
                                         afno.AFNO_DTYPE_BF16, *(o.data_ptr() for o in outs), ws, have, handle)

    fenced = torch.full((need + 512,), 9, dtype=torch.uint8, device="cuda")
    for ws, have in ((None, 0), (fenced.data_ptr() + 256, need)):
        [o.zero_() for o in outs]
        assert call(ws, have) == afno.AFNO_OK
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits(outs), bits(want.values())))
    assert (fenced[:256] == 9).all() and (fenced[-256:] == 9).all()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        x.add_(0)
        assert call(None, 0, s.cuda_stream) == afno.AFNO_ERR_UNSUPPORTED
    assert "captured" in afno.afno_last_error()

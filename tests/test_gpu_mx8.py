"""The operators in eight bits and the root-mean-square norm on the GPU against the float64 oracle (oracle/mx8.py,
oracle/train.py) on the same stored inputs, elementwise.

Bounds as in test_gpu_train.py: u = 2^-24, h one rounding of the storage type, k(n) u for sums of n terms.  The mean of C
squares, all positive, is off by k(C) u of itself, and the norm's factor by half of that and a few u: e = k(C) u bounds
every factor of it.  A result in eight bits whose value before is off by t is off by t and one rounding, half a step
of E4M3 at its size under its block's scale (om.half_step).

Products in bf16 run on the eight-bit instruction, which drops of eight neighbouring k's products what lies below 2^-13
of the largest's power of two: at most 2^-13 of the largest from each of the seven others, toward zero, by signs that
are as random as the products'.  Its square over a group is at most 7 (2^-13)^2 / 3 of the largest's square on average (the
part dropped is anything from none to all), the largest's square at most the sum of the group's: 6 standard deviations
are 6 sqrt(7 / 3) 2^-13 = 9.2 2^-13 of the root of the sum of all squared products (and no less than 7 2^-13 of a single
group's largest, which nothing exceeds)."""
import numpy as np
import pytest

import paper_2208_05419_amd as afno
import test_gpu_train as tg
from gpu_util import say, to_f64
from oracle import mx8 as om
from oracle import train as ot
from test_gpu_train import HALF, OFFSET, SEED, U, close, k, misplaced, scale_of, store

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    afno.load_library()


def raw(t):
    """Codes and scale bytes of an Mx8, as rows."""
    q = t.values.view(torch.uint8).cpu().numpy()
    s = t.scales.view(torch.uint8).cpu().numpy()
    return q.reshape(-1, q.shape[-1]), s.reshape(-1, s.shape[-1])


def value8(t):
    """What an Mx8 stands for (float64), its zeros behind the channels and its scales' range checked."""
    q, s = raw(t)
    assert not q[:, t.channels:].any() and (s >= 10).all() and (s <= 246).all()
    return om.unpack(q, s, t.channels)


def packed(a):
    """Rows of float64 numbers in eight bits, by the oracle: their values and the Mx8 on the GPU."""
    q, s = om.pack(a)
    t = afno.Mx8(torch.from_numpy(q).cuda().view(torch.float8_e4m3fn), torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu),
                 a.shape[1])
    return om.unpack(q, s, a.shape[1]), t


def close8(name, got, ref, tol):
    close(name, value8(got), ref, tol + 1.0001 * om.half_step(np.abs(ref) + tol))
    top, low = om.pack(np.abs(ref) + tol)[1], om.pack(np.maximum(np.abs(ref) - tol, 0.0))[1]
    s = raw(got)[1]
    assert (s <= top).all() and (s >= low).all(), name


# ---------------------------------------------------------------- to eight bits and back

SHAPES = [(1, 1), (1, 7), (3, 8), (2, 31), (5, 32), (4, 33), (7, 64), (130, 333), (65, 768), (33, 1024), (1000, 96), (3, 9001), (4100, 24)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,C", SHAPES)
def test_pack(M, C, dtype):
    """The oracle's bits, and the values that they stand for in both types, from and to any address."""
    say(f"[pack] {M}x{C} {dtype}")
    r = np.random.default_rng(M + C)
    for put in (store, misplaced):
        x, xd = put(r.standard_normal((M, C)) * 2.0 ** r.integers(-30, 30, (M, 1)), dtype)
        q, s = om.pack(x)
        t = afno.mx8_pack(xd)
        got = raw(t)
        assert (got[0] == q).all() and (got[1] == s).all()
        want = om.unpack(q, s, C)
        for dt in (torch.float32, torch.bfloat16):
            assert (to_f64(afno.mx8_unpack(t, dtype=dt)) == want).all()
            flat = torch.full((M * C + 65,), 7.0, dtype=dt, device="cuda")
            out = flat[33:33 + M * C].reshape(M, C)  # odd addresses, fenced
            assert afno.mx8_unpack(t, out=out) is out and (to_f64(out) == want).all()
            assert (flat[:33] == 7).all() and (flat[33 + M * C:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_pack_of_every_kind_of_value(dtype):
    """Zeros, ties, the smallest and largest numbers, blocks over all scales, NaN and infinities."""
    mid = (om.CODES[:-1] + om.CODES[1:]) / 2
    rows = [np.zeros(64), -np.zeros(64), np.resize(mid, 64), np.resize(np.append(448.0, om.CODES), 64)]
    rows += [np.resize([1.0, 0.3, -0.7, 1.75, 1.7500001, 2.0 ** -9], 64) * 2.0 ** e for e in range(-126, 127, 9)]
    rows += [np.resize([v, -v / 3, 1.0], 64) for v in (3.3e38, 2.0 ** 127 * 1.9, 448 * 2.0 ** 119, 2.0 ** -149, 2.0 ** -126, 1e-36)]
    rows += [np.resize([np.nan, 5.0, -5.0], 64), np.resize([np.inf, 0.1, -np.inf], 64), np.full(64, np.inf), np.full(64, np.nan)]
    rows[2][0] = 448.0
    x, xd = store(np.array(rows), dtype)
    q, s = om.pack(x)
    got = raw(afno.mx8_pack(xd))
    nan = np.isnan(x) | np.isinf(x)
    assert (got[1] == s).all()
    assert ((got[0] == q) | (nan & (got[0] & 127 == 127))).all()
    t = afno.mx8_pack(xd)
    want = om.unpack(q, s, 64)
    for dt in (torch.float32, torch.bfloat16):
        np.testing.assert_array_equal(to_f64(afno.mx8_unpack(t, dtype=dt)), want)
    assert np.isfinite(want[~nan]).all()


def test_unpack_of_every_code():
    """All 256 codes under every scale that the format has."""
    q = np.tile(np.arange(256, dtype=np.uint8), (237, 1))
    s = np.repeat(np.arange(10, 247, dtype=np.uint8)[:, None], 8, 1)
    t = afno.Mx8(torch.from_numpy(q).cuda().view(torch.float8_e4m3fn), torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu), 256)
    want = om.unpack(q, s, 256)
    for dt in (torch.float32, torch.bfloat16):
        np.testing.assert_array_equal(to_f64(afno.mx8_unpack(t, dtype=dt)), want)


# ---------------------------------------------------------------- the norm

NORM = [(1, 1), (1, 8), (3, 2), (7, 64), (130, 333), (65, 768), (33, 1024), (9, 2048), (1000, 96), (5, 2049), (70, 5000), (2, 8192),
        (4100, 24), (3, 9001), (1500, 3000), (2, 8190)]


def check_norm(M, C, residual, dtype, put, scale=1.0):
    say(f"[rms] {M}x{C} {dtype} residual={residual}")
    r = np.random.default_rng(M + C)
    h, eps = HALF[dtype], 1e-6
    x, xd = put(scale * (0.5 + r.standard_normal((M, C)) * r.uniform(0.5, 2.0, C)), dtype)
    res, resd = put(scale * r.standard_normal((M, C)), dtype) if residual else (0.0, None)
    ga, gad = put(1 + 0.1 * r.standard_normal(C), dtype)
    s, out8 = torch.empty_like(xd), afno.mx8_empty((M, C), "cuda")
    out = torch.empty_like(xd)
    assert afno.rms_norm_forward(xd, gad, residual=resd, sum_out=s, out=out, out8=out8, eps=eps) is out
    torch.cuda.synchronize()
    close("sum", s, x + res, h * np.abs(x + res) * 1.01)
    v = to_f64(s)  # the norm is of the stored sum
    assert residual or (v == x).all()
    ref, e = om.rms_norm(v, ga, eps), k(C) * U
    close("out", out, ref, (e + h * 1.01) * np.abs(ref))
    close8("out8", out8, ref, e * np.abs(ref))
    # each output by itself, the same bits
    alone = afno.mx8_empty((M, C), "cuda")
    assert afno.rms_norm_forward(xd, gad, residual=resd, out8=alone, eps=eps) is alone
    assert all((a == b).all() for a, b in zip(raw(alone), raw(out8)))
    assert torch.equal(afno.rms_norm_forward(xd, gad, residual=resd, eps=eps), out)
    g, gd = put(r.standard_normal((M, C)), dtype)
    d = afno.rms_norm_backward(gd, s, gad, eps=eps, gsum=resd)
    torch.cuda.synchronize()
    dx, dga = om.rms_norm_backward(g, v, ga, eps, res)
    rms = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    a, hh = np.abs(g * ga), np.abs(v * rms)
    # a by u, h and the factor by e each, the mean by e and its terms by e + u
    close("dx", d["dx"], dx, rms * (2 * e * a + 5 * e * hh * (a * hh).mean(-1, keepdims=True)) + 2 * U * np.abs(res) + h * np.abs(dx) * 1.01)
    close("dgamma", d["dgamma"], dga, (np.abs(g) * hh * (e + k(M) * U)).sum(0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,C", NORM)
def test_rms_norm(M, C, residual, dtype):
    check_norm(M, C, residual, dtype, store)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,C", [(6, 64), (40, 1024), (3, 4096)])
def test_rms_norm_at_odd_addresses(M, C, dtype):
    check_norm(M, C, True, dtype, misplaced)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rms_norm_of_very_wide_and_very_large_rows(dtype):
    check_norm(3, 2 ** 17 + 5, True, dtype, store)
    check_norm(3, 2 ** 20, True, dtype, store)
    check_norm(20, 200, False, dtype, store, scale=1e12)
    check_norm(20, 200, False, dtype, store, scale=1e-9)  # eps alone divides


def test_rms_norm_of_zeros_infinities_and_nan():
    """A row of zeros gives zeros and passes the residual's gradient on; what is not finite stays in its row."""
    x = torch.randn(6, 96, device="cuda")
    x[1], x[3, 5], x[4, 7] = 0.0, float("nan"), float("inf")
    ga, g = torch.ones(96, device="cuda"), torch.randn(6, 96, device="cuda")
    out8 = afno.mx8_empty((6, 96), "cuda")
    out = torch.empty_like(x)
    afno.rms_norm_forward(x, ga, out=out, out8=out8)
    keep = [0, 1, 2, 5]
    y8 = om.unpack(*raw(out8), 96)
    assert not out[1].any() and not y8[1].any()
    assert torch.isnan(out[3]).all() and np.isnan(y8[3]).all() and torch.isnan(out[4, 7]) and np.isnan(y8[4, 7])
    assert torch.isfinite(out[keep]).all() and np.isfinite(y8[keep]).all()
    d = afno.rms_norm_backward(g, x, ga, gsum=g)
    assert torch.isfinite(d["dx"][keep]).all()
    assert torch.allclose(d["dx"][1], g[1] * 1e3 + g[1], rtol=1e-5)  # rms of zeros: 1 / sqrt(eps)


# ---------------------------------------------------------------- products

def dropped(x, w, dtype):
    """What the eight-bit instruction may drop of x w."""
    return 9.2 * 2.0 ** -13 * np.sqrt((x * x) @ (w * w)) if dtype == "bf16" else 0.0


def check_linear(M, K, N, dtype, act, p=0.0, bias=True, residual=False, backward=True, odd=False, seed=0):
    say(f"[mx8 linear] {M}x{K}x{N} {dtype} {act} p={p} bias={bias} residual={residual} odd={odd}")
    r = np.random.default_rng(seed)
    put = (lambda a: misplaced(a, dtype)) if odd else (lambda a: store(a, dtype))
    x, xd = packed(r.standard_normal((M, K)) * r.uniform(0.3, 3.0, K))
    wt, wd = packed(r.standard_normal((N, K)) / np.sqrt(K))
    w = wt.T
    b, bd = put(r.standard_normal(N)) if bias else (None, None)
    res, resd = put(r.standard_normal((M, N))) if residual else (None, None)
    call, want = tg.rng_args(p, 77)
    ref, z = ot.linear(x, w, b, act, res, **want)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    out8, pre8 = (afno.mx8_empty((M, N), "cuda") for _ in range(2))
    if odd:
        flat = torch.full((M * N + 65,), 7.0, dtype=dt, device="cuda")
        out = flat[33:33 + M * N].reshape(M, N)
    else:
        out = torch.empty(M, N, dtype=dt, device="cuda")
    kw = dict(activation=act, residual=resd, dtype=dt, **call)
    assert afno.mx8_linear_forward(xd, wd, bd, out=out, out8=out8, pre8=pre8, **kw) is out
    torch.cuda.synchronize()
    if odd:
        assert (flat[:33] == 7).all() and (flat[33 + M * N:] == 7).all()
    h = HALF[dtype]
    ez = k(K) * U * (np.abs(x) @ np.abs(w) + (0.0 if b is None else np.abs(b))) + dropped(x, w, dtype)
    close8("pre8", pre8, z, ez)
    y = ot.act(z, act)
    # GELU: within 7e-7 of its size (7e-6 below -3); the short one of bf16 within 1.3e-5, and 1.2e-18 below -9
    fit = 1.3e-5 * np.abs(y) + 1.2e-18 if dtype == "bf16" else np.where(z < -3, 7e-6, 7e-7) * np.abs(y)
    ey = 1.13 * ez + fit * (act == "gelu") + 1e-37
    keep = ot.keep(M * N, p, SEED, OFFSET, 77).reshape(M, N)
    tol = keep * scale_of(p) * (ey + 2 * U * np.abs(y)) + U * (0 if res is None else np.abs(res)) + U * np.abs(ref)
    close("out", out, ref, (tol + h * np.abs(ref)) * 1.01)
    close8("out8", out8, ref, tol * 1.01)
    # each output by itself, the same bits
    alone = afno.mx8_empty((M, N), "cuda")
    assert afno.mx8_linear_forward(xd, wd, bd, out8=alone, **kw) is alone
    assert all((a == b_).all() for a, b_ in zip(raw(alone), raw(out8)))
    assert torch.equal(afno.mx8_linear_forward(xd, wd, bd, **kw), out)
    if not backward:
        return
    g, gd = put(r.standard_normal((M, N)))
    w, wd = put(r.standard_normal((K, N)) / np.sqrt(K))
    zs = value8(pre8)
    d = afno.mx8_linear_backward(gd, xd, wd, pre8=pre8, activation=act, bias=bias, **call)
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
    # the gradient of what the eight bits stand for, through the operators that read the storage type: the same bits
    e = afno.linear_backward(gd, afno.mx8_unpack(xd, dtype=dt), wd, pre=afno.mx8_unpack(pre8, dtype=dt), activation=act,
                             bias=bias, **call)
    for n in ("dx", "db"):
        assert d[n] is None or torch.equal(d[n], e[n]), n


LINEAR = [
    # M, K, N, activation, p, bias, residual
    (1, 1, 1, "none", 0.0, True, True),
    (1, 8, 8, "gelu", 0.0, False, False),
    (1, 64, 256, "gelu", 0.1, True, False),          # a single token
    (1, 4096, 1024, "none", 0.0, True, True),
    (2, 1024, 96, "none", 0.0, True, True),
    (3, 7, 5, "relu", 0.5, True, True),
    (5, 160, 40, "gelu", 0.1, True, False),
    (8, 1000, 129, "gelu", 0.0, True, True),
    (16, 1056, 520, "none", 0.0, True, True),
    (17, 33, 9, "gelu", 0.25, True, False),
    (31, 40, 24, "gelu", 0.1, False, True),
    (64, 64, 64, "none", 0.0, False, False),
    (65, 72, 136, "relu", 0.0, True, False),          # one row more than a tile
    (64, 3000, 70, "gelu", 0.0, True, True),          # few tiles of a long sum
    (127, 129, 131, "gelu", 0.9, True, True),
    (300, 333, 77, "gelu", 0.1, True, False),
    (513, 264, 520, "gelu", 0.1, True, True),
    (1000, 96, 384, "gelu", 0.0, True, False),
    (2049, 512, 256, "none", 0.1, True, True),
    (5000, 256, 640, "gelu", 0.1, True, False),
    (8008, 200, 1032, "gelu", 0.1, True, True),       # many ragged tiles, k behind the last whole stage
    (4104, 2056, 264, "relu", 0.25, True, False),
    (8200, 40, 1024, "none", 0.0, False, True),       # less than one stage of k
    (4111, 333, 205, "gelu", 0.1, True, True),
    (16500, 264, 1544, "gelu", 0.3, False, False),
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
def test_without_rows(dtype):
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    x, ga = torch.empty(0, 12, dtype=dt, device="cuda"), torch.ones(12, dtype=dt, device="cuda")
    t = afno.mx8_pack(x)
    assert t.shape == (0, 12) and t.values.shape == (0, 32) and t.scales.shape == (0, 1)
    assert afno.mx8_unpack(t).shape == (0, 12) and afno.rms_norm_forward(x, ga).shape == (0, 12)
    assert not afno.rms_norm_backward(x, x, ga)["dgamma"].any()
    w = afno.mx8_pack(torch.ones(20, 12, dtype=dt, device="cuda"))
    assert afno.mx8_linear_forward(t, w).shape == (0, 20)
    d = afno.mx8_linear_backward(torch.empty(0, 20, dtype=dt, device="cuda"), t, torch.ones(12, 20, dtype=dt, device="cuda"))
    torch.cuda.synchronize()
    assert d["dx"].shape == (0, 12) and d["dw"].shape == (12, 20) and not d["dw"].any() and not d["db"].any()


@pytest.mark.parametrize("M,K,N", [(70, 64, 128), (300, 512, 256), (9, 40, 33), (1, 100, 65), (1000, 130, 300)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_keeps_its_bounds_and_rows_apart(M, K, N, dtype):
    """Nothing is written beside the outputs, and a NaN stays in its row of the product, forward and backward."""
    r = np.random.default_rng(1)
    x, xd = packed(r.standard_normal((M, K)))
    _, wd = packed(r.standard_normal((N, K)))
    blocks = -(-N // 32)
    fences = []

    def fenced(cols, dt):
        f = torch.full((M * cols + 64,), 7, dtype=torch.uint8, device="cuda")
        fences.append(f)
        return f[32:32 + M * cols].view(dt).reshape(M, cols)

    out8, pre8 = (afno.Mx8(fenced(32 * blocks, torch.float8_e4m3fn), fenced(blocks, torch.float8_e8m0fnu), N) for _ in range(2))
    kw = dict(activation="gelu", dtype=torch.float32 if dtype == "fp32" else torch.bfloat16)
    clean = afno.mx8_linear_forward(xd, wd, **kw)
    afno.mx8_linear_forward(xd, wd, out8=out8, pre8=pre8, **kw)
    assert all((f[:32] == 7).all() and (f[-32:] == 7).all() for f in fences)
    x[M // 2, K // 3] = np.nan
    _, xd = packed(x)
    got = afno.mx8_linear_forward(xd, wd, **kw)
    out8 = afno.mx8_linear_forward(xd, wd, out8=out8, **kw)
    rest = torch.arange(M, device="cuda") != M // 2
    assert torch.isnan(got[M // 2]).all() and torch.equal(got[rest], clean[rest])
    y8 = om.unpack(*raw(out8), N)
    assert np.isnan(y8[M // 2]).all() and np.isfinite(y8[rest.cpu().numpy()]).all()
    w = torch.randn(K, N, device="cuda").to(clean.dtype)
    d = afno.mx8_linear_backward(clean, xd, w)
    torch.cuda.synchronize()
    assert torch.isnan(d["dw"][K // 3]).all() and torch.isfinite(d["dx"]).all()
    assert torch.isfinite(d["dw"][torch.arange(K, device="cuda") != K // 3]).all()


def test_linear_over_all_scales():
    """Rows and weights whose blocks have very different scales, and products of far powers of two."""
    r = np.random.default_rng(3)
    x = r.standard_normal((200, 256)) * 2.0 ** np.repeat(r.integers(-40, 40, (200, 8)), 32, -1)
    x, xd = packed(x)
    w, wd = packed(r.standard_normal((96, 256)) * 2.0 ** np.repeat(r.integers(-40, 40, (96, 8)), 32, -1))
    mags = np.abs(x) @ np.abs(w).T
    out = afno.mx8_linear_forward(xd, wd, dtype=torch.float32)
    close("out", out, x @ w.T, k(256) * U * mags)
    out = afno.mx8_linear_forward(xd, wd)
    close("out", out, x @ w.T, k(256) * U * mags + dropped(x, w.T, "bf16") + HALF["bf16"] * 1.01 * np.abs(x @ w.T))


def test_partial_gradients():
    r = np.random.default_rng(2)
    (_, x), (_, pre) = packed(r.standard_normal((90, 64))), packed(r.standard_normal((90, 72)))
    (_, w), (_, g) = store(r.standard_normal((64, 72)), "bf16"), store(r.standard_normal((90, 72)), "bf16")
    call = dict(pre8=pre, activation="gelu")
    full = afno.mx8_linear_backward(g, x, w, **call)
    for kw in (dict(bias=False), dict(need_dx=False), dict(need_dw=False), dict(bias=False, need_dw=False)):
        d = afno.mx8_linear_backward(g, x, w, **call, **kw)
        torch.cuda.synchronize()
        assert (d["db"] is None) == (kw.get("bias") is False) and (d["dx"] is None) == (kw.get("need_dx") is False)
        for n, v in d.items():
            assert v is None or torch.equal(v, full[n]), n


# ---------------------------------------------------------------- together, streams, graphs

def mlp_step(v, p, r, gout, buf, stream=None):
    """The channel MLP half of a block in training with everything kept in eight bits: u + x -> norm -> C x 4C, GELU,
    drop -> 4C x C, drop, residual; and its gradients for gout."""
    kw = dict(stream=stream)
    w8a, w8b = afno.mx8_pack(p["wat"], out=buf["w8a"], **kw), afno.mx8_pack(p["wbt"], out=buf["w8b"], **kw)
    afno.rms_norm_forward(v["u"], p["g"], residual=v["x"], sum_out=buf["v"], out8=buf["n"], **kw)
    afno.mx8_linear_forward(buf["n"], w8a, p["ba"], activation="gelu", out8=buf["h"], pre8=buf["pre"], **r[0], **kw)
    out = afno.mx8_linear_forward(buf["h"], w8b, p["bb"], residual=buf["v"], out=buf["out"], **r[1], **kw)
    d2 = afno.mx8_linear_backward(gout, buf["h"], p["wb"], **r[1], **kw)
    d1 = afno.mx8_linear_backward(d2["dx"], buf["n"], p["wa"], pre8=buf["pre"], activation="gelu", **r[0], **kw)
    d0 = afno.rms_norm_backward(d1["dx"], buf["v"], p["g"], gsum=gout, **kw)
    return [out, d0["dx"], d0["dgamma"], d1["dw"], d1["db"], d2["dw"], d2["db"]]


def mlp_setup(M, C, dtype, seed=0):
    r = np.random.default_rng(seed)
    n = lambda s, sd=1.0, mean=0.0: store(mean + sd * r.standard_normal(s), dtype)  # noqa: E731
    v = {"x": n((M, C)), "u": n((M, C))}
    p = {"g": n(C, 0.1, 1.0), "wa": n((C, 4 * C), C ** -0.5), "ba": n(4 * C, 0.1), "wb": n((4 * C, C), (4 * C) ** -0.5), "bb": n(C, 0.1)}
    for w in ("wa", "wb"):
        p[w + "t"] = (p[w][0].T, p[w][1].t().contiguous())
    g = n((M, C))
    buf = {k_: torch.empty(M, C, dtype=g[1].dtype, device="cuda") for k_ in ("v", "out")}
    buf |= {k_: afno.mx8_empty((M, c), "cuda") for k_, c in (("n", C), ("pre", 4 * C), ("h", 4 * C))}
    buf |= {"w8a": afno.mx8_empty((4 * C, C), "cuda"), "w8b": afno.mx8_empty((C, 4 * C), "cuda")}
    return v, p, g, buf


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,C", [(60, 64), (500, 256)])
def test_channel_mlp_in_eight_bits(M, C, dtype):
    """All operators together against the float64 chain without eight bits, by the relative 2-norm: an E4M3 rounding
    is off by at most 2^-3 / sqrt(12) of a value in the mean square, the step's width over the smallest value that has it,
    0.036; at most six of them (n, wa, pre, h, wb, and a gradient's own factor) meet in a result, independent: 0.088."""
    v, p, g, buf = mlp_setup(M, C, dtype)
    step = torch.tensor([41], dtype=torch.int64, device="cuda")
    r = [dict(p=0.1, seed=SEED, offset=i << 40, counter=step) for i in (1, 2)]
    o = [dict(p=0.1, seed=SEED, offset=i << 40, counter=41) for i in (1, 2)]
    dev = lambda d: {k_: t[1] for k_, t in d.items()}  # noqa: E731
    got = mlp_step(dev(v), dev(p), r, g[1], buf)
    torch.cuda.synchronize()
    w = {k_: t[0] for k_, t in {**v, **p}.items()}
    s = w["x"] + w["u"]
    n = om.rms_norm(s, w["g"], 1e-6)
    h, pre = ot.linear(n, w["wa"], w["ba"], "gelu", **o[0])
    out, _ = ot.linear(h, w["wb"], w["bb"], residual=s, **o[1])
    dh, dwb, dbb, _ = ot.linear_backward(g[0], h, w["wb"], **o[1])
    dn, dwa, dba, _ = ot.linear_backward(dh, n, w["wa"], pre, "gelu", **o[0])
    dv, dga = om.rms_norm_backward(dn, s, w["g"], 1e-6, g[0])
    for name, a, b in zip(("out", "dv", "dgamma", "dwa", "dba", "dwb", "dbb"), got, (out, dv, dga, dwa, dba, dwb, dbb)):
        e = np.linalg.norm(to_f64(a) - b) / np.linalg.norm(b)
        say(f"  {name} {e:.2e}")
        assert e <= 0.088, name


def bits(ts):
    return [t.view(torch.int16 if t.element_size() == 2 else torch.int32).clone() for t in ts]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_repeated_calls_other_streams_and_graphs(dtype):
    """The same bits again, on another stream, and from a graph replayed between eager calls; the counter on the
    device draws another mask in a replay."""
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
    fresh = mlp_setup(300, 64, dtype, seed=5)[3]
    for s in (3, 1, 2, 1):
        step.fill_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits(held), eager[s])), s
        mlp_step(v, p, r, g, fresh)
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

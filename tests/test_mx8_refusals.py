"""What the operators in eight bits and the root-mean-square norm refuse, before any HIP call: fake addresses through
the C ABI and CPU tensors through the Python wrappers, so nothing here reaches a GPU."""
import math

import pytest

import paper_2208_05419_amd as afno

INV, UNS, ALI = afno.AFNO_ERR_INVALID_ARG, afno.AFNO_ERR_UNSUPPORTED, afno.AFNO_ERR_ALIAS
A = [0x10000000 * (i + 1) for i in range(14)]
BF16 = afno.AFNO_DTYPE_BF16


def pack(**kw):
    a = dict(x=A[0], M=16, C=40, dtype=BF16, q=A[1], s=A[2])
    a.update(kw)
    return afno.afno_mx8_pack(*a.values(), None)


def unpack(**kw):
    a = dict(q=A[0], s=A[1], M=16, C=40, dtype=BF16, out=A[2])
    a.update(kw)
    return afno.afno_mx8_unpack(*a.values(), None)


def norm(**kw):
    a = dict(x=A[0], residual=A[1], gamma=A[2], M=16, C=40, eps=1e-6, dtype=BF16, out=A[3], sum=A[4], q=A[5], s=A[6])
    a.update(kw)
    return afno.afno_rms_norm_forward(*a.values(), None)


def norm_bwd(**kw):
    a = dict(g=A[0], x=A[1], gamma=A[2], gsum=A[3], M=16, C=40, eps=1e-6, dtype=BF16, dx=A[4], dgamma=A[5], ws=None, have=0)
    a.update(kw)
    return afno.afno_rms_norm_backward(*a.values(), None)


def linear(**kw):
    a = dict(xq=A[0], xs=A[1], wq=A[2], ws_=A[3], b=A[4], residual=A[5], M=16, K=64, N=40, act=2, p=0.1, seed=1, offset=2,
             counter=A[6], dtype=BF16, out=A[7], oq=A[8], os=A[9], pq=A[10], ps=A[11], ws=None, have=0)
    a.update(kw)
    return afno.afno_mx8_linear_forward(*a.values(), None)


def linear_bwd(**kw):
    a = dict(g=A[0], xq=A[1], xs=A[2], w=A[3], pq=A[4], ps=A[5], M=16, K=64, N=40, act=2, p=0.1, seed=1, offset=2, counter=A[6],
             dtype=BF16, dx=A[7], dw=A[8], db=A[9], ws=None, have=0)
    a.update(kw)
    return afno.afno_mx8_linear_backward(*a.values(), None)


REFUSED = [
    (pack, INV, dict(x=None)), (pack, INV, dict(q=None)), (pack, INV, dict(s=None)), (pack, INV, dict(q=None, s=None)),
    (pack, INV, dict(M=-1)), (pack, INV, dict(C=0)), (pack, INV, dict(dtype=2)), (pack, UNS, dict(q=A[1] + 8)),
    (pack, UNS, dict(x=A[0] + 1)), (pack, UNS, dict(dtype=0, x=A[0] + 2)), (pack, UNS, dict(C=2 ** 20 + 1)), (pack, UNS, dict(M=2 ** 25 + 1)),
    (pack, UNS, dict(M=2 ** 20, C=2 ** 15)), (pack, ALI, dict(q=A[0])), (pack, ALI, dict(q=A[0] + 16 * 40 * 2 - 16)), (pack, ALI, dict(s=A[1])),
    (pack, ALI, dict(s=A[1] + 16 * 64 - 1)), (pack, ALI, dict(q=A[0] - 16 * 64 + 16)),
    (unpack, INV, dict(q=None)), (unpack, INV, dict(s=None)), (unpack, INV, dict(out=None)), (unpack, INV, dict(C=-1)),
    (unpack, INV, dict(dtype=-1)), (unpack, UNS, dict(q=A[0] + 4)), (unpack, UNS, dict(out=A[2] + 1)), (unpack, ALI, dict(out=A[0])),
    (unpack, ALI, dict(out=A[1])), (unpack, UNS, dict(M=2 ** 62)),
    (norm, INV, dict(x=None)), (norm, INV, dict(gamma=None)), (norm, INV, dict(out=None, q=None, s=None)), (norm, INV, dict(s=None)),
    (norm, INV, dict(q=None)), (norm, INV, dict(M=-1)), (norm, INV, dict(C=0)), (norm, INV, dict(eps=-1.0)), (norm, INV, dict(eps=math.nan)),
    (norm, INV, dict(eps=math.inf)), (norm, INV, dict(dtype=3)), (norm, UNS, dict(x=A[0] + 1)), (norm, UNS, dict(q=A[5] + 2)),
    (norm, UNS, dict(C=2 ** 20 + 64)), (norm, UNS, dict(M=2 ** 24, C=2048)), (norm, ALI, dict(out=A[1])), (norm, ALI, dict(sum=A[0])),
    (norm, ALI, dict(sum=A[3])), (norm, ALI, dict(q=A[3])), (norm, ALI, dict(q=A[0])), (norm, ALI, dict(s=A[5])), (norm, ALI, dict(q=A[4])),
    (norm_bwd, INV, dict(g=None)), (norm_bwd, INV, dict(x=None)), (norm_bwd, INV, dict(gamma=None)), (norm_bwd, INV, dict(dx=None)),
    (norm_bwd, INV, dict(dgamma=None)), (norm_bwd, INV, dict(eps=-1e-6)), (norm_bwd, UNS, dict(dgamma=A[5] + 2)), (norm_bwd, ALI, dict(dx=A[0])),
    (norm_bwd, ALI, dict(dgamma=A[4])), (norm_bwd, ALI, dict(dgamma=A[3])), (norm_bwd, INV, dict(ws=A[8], have=8)),
    (norm_bwd, INV, dict(ws=A[8], have=-1)), (norm_bwd, UNS, dict(ws=A[8] + 8, have=1 << 26)), (norm_bwd, ALI, dict(ws=A[1], have=1 << 26)),
    (linear, INV, dict(xq=None)), (linear, INV, dict(xs=None)), (linear, INV, dict(wq=None, ws_=None)), (linear, INV, dict(ws_=None)),
    (linear, INV, dict(out=None, oq=None, os=None)), (linear, INV, dict(os=None)), (linear, INV, dict(pq=None)), (linear, INV, dict(M=-1)),
    (linear, INV, dict(K=0)), (linear, INV, dict(N=0)), (linear, INV, dict(act=3)), (linear, INV, dict(dtype=2)), (linear, INV, dict(p=1.0)),
    (linear, INV, dict(p=math.nan)), (linear, UNS, dict(xq=A[0] + 8)), (linear, UNS, dict(wq=A[2] + 1)), (linear, UNS, dict(oq=A[8] + 4)),
    (linear, UNS, dict(pq=A[10] + 8)), (linear, UNS, dict(b=A[4] + 1)), (linear, UNS, dict(counter=A[6] + 4)), (linear, UNS, dict(K=2 ** 20 + 1)),
    (linear, UNS, dict(M=2 ** 25 + 1)), (linear, UNS, dict(M=2 ** 25, N=1024)), (linear, UNS, dict(M=2 ** 62)), (linear, UNS, dict(N=2 ** 21)),
    (linear, ALI, dict(out=A[0])), (linear, ALI, dict(out=A[5])), (linear, ALI, dict(oq=A[7])), (linear, ALI, dict(os=A[8] + 16 * 64 - 1)),
    (linear, ALI, dict(pq=A[2])), (linear, ALI, dict(ps=A[9] + 1)), (linear, ALI, dict(pq=A[8])), (linear, ALI, dict(out=A[6])),
    (linear, ALI, dict(out=A[3])), (linear, ALI, dict(K=8192, ws=A[0], have=1 << 26)), (linear, INV, dict(K=8192, ws=A[12], have=16)),
    (linear_bwd, INV, dict(g=None)), (linear_bwd, INV, dict(xq=None)), (linear_bwd, INV, dict(xq=None, xs=None)), (linear_bwd, INV, dict(w=None)),
    (linear_bwd, INV, dict(pq=None, ps=None)), (linear_bwd, INV, dict(ps=None)), (linear_bwd, INV, dict(dx=None, dw=None, db=None)),
    (linear_bwd, INV, dict(N=-1)), (linear_bwd, INV, dict(p=2.0)), (linear_bwd, UNS, dict(xq=A[1] + 8)), (linear_bwd, UNS, dict(pq=A[4] + 1)),
    (linear_bwd, UNS, dict(db=A[9] + 1)), (linear_bwd, ALI, dict(dx=A[0])), (linear_bwd, ALI, dict(dw=A[1])), (linear_bwd, ALI, dict(dx=A[2])),
    (linear_bwd, ALI, dict(db=A[7])), (linear_bwd, ALI, dict(dx=A[4])), (linear_bwd, INV, dict(ws=A[10], have=16)),
    (linear_bwd, UNS, dict(ws=A[10] + 8, have=1 << 26)), (linear_bwd, ALI, dict(ws=A[1] - 64, have=1 << 26)),
]


@pytest.mark.parametrize("call,want,kw", REFUSED)
def test_refused(call, want, kw):
    assert call(**kw) == want
    assert afno.afno_last_error() != ""


def test_nothing_to_do_needs_no_gpu():
    assert pack(M=0, x=None, q=None, s=None) == afno.AFNO_OK
    assert unpack(M=0, q=None, s=None, out=None) == afno.AFNO_OK
    assert norm(M=0, x=None, out=None, q=None, s=None) == afno.AFNO_OK
    assert linear(M=0, xq=None, xs=None, out=None, oq=None, os=None, pq=None, ps=None) == afno.AFNO_OK
    assert linear_bwd(M=0, dw=None, db=None, xq=None, xs=None) == afno.AFNO_OK
    assert linear(M=0, K=0) == INV and pack(M=0, C=0) == INV  # sizes are checked all the same


def test_workspace_sizes():
    fwd, bwd, nrm = (afno.afno_mx8_linear_forward_workspace, afno.afno_mx8_linear_backward_workspace,
                     afno.afno_rms_norm_backward_workspace)
    for f, sizes, more in ((fwd, (16, 64, 32), ()), (bwd, (16, 64, 32), (1,)), (bwd, (16, 64, 32), (0,)), (nrm, (16, 64), ())):
        assert f(*sizes, 0, *more) >= 0 and f(*sizes, BF16, *more) >= 0
        assert f(0, *sizes[1:], 0, *more) == 0
        assert f(-1, *sizes[1:], 0, *more) == INV and f(sizes[0], 0, *sizes[2:], 0, *more) == INV
        assert f(*sizes, 5, *more) == INV and f(2 ** 31, *sizes[1:], 0, *more) == UNS
    # x in the storage type, dz and the chunks' sums at least
    assert bwd(1000, 64, 32, 0, 1) >= 1000 * (64 + 32) * 4 + 32 * 4
    assert nrm(1000, 64, 0) >= 64 * 4 and nrm(3, 2 ** 20, 0) >= 2 ** 20 * 4 + 3 * 4 and nrm(3, 2 ** 20 + 1, 0) == UNS


def test_python_refusals():
    torch = pytest.importorskip("torch")
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    e = lambda *s: afno.mx8_empty(s, "cpu")  # noqa: E731
    x, x8 = z(3, 40), e(3, 40)
    assert x8.values.shape == (3, 64) and x8.scales.shape == (3, 2) and x8.shape == (3, 40)
    wrong = afno.Mx8(x8.values.view(torch.uint8), x8.scales, 40)
    strided = afno.Mx8(e(3, 80).values[:, :64], x8.scales, 40)
    bad = [
        (ValueError, lambda: afno.mx8_pack(None)), (ValueError, lambda: afno.mx8_pack(z(3, 0))), (TypeError, lambda: afno.mx8_pack(x.half())),
        (ValueError, lambda: afno.mx8_pack(x)), (ValueError, lambda: afno.mx8_pack(x.t())),
        (TypeError, lambda: afno.mx8_unpack(x)), (ValueError, lambda: afno.mx8_unpack(None)), (TypeError, lambda: afno.mx8_unpack(wrong)),
        (ValueError, lambda: afno.mx8_unpack(afno.Mx8(x8.values, x8.scales, 65))), (ValueError, lambda: afno.mx8_unpack(strided)),
        (ValueError, lambda: afno.mx8_unpack(afno.Mx8(x8.values, e(3, 65).scales, 40))), (ValueError, lambda: afno.mx8_unpack(x8)),
        (ValueError, lambda: afno.rms_norm_forward(x, z(41))), (ValueError, lambda: afno.rms_norm_forward(x, None)),
        (TypeError, lambda: afno.rms_norm_forward(x, z(40, dtype=torch.bfloat16))), (ValueError, lambda: afno.rms_norm_forward(x, z(40))),
        (ValueError, lambda: afno.rms_norm_backward(None, x, z(40))), (ValueError, lambda: afno.rms_norm_backward(x, x, z(40), gsum=z(3))),
        (TypeError, lambda: afno.mx8_linear_forward(x, e(5, 40))), (ValueError, lambda: afno.mx8_linear_forward(x8, None)),
        (ValueError, lambda: afno.mx8_linear_forward(x8, e(5, 41))), (ValueError, lambda: afno.mx8_linear_forward(x8, e(40))),
        (ValueError, lambda: afno.mx8_linear_forward(x8, e(5, 40))),
        (TypeError, lambda: afno.mx8_linear_backward(z(3, 5), x, z(40, 5))), (ValueError, lambda: afno.mx8_linear_backward(None, x8, z(40, 5))),
        (ValueError, lambda: afno.mx8_linear_backward(z(3, 6), x8, z(40, 5))), (ValueError, lambda: afno.mx8_linear_backward(z(3, 5), x8, z(5))),
        (TypeError, lambda: afno.mx8_linear_backward(z(3, 5), x8, z(40, 5, dtype=torch.bfloat16))),
        (ValueError, lambda: afno.mx8_linear_backward(z(3, 5), x8, z(40, 5))),
    ]
    for i, (kind, f) in enumerate(bad):
        with pytest.raises(kind):
            f()
            pytest.fail(f"call {i} was taken")


def test_python_checks_of_eight_bit_tensors():
    """_expect8 by itself, which on the GPU stands between a wrong tensor and a kernel."""
    torch = pytest.importorskip("torch")
    from paper_2208_05419_amd.mx8 import _expect8
    cpu, ok = torch.device("cpu"), afno.mx8_empty((2, 3, 33), "cpu")
    for kind, t, shape, device in (
            (ValueError, None, (2, 3, 33), cpu), (TypeError, tuple(ok), (2, 3, 33), cpu), (ValueError, ok, (6, 33), cpu),
            (ValueError, ok, (2, 3, 34), cpu), (ValueError, ok, (2, 3, 33), torch.device("meta")),
            (TypeError, afno.Mx8(ok.values, ok.scales.view(torch.uint8), 33), (2, 3, 33), cpu),
            (TypeError, afno.Mx8(ok.values.view(torch.float8_e5m2), ok.scales, 33), (2, 3, 33), cpu),
            (ValueError, afno.Mx8(ok.values, ok.scales, 32), (2, 3, 32), cpu),
            (ValueError, afno.Mx8(ok.values, ok.scales[..., :1], 33), (2, 3, 33), cpu),
            (ValueError, afno.Mx8(ok.values.transpose(0, 1).contiguous().transpose(0, 1), ok.scales, 33), (2, 3, 33), cpu),
            (ValueError, ok, (2, 3, 33), cpu)):  # as it should be, but on the CPU
        with pytest.raises(kind):
            _expect8("t", t, shape, device)

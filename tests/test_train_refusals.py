"""What the linear products, LayerNorm and dropout refuse, before any HIP call: fake addresses through
the C ABI and CPU tensors through the Python wrappers, so nothing here reaches a GPU."""
import math

import pytest

import paper_2208_05419_amd as afno

INV, UNS, ALI = afno.AFNO_ERR_INVALID_ARG, afno.AFNO_ERR_UNSUPPORTED, afno.AFNO_ERR_ALIAS
A = [0x10000000 * (i + 1) for i in range(9)]
BF16 = afno.AFNO_DTYPE_BF16


def linear(**kw):
    a = dict(x=A[0], w=A[1], b=A[2], residual=A[3], M=16, K=64, N=32, act=2, p=0.1, seed=1, offset=2,
             counter=A[6], dtype=BF16, out=A[4], pre=A[5], ws=None, have=0)
    a.update(kw)
    return afno.afno_linear_forward(*a.values(), None)


def linear_bwd(**kw):
    a = dict(g=A[0], x=A[1], w=A[2], pre=A[3], M=16, K=64, N=32, act=2, p=0.1, seed=1, offset=2,
             counter=A[7], dtype=BF16, dx=A[4], dw=A[5], db=A[6], ws=None, have=0)
    a.update(kw)
    return afno.afno_linear_backward(*a.values(), None)


def norm(**kw):
    a = dict(x=A[0], residual=A[1], gamma=A[2], beta=A[3], M=16, C=64, eps=1e-6, dtype=BF16, out=A[4], sum=A[5])
    a.update(kw)
    return afno.afno_layer_norm_forward(*a.values(), None)


def norm_bwd(**kw):
    a = dict(g=A[0], x=A[1], gamma=A[2], gsum=A[3], M=16, C=64, eps=1e-6, dtype=BF16, dx=A[4], dgamma=A[5],
             dbeta=A[6], ws=None, have=0)
    a.update(kw)
    return afno.afno_layer_norm_backward(*a.values(), None)


def drop(**kw):
    a = dict(x=A[0], residual=A[1], n=100, p=0.1, seed=1, offset=2, counter=A[3], dtype=BF16, out=A[2])
    a.update(kw)
    return afno.afno_dropout_forward(*a.values(), None)


@pytest.mark.parametrize("call,want,kw", [
    (linear, INV, dict(x=None)), (linear, INV, dict(w=None)), (linear, INV, dict(out=None)),
    (linear, INV, dict(M=-1)), (linear, INV, dict(K=0)), (linear, INV, dict(N=0)), (linear, INV, dict(act=3)),
    (linear, INV, dict(act=-1)), (linear, INV, dict(dtype=2)), (linear, INV, dict(p=1.0)),
    (linear, INV, dict(p=-0.1)), (linear, INV, dict(p=math.nan)), (linear, INV, dict(p=1 - 2.0 ** -18)),
    (linear, UNS, dict(x=A[0] + 1)), (linear, UNS, dict(b=A[2] + 1)), (linear, UNS, dict(counter=A[6] + 4)),
    (linear, UNS, dict(dtype=0, w=A[1] + 2)), (linear, UNS, dict(K=2 ** 20 + 1)), (linear, UNS, dict(M=2 ** 25 + 1)),
    (linear, UNS, dict(M=2 ** 25, N=1024)), (linear, UNS, dict(M=2 ** 62)), (norm, UNS, dict(M=2 ** 24, C=2048)),
    (linear, UNS, dict(N=2 ** 21)), (linear, ALI, dict(out=A[0])), (linear, ALI, dict(out=A[1] + 64)),
    (linear, ALI, dict(out=A[3])), (linear, ALI, dict(pre=A[4] + 16 * 32 * 2 - 2)), (linear, ALI, dict(pre=A[2])),
    (linear, ALI, dict(out=A[6])),
    (linear_bwd, INV, dict(g=None)), (linear_bwd, INV, dict(x=None)), (linear_bwd, INV, dict(w=None)),
    (linear_bwd, INV, dict(pre=None)), (linear_bwd, INV, dict(dx=None, dw=None, db=None)),
    (linear_bwd, INV, dict(K=-1)), (linear_bwd, INV, dict(p=2.0)), (linear_bwd, UNS, dict(db=A[6] + 1)),
    (linear_bwd, ALI, dict(dx=A[0])), (linear_bwd, ALI, dict(dw=A[2])), (linear_bwd, ALI, dict(db=A[4])),
    (linear_bwd, ALI, dict(dx=A[3])),
    (norm, INV, dict(x=None)), (norm, INV, dict(gamma=None)), (norm, INV, dict(beta=None)),
    (norm, INV, dict(out=None)), (norm, INV, dict(M=-1)), (norm, INV, dict(C=0)), (norm, INV, dict(eps=-1.0)),
    (norm, INV, dict(eps=math.inf)), (norm, INV, dict(eps=math.nan)), (norm, INV, dict(dtype=-1)),
    (norm, UNS, dict(x=A[0] + 1)), (norm, UNS, dict(C=2 ** 20 + 64)), (norm, ALI, dict(out=A[1])),
    (norm, ALI, dict(sum=A[0])), (norm, ALI, dict(sum=A[4])),
    (norm_bwd, INV, dict(g=None)), (norm_bwd, INV, dict(dx=None)), (norm_bwd, INV, dict(dgamma=None)),
    (norm_bwd, INV, dict(dbeta=None)), (norm_bwd, INV, dict(eps=-1e-6)), (norm_bwd, UNS, dict(dgamma=A[5] + 2)),
    (norm_bwd, ALI, dict(dx=A[0])), (norm_bwd, ALI, dict(dbeta=A[5] + 4)), (norm_bwd, ALI, dict(dgamma=A[3])),
    (linear_bwd, INV, dict(ws=A[8], have=16)), (linear_bwd, INV, dict(ws=A[8], have=-1)),
    (linear_bwd, UNS, dict(ws=A[8] + 8, have=1 << 26)), (linear_bwd, ALI, dict(ws=A[4], have=1 << 26)),
    (linear_bwd, ALI, dict(ws=A[0] - 64, have=1 << 26)), (norm_bwd, INV, dict(ws=A[8], have=8)),
    (norm_bwd, ALI, dict(ws=A[1], have=1 << 26)), (linear, ALI, dict(K=4096, ws=A[0], have=1 << 26)),
    (drop, INV, dict(x=None)), (drop, INV, dict(out=None)), (drop, INV, dict(n=-1)), (drop, INV, dict(p=1.0)),
    (drop, INV, dict(dtype=7)), (drop, UNS, dict(x=A[0] + 1)), (drop, UNS, dict(n=2 ** 34 + 1)), (drop, UNS, dict(n=2 ** 62)),
    (drop, ALI, dict(out=A[0])), (drop, ALI, dict(out=A[1] + 4)),
])
def test_refused(call, want, kw):
    assert call(**kw) == want
    assert afno.afno_last_error() != ""


def test_nothing_to_do_needs_no_gpu():
    assert linear(M=0, x=None, out=None, pre=None) == afno.AFNO_OK
    assert linear_bwd(M=0, dw=None, db=None) == afno.AFNO_OK
    assert norm(M=0, x=None, out=None) == afno.AFNO_OK
    assert drop(n=0, x=None, out=None) == afno.AFNO_OK
    assert afno.afno_dropout_backward(None, 0, 0.5, 1, 2, None, BF16, None, None) == afno.AFNO_OK
    assert linear(M=0, K=0) == INV  # sizes are checked all the same


def test_workspace_sizes():
    for f, sizes, more in ((afno.afno_linear_forward_workspace, (16, 64, 32), (1,)),
                           (afno.afno_linear_forward_workspace, (16, 64, 32), (0,)),
                           (afno.afno_linear_backward_workspace, (16, 64, 32), (1,)),
                           (afno.afno_layer_norm_backward_workspace, (16, 64), ())):
        assert f(*sizes, 0, *more) >= 0 and f(*sizes, BF16, *more) >= 0
        assert f(0, *sizes[1:], 0, *more) == 0
        assert f(-1, *sizes[1:], 0, *more) == INV and f(sizes[0], 0, *sizes[2:], 0, *more) == INV
        assert f(*sizes, 5, *more) == INV and f(2 ** 31, *sizes[1:], 0, *more) == UNS
    # the factor dz and the chunks' sums at least, and copies of rows that are no 16-byte units
    assert afno.afno_linear_backward_workspace(1000, 64, 32, 0, 1) >= 1000 * 32 * 4 + 32 * 4
    assert afno.afno_layer_norm_backward_workspace(1000, 64, 0) >= 2 * 64 * 4
    for f in (afno.afno_linear_forward_workspace, afno.afno_linear_backward_workspace):
        assert f(9000, 512, 512, BF16, 0) > f(9000, 512, 512, BF16, 1)
        assert f(9000, 513, 512, BF16, 1) >= 9000 * 520 * 2


def test_workspace_sizes_of_the_widest_rows():
    """What a call takes its workspace query takes: a norm has no array of C x C."""
    for C in (2 ** 17 + 1, 2 ** 20):
        assert afno.afno_layer_norm_backward_workspace(3, C, 0) >= 2 * C * 4 + 3 * 8
    assert afno.afno_layer_norm_backward_workspace(3, 2 ** 20 + 1, 0) == UNS


def test_python_refusals():
    torch = pytest.importorskip("torch")
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    x, w = z(3, 4), z(4, 5)
    bad = [
        (ValueError, lambda: afno.linear_forward(x, z(5, 5))),
        (ValueError, lambda: afno.linear_forward(x, z(4))),
        (ValueError, lambda: afno.linear_forward(x, None)),
        (ValueError, lambda: afno.linear_forward(z(3, 0), z(0, 5))),
        (TypeError, lambda: afno.linear_forward(x, z(4, 5, dtype=torch.bfloat16))),
        (TypeError, lambda: afno.linear_forward(x.half(), w.half())),
        (ValueError, lambda: afno.linear_forward(x, w, z(4))),
        (ValueError, lambda: afno.linear_forward(x, w, residual=z(3, 4))),
        (ValueError, lambda: afno.linear_forward(x, w, out=z(5, 3))),
        (ValueError, lambda: afno.linear_forward(x, z(5, 4).t())),  # not contiguous
        (ValueError, lambda: afno.linear_forward(x, w)),  # not on the GPU
        (ValueError, lambda: afno.linear_backward(z(3, 5), x, w, activation="gelu")),  # pre is missing
        (ValueError, lambda: afno.linear_backward(z(3, 4), x, w)),
        (ValueError, lambda: afno.layer_norm_forward(x, z(5), z(4))),
        (ValueError, lambda: afno.layer_norm_forward(x, z(4), z(4), residual=z(4, 4))),
        (TypeError, lambda: afno.layer_norm_forward(x, z(4), z(4, dtype=torch.bfloat16))),
        (ValueError, lambda: afno.layer_norm_backward(z(3, 5), x, z(4))),
        (ValueError, lambda: afno.layer_norm_backward(z(3, 4), x, z(4), gsum=z(3))),
        (ValueError, lambda: afno.dropout_forward(x, 0.1, 1, residual=z(4, 3))),
        (ValueError, lambda: afno.dropout_forward(x, 0.1, 1)),
        (TypeError, lambda: afno.dropout_forward(x.long(), 0.1, 1)),
        (ValueError, lambda: afno.dropout_backward(x, 0.1, 1, out=z(3, 5))),
    ]
    for kind, f in bad:
        with pytest.raises(kind):
            f()


def test_python_random_arguments():
    from paper_2208_05419_amd import train
    torch = pytest.importorskip("torch")
    x = torch.zeros(3)
    for seed, offset in ((-1, 0), (0, 2 ** 64), (1.5, 0), (0, None)):
        with pytest.raises(ValueError):
            train._random(x, 0.1, seed, offset, None)
    for c in (torch.zeros(2, dtype=torch.int64), torch.zeros(1)):
        with pytest.raises(TypeError):
            train._random(x, 0.1, 0, 0, c)
    assert train._random(x, 0.1, 2 ** 64 - 1, 3, None) == (0.1, 2 ** 64 - 1, 3, None)
    with pytest.raises(ValueError):
        train._activation("softplus")

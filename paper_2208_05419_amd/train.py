"""Python binding of the operators that train a network around the filter (include/afno.h): linear
products with their epilogue, LayerNorm of a residual sum, dropout, each with its gradient.

As in ``afno.py`` this is argument marshalling only.  Tensors are rows of channels with any leading
shape ([B, H, W, C] grids, [M, C] tokens), float32 or bfloat16, contiguous, on one GPU.  With a stream of the
caller's, the tensors that a call returns are allocated for that stream, and what it reads is recorded on it.
"""
from __future__ import annotations

import contextlib
import functools

from .afno import (AFNO_ACT_GELU, AFNO_ACT_NONE, AFNO_ACT_RELU, _check, _dtype_code, _expect,
                   load_library)

ACTIVATIONS = {"none": AFNO_ACT_NONE, "relu": AFNO_ACT_RELU, "gelu": AFNO_ACT_GELU}


def afno_linear_forward(x, w, b, residual, M, K, N, activation, p, seed, offset, counter, dtype, out,
                        pre, workspace, workspace_bytes, stream) -> int:
    """Raw call: pointers as ints (or None), returns the C return code."""
    return load_library().afno_linear_forward(x, w, b, residual, M, K, N, activation, p, seed, offset,
                                              counter, dtype, out, pre, workspace, workspace_bytes,
                                              stream)


def afno_linear_backward(g, x, w, pre, M, K, N, activation, p, seed, offset, counter, dtype, dx, dw, db,
                         workspace, workspace_bytes, stream) -> int:
    return load_library().afno_linear_backward(g, x, w, pre, M, K, N, activation, p, seed, offset,
                                               counter, dtype, dx, dw, db, workspace, workspace_bytes,
                                               stream)


def afno_layer_norm_forward(x, residual, gamma, beta, M, C, eps, dtype, out, sum_out, stream) -> int:
    return load_library().afno_layer_norm_forward(x, residual, gamma, beta, M, C, eps, dtype, out,
                                                  sum_out, stream)


def afno_layer_norm_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, dbeta, workspace,
                             workspace_bytes, stream) -> int:
    return load_library().afno_layer_norm_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma,
                                                   dbeta, workspace, workspace_bytes, stream)


def afno_dropout_forward(x, residual, n, p, seed, offset, counter, dtype, out, stream) -> int:
    return load_library().afno_dropout_forward(x, residual, n, p, seed, offset, counter, dtype, out,
                                               stream)


def afno_dropout_backward(g, n, p, seed, offset, counter, dtype, dx, stream) -> int:
    return load_library().afno_dropout_backward(g, n, p, seed, offset, counter, dtype, dx, stream)


def afno_linear_forward_workspace(M, K, N, dtype, aligned) -> int:
    """Bytes of workspace that the call may need, or a (negative) error code."""
    return load_library().afno_linear_forward_workspace(M, K, N, dtype, aligned)


def afno_linear_backward_workspace(M, K, N, dtype, aligned) -> int:
    return load_library().afno_linear_backward_workspace(M, K, N, dtype, aligned)


def afno_layer_norm_backward_workspace(M, C, dtype) -> int:
    return load_library().afno_layer_norm_backward_workspace(M, C, dtype)


# ---------------------------------------------------------------- torch-level wrappers


def _address(t):
    """Address of a tensor that _expect has checked, or None."""
    return None if t is None else t.data_ptr() or None


def _aligned(*addresses) -> bool:
    """Whether all are multiples of 16 (None counts)."""
    return all(not a or a % 16 == 0 for a in addresses)


def _fit(x, *pairs) -> bool:
    """Whether _expect would pass: every tensor (or None) of the (tensor, shape) pairs has that shape
    and x's dtype and device, all are contiguous, and x is on the GPU.  Small calls take about as long as
    their checks, and this is the quick one; _expect says what is wrong."""
    dtype, device = x.dtype, x.device
    for t, shape in pairs:
        if t is not None and (t.shape != shape or t.dtype != dtype or t.device != device
                              or not t.is_contiguous()):
            return False
    return x.is_contiguous() and x.is_cuda


def _rows(name, x):
    """(M, C, dtype code) of a tensor seen as rows of channels."""
    if x is None:
        raise ValueError(f"{name} is missing")
    if x.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    code, C = _dtype_code(x), x.shape[-1]
    if C == 0:
        raise ValueError(f"{name} has no channels")
    return x.numel() // C, C, code


def _activation(activation) -> int:
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {activation!r}")
    return ACTIVATIONS[activation]


def _random(x, p, seed, offset, counter):
    """Dropout's arguments checked: p, the two 64-bit numbers, the counter's address."""
    if not (isinstance(seed, int) and isinstance(offset, int) and 0 <= seed < 2 ** 64 and 0 <= offset < 2 ** 64):
        raise ValueError(f"seed and offset must be ints in [0, 2^64), got {seed!r} and {offset!r}")
    if counter is not None:
        import torch
        if counter.dtype != torch.int64 or counter.numel() != 1:
            raise TypeError("counter must be an int64 tensor of one element")
        if counter.device != x.device:
            raise ValueError(f"counter is on {counter.device}, the input on {x.device}")
    return float(p), seed, offset, None if counter is None else counter.data_ptr()


def _launch(x, stream, tensors, call):
    """call(stream handle) with x's device current and new tensors allocated for that stream.  A
    caller's stream other than torch's current one is recorded on the tensors that the call reads, so
    that their memory is not handed out again before it has run."""
    import torch
    device = x.get_device()
    here = torch._C._cuda_getDevice() == device
    if stream is None and here:
        return call(torch._C._cuda_getCurrentRawStream(device))
    with contextlib.ExitStack() as stack:
        if not here:
            stack.enter_context(torch.cuda.device(device))
        if stream is None:
            return call(torch._C._cuda_getCurrentRawStream(device))
        if stream.device != x.device:
            raise ValueError(f"stream is on {stream.device}, the tensors on {x.device}")
        if stream.cuda_stream != torch._C._cuda_getCurrentRawStream(device):
            stack.enter_context(torch.cuda.stream(stream))
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
        return call(stream.cuda_stream)


@functools.lru_cache(maxsize=1024)
def _bytes(query, *sizes) -> int:
    """The workspace query of these sizes (a function of them alone)."""
    n = query(*sizes)
    _check(min(n, 0))
    return n


def _workspace(x, nbytes: int):
    """(address, bytes) of a workspace from torch's allocator, which a captured graph keeps, and the
    tensor that holds it."""
    if nbytes == 0:
        return None, 0, None
    t = x.new_empty(-(-nbytes // x.element_size()))
    return t.data_ptr(), nbytes, t


def linear_forward(x, w, b=None, *, activation="none", residual=None, p=0.0, seed=0, offset=0,
                   counter=None, out=None, pre=None, stream=None):
    """out = drop(act(x w + b)) + residual for x [..., K], w [K, N], b [N] or None, residual and out
    [..., N]; activation "none", "relu" or "gelu" (the exact one).  pre: a tensor like out that
    receives x w + b, which linear_backward takes where there is an activation.

    Dropout with probability p (in units of 2^-16; 0: none) keeps an element by its flat index, seed
    and offset (+ counter[0], an int64 tensor on x's device that is read when the kernel runs): the
    same numbers give the same mask, so a model gives each of its dropouts an offset range of its own
    and counts its steps in counter.  Enqueued on ``stream`` (default: torch's current stream)."""
    M, K, code = _rows("x", x)
    if w is None or w.dim() != 2:
        raise ValueError("w must be [K, N]")
    N = w.shape[1]
    shape = (*x.shape[:-1], N)
    if not _fit(x, (w, (K, N)), (b, (N,)), (residual, shape), (out, shape), (pre, shape)):
        _expect(x, [("w", w, (K, N), None)] + [(n, t, s, None) for n, t, s in (
            ("b", b, (N,)), ("residual", residual, shape), ("out", out, shape), ("pre", pre, shape)) if t is not None])
    act, drop = _activation(activation), _random(x, p, seed, offset, counter)

    def call(handle):
        y = x.new_empty(shape) if out is None else out
        px, pw = _address(x), _address(w)
        ws, nbytes, _held = _workspace(x, _bytes(afno_linear_forward_workspace, M, K, N, code,
                                                 _aligned(px, pw)))
        _check(afno_linear_forward(px, pw, _address(b), _address(residual), M, K, N, act, *drop,
                                   code, _address(y), _address(pre), ws, nbytes, handle))
        return y

    return _launch(x, stream, (x, w, b, residual, out, pre, counter), call)


def linear_backward(g, x, w, *, pre=None, activation="none", p=0.0, seed=0, offset=0, counter=None,
                    bias=True, need_dx=True, need_dw=True, stream=None):
    """Gradients of linear_forward for g = dL/dout [..., N] (the residual's gradient is g itself):
    a dict with dx like x, dw like w, db [N], in x's dtype, None where bias, need_dx or need_dw says
    that it is not wanted.  activation, p, seed, offset and the counter's value as in the forward
    call, pre the tensor that it filled (not read without an activation).  ReLU passes on 0 where pre is not
    above 0, whatever g is there."""
    M, K, code = _rows("x", x)
    if w is None or w.dim() != 2:
        raise ValueError("w must be [K, N]")
    N = w.shape[1]
    act = _activation(activation)
    shape = (*x.shape[:-1], N)
    if act == AFNO_ACT_NONE:
        pre = None  # not read
    if g is None or (act and pre is None) or not _fit(x, (w, (K, N)), (g, shape), (pre, shape)):
        _expect(x, [("w", w, (K, N), None), ("g", g, shape, None)] + ([("pre", pre, shape, None)] if act else []))
    if not (bias or need_dx or need_dw):
        raise ValueError("no gradient is asked for")
    drop = _random(x, p, seed, offset, counter)

    def call(handle):
        dx = x.new_empty(x.shape) if need_dx else None
        dw = x.new_empty((K, N)) if need_dw else None
        db = x.new_empty(N) if bias else None
        pg, px, pw = _address(g), _address(x), _address(w)
        ws, nbytes, _held = _workspace(x, _bytes(afno_linear_backward_workspace, M, K, N, code,
                                                 _aligned(pg, px, pw)))
        _check(afno_linear_backward(pg, px, pw, _address(pre), M, K, N, act, *drop, code, _address(dx),
                                    _address(dw), _address(db), ws, nbytes, handle))
        return {"dx": dx, "dw": dw, "db": db}

    return _launch(x, stream, (g, x, w, pre, counter), call)


def layer_norm_forward(x, gamma, beta, *, eps=1e-6, residual=None, out=None, sum_out=None, stream=None):
    """LayerNorm over the last axis of v = x + residual (rounded to x's dtype; None: v = x):
    (v - mean) / sqrt(var + eps) * gamma + beta with the biased variance.  sum_out: a tensor like x
    that receives v, the residual stream and what layer_norm_backward takes."""
    M, C, code = _rows("x", x)
    shape = x.shape
    if gamma is None or beta is None or not _fit(x, (gamma, (C,)), (beta, (C,)), (residual, shape), (out, shape),
                                                 (sum_out, shape)):
        _expect(x, [("gamma", gamma, (C,), None), ("beta", beta, (C,), None)] + [
            (n, t, tuple(shape), None) for n, t in (("residual", residual), ("out", out), ("sum_out", sum_out))
            if t is not None])

    def call(handle):
        y = x.new_empty(shape) if out is None else out
        _check(afno_layer_norm_forward(_address(x), _address(residual), _address(gamma), _address(beta), M, C, eps,
                                       code, _address(y), _address(sum_out), handle))
        return y

    return _launch(x, stream, (x, gamma, beta, residual, out, sum_out), call)


def layer_norm_backward(g, x, gamma, *, eps=1e-6, gsum=None, stream=None):
    """Gradients of the norm of x (the v that the forward call stored) for g = dL/dout: a dict with dx
    (x's dtype; gsum, the gradient that reaches v along the residual stream, is added to it) and
    dgamma, dbeta (float32)."""
    import torch
    M, C, code = _rows("x", x)
    shape = x.shape
    if gamma is None or g is None or not _fit(x, (gamma, (C,)), (g, shape), (gsum, shape)):
        _expect(x, [("gamma", gamma, (C,), None), ("g", g, tuple(shape), None)] + (
            [] if gsum is None else [("gsum", gsum, tuple(shape), None)]))

    def call(handle):
        dx = x.new_empty(shape)
        dgamma, dbeta = x.new_empty(C, dtype=torch.float32), x.new_empty(C, dtype=torch.float32)
        ws, nbytes, _held = _workspace(x, _bytes(afno_layer_norm_backward_workspace, M, C, code))
        _check(afno_layer_norm_backward(_address(g), _address(x), _address(gamma), _address(gsum), M, C, eps, code,
                                        _address(dx), _address(dgamma), _address(dbeta), ws, nbytes, handle))
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}

    return _launch(x, stream, (g, x, gamma, gsum), call)


def dropout_forward(x, p, seed, *, offset=0, counter=None, residual=None, out=None, stream=None):
    """drop(x) + residual for a tensor of any shape; dropout's numbers as in linear_forward."""
    if x is None:
        raise ValueError("x is missing")
    code, shape = _dtype_code(x), x.shape
    if not _fit(x, (residual, shape), (out, shape)):
        _expect(x, [(n, t, tuple(shape), None) for n, t in (("residual", residual), ("out", out)) if t is not None])
    drop = _random(x, p, seed, offset, counter)

    def call(handle):
        y = x.new_empty(shape) if out is None else out
        _check(afno_dropout_forward(_address(x), _address(residual), x.numel(), *drop, code, _address(y), handle))
        return y

    return _launch(x, stream, (x, residual, out, counter), call)


def dropout_backward(g, p, seed, *, offset=0, counter=None, out=None, stream=None):
    """drop(g), the gradient of dropout_forward's x for g = dL/dout (the residual's is g)."""
    if g is None:
        raise ValueError("g is missing")
    code, shape = _dtype_code(g), g.shape
    if not _fit(g, (out, shape)):
        _expect(g, [] if out is None else [("out", out, tuple(shape), None)])
    drop = _random(g, p, seed, offset, counter)

    def call(handle):
        dx = g.new_empty(shape) if out is None else out
        _check(afno_dropout_backward(_address(g), g.numel(), *drop, code, _address(dx), handle))
        return dx

    return _launch(g, stream, (g, out, counter), call)

"""Python binding of the operators in eight bits and of the root-mean-square norm (include/afno.h): a block's channel
MLP with its rows kept and multiplied in half the memory of bfloat16.

As in ``train.py`` this is argument marshalling only, for rows of channels with any leading shape, contiguous, on one
GPU, and a caller's stream is treated as there.
"""
from __future__ import annotations

from typing import NamedTuple

from .afno import (AFNO_ACT_NONE, AFNO_DTYPE_BF16, AFNO_DTYPE_FP32, _check, _dtype_code, _expect,
                   load_library)
from .train import (_activation, _address, _aligned, _bytes, _fit, _launch, _random, _rows, _workspace)

BLOCK = 32  # channels to a scale


def afno_mx8_pack(x, M, C, dtype, values, scales, stream) -> int:
    """Raw call: pointers as ints (or None), returns the C return code."""
    return load_library().afno_mx8_pack(x, M, C, dtype, values, scales, stream)


def afno_mx8_unpack(values, scales, M, C, dtype, out, stream) -> int:
    return load_library().afno_mx8_unpack(values, scales, M, C, dtype, out, stream)


def afno_rms_norm_forward(x, residual, gamma, M, C, eps, dtype, out, sum_out, out_values, out_scales, stream) -> int:
    return load_library().afno_rms_norm_forward(x, residual, gamma, M, C, eps, dtype, out, sum_out, out_values,
                                                out_scales, stream)


def afno_rms_norm_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, workspace, workspace_bytes, stream) -> int:
    return load_library().afno_rms_norm_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, workspace,
                                                 workspace_bytes, stream)


def afno_mx8_linear_forward(x_values, x_scales, w_values, w_scales, b, residual, M, K, N, activation, p, seed, offset,
                            counter, dtype, out, out_values, out_scales, pre_values, pre_scales, workspace,
                            workspace_bytes, stream) -> int:
    return load_library().afno_mx8_linear_forward(x_values, x_scales, w_values, w_scales, b, residual, M, K, N,
                                                  activation, p, seed, offset, counter, dtype, out, out_values,
                                                  out_scales, pre_values, pre_scales, workspace, workspace_bytes,
                                                  stream)


def afno_mx8_linear_backward(g, x_values, x_scales, w, pre_values, pre_scales, M, K, N, activation, p, seed, offset,
                             counter, dtype, dx, dw, db, workspace, workspace_bytes, stream) -> int:
    return load_library().afno_mx8_linear_backward(g, x_values, x_scales, w, pre_values, pre_scales, M, K, N,
                                                   activation, p, seed, offset, counter, dtype, dx, dw, db,
                                                   workspace, workspace_bytes, stream)


def afno_rms_norm_backward_workspace(M, C, dtype) -> int:
    """Bytes of workspace that the call may need, or a (negative) error code."""
    return load_library().afno_rms_norm_backward_workspace(M, C, dtype)


def afno_mx8_linear_forward_workspace(M, K, N, dtype) -> int:
    return load_library().afno_mx8_linear_forward_workspace(M, K, N, dtype)


def afno_mx8_linear_backward_workspace(M, K, N, dtype, aligned) -> int:
    return load_library().afno_mx8_linear_backward_workspace(M, K, N, dtype, aligned)


# ---------------------------------------------------------------- torch-level wrappers


class Mx8(NamedTuple):
    """Rows of ``channels`` channels in eight bits: values float8_e4m3fn [..., 32 blocks], zeros behind the
    channels, and scales float8_e8m0fnu [..., blocks], a power of two for each 32 channels."""
    values: object
    scales: object
    channels: int

    @property
    def shape(self):
        return (*self.values.shape[:-1], self.channels)


def mx8_empty(shape, device) -> Mx8:
    """Uninitialised room for a tensor of this shape in eight bits."""
    import torch
    *lead, C = shape
    blocks = -(-C // BLOCK)
    return Mx8(torch.empty((*lead, BLOCK * blocks), dtype=torch.float8_e4m3fn, device=device),
               torch.empty((*lead, blocks), dtype=torch.float8_e8m0fnu, device=device), C)


def _new8(like, lead, C) -> Mx8:
    """mx8_empty on the device of a tensor."""
    import torch
    blocks = -(-C // BLOCK)
    return Mx8(like.new_empty((*lead, BLOCK * blocks), dtype=torch.float8_e4m3fn),
               like.new_empty((*lead, blocks), dtype=torch.float8_e8m0fnu), C)


def _fit8(t, lead, C, device) -> bool:
    """Whether _expect8 would pass an Mx8 (or None): the quick check, as train.py's _fit."""
    import torch
    if t is None:
        return True
    if type(t) is not Mx8 or t.channels != C or C < 1:
        return False
    values, scales, _ = t
    blocks = -(-C // BLOCK)
    return (values.shape == (*lead, BLOCK * blocks) and scales.shape == (*lead, blocks)
            and values.dtype is torch.float8_e4m3fn and scales.dtype is torch.float8_e8m0fnu
            and values.device == device and scales.device == device and values.is_cuda
            and values.is_contiguous() and scales.is_contiguous())


def _expect8(name, t, shape, device):
    """Checks, before any GPU call, that t holds a tensor of this shape in eight bits on the device."""
    import torch
    if t is None:
        raise ValueError(f"{name} is missing")
    if not isinstance(t, Mx8):
        raise TypeError(f"{name} must be an Mx8")
    values, scales, C = t
    if values.dtype != torch.float8_e4m3fn or scales.dtype != torch.float8_e8m0fnu:
        raise TypeError(f"{name} must have float8_e4m3fn values and float8_e8m0fnu scales")
    if C < 1:
        raise ValueError(f"{name} has no channels")
    if C != shape[-1]:
        raise ValueError(f"{name} has {C} channels, expected {shape[-1]}")
    blocks = -(-C // BLOCK)
    if values.shape != (*shape[:-1], BLOCK * blocks) or scales.shape != (*shape[:-1], blocks):
        raise ValueError(f"{name} has values {tuple(values.shape)} and scales {tuple(scales.shape)}, expected those of "
                         f"{tuple(shape)}")
    if values.device != device or scales.device != device:
        raise ValueError(f"{name} is on {values.device}, x on {device}")
    if not (values.is_contiguous() and scales.is_contiguous()):
        raise ValueError(f"{name} must be contiguous")
    if not values.is_cuda:
        raise ValueError("tensors must be on the GPU")


def _code(dtype) -> int:
    import torch
    if dtype == torch.bfloat16:
        return AFNO_DTYPE_BF16
    if dtype == torch.float32:
        return AFNO_DTYPE_FP32
    raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")


def _addresses8(t):
    return (None, None) if t is None else (_address(t.values), _address(t.scales))


def _tensors8(*ts):
    return [v for t in ts if t is not None for v in (t.values, t.scales)]


def _shape8(name, t):
    if t is None:
        raise ValueError(f"{name} is missing")
    if not isinstance(t, Mx8):
        raise TypeError(f"{name} must be an Mx8")
    if t.values.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    return t.shape


def mx8_pack(x, *, out=None, stream=None) -> Mx8:
    """x [..., C] in eight bits (out: an Mx8 of that shape that receives them).  Weights w [K, N] go in as
    mx8_pack(w.t().contiguous())."""
    M, C, code = _rows("x", x)
    shape = x.shape
    if not _fit(x):
        _expect(x, [])
    if not _fit8(out, shape[:-1], C, x.device):
        _expect8("out", out, shape, x.device)

    def call(handle):
        y = _new8(x, shape[:-1], C) if out is None else out
        _check(afno_mx8_pack(_address(x), M, C, code, *_addresses8(y), handle))
        return y

    return _launch(x, stream, (x, *_tensors8(out)), call)


def mx8_unpack(x: Mx8, *, dtype=None, out=None, stream=None):
    """The values that x stands for as a tensor of dtype (default: out's, else bfloat16; exact in float32 and
    bfloat16)."""
    import torch
    shape = _shape8("x", x)
    values = x.values
    if not _fit8(x, shape[:-1], shape[-1], values.device):
        _expect8("x", x, shape, values.device)
    if dtype is None:
        dtype = torch.bfloat16 if out is None else out.dtype
    if out is not None:
        _expect(values, [("out", out, shape, dtype)])
    code = _code(dtype)
    M = x.scales.numel() // x.scales.shape[-1]

    def call(handle):
        y = values.new_empty(shape, dtype=dtype) if out is None else out
        _check(afno_mx8_unpack(*_addresses8(x), M, shape[-1], code, _address(y), handle))
        return y

    return _launch(values, stream, (*_tensors8(x), out), call)


def rms_norm_forward(x, gamma, *, eps=1e-6, residual=None, out=None, sum_out=None, out8=None, stream=None):
    """The root-mean-square norm over the last axis of v = x + residual (rounded to x's dtype; None: v = x):
    v / sqrt(mean(v^2) + eps) * gamma.  sum_out: a tensor like x that receives v, the residual stream and what
    rms_norm_backward takes.  out8: an Mx8 (mx8_empty) that receives the result in eight bits; with it and
    without out, nothing is written in x's dtype and out8 is what the call returns."""
    M, C, code = _rows("x", x)
    shape = x.shape
    if gamma is None or not _fit(x, (gamma, (C,)), (residual, shape), (out, shape), (sum_out, shape)):
        _expect(x, [("gamma", gamma, (C,), None)] + [
            (n, t, tuple(shape), None) for n, t in (("residual", residual), ("out", out), ("sum_out", sum_out))
            if t is not None])
    if not _fit8(out8, shape[:-1], C, x.device):
        _expect8("out8", out8, shape, x.device)

    def call(handle):
        y = x.new_empty(shape) if out is None and out8 is None else out
        _check(afno_rms_norm_forward(_address(x), _address(residual), _address(gamma), M, C, eps, code, _address(y),
                                     _address(sum_out), *_addresses8(out8), handle))
        return out8 if y is None else y

    return _launch(x, stream, (x, gamma, residual, out, sum_out, *_tensors8(out8)), call)


def rms_norm_backward(g, x, gamma, *, eps=1e-6, gsum=None, stream=None):
    """Gradients of the norm of x (the v that the forward call stored) for g = dL/dout: a dict with dx (x's
    dtype; gsum, the gradient that reaches v along the residual stream, is added to it) and dgamma (float32)."""
    import torch
    M, C, code = _rows("x", x)
    shape = x.shape
    if gamma is None or g is None or not _fit(x, (gamma, (C,)), (g, shape), (gsum, shape)):
        _expect(x, [("gamma", gamma, (C,), None), ("g", g, tuple(shape), None)] + (
            [] if gsum is None else [("gsum", gsum, tuple(shape), None)]))

    def call(handle):
        dx, dgamma = x.new_empty(shape), x.new_empty(C, dtype=torch.float32)
        ws, nbytes, _held = _workspace(x, _bytes(afno_rms_norm_backward_workspace, M, C, code))
        _check(afno_rms_norm_backward(_address(g), _address(x), _address(gamma), _address(gsum), M, C, eps, code,
                                      _address(dx), _address(dgamma), ws, nbytes, handle))
        return {"dx": dx, "dgamma": dgamma}

    return _launch(x, stream, (g, x, gamma, gsum), call)


def mx8_linear_forward(x: Mx8, w: Mx8, b=None, *, activation="none", residual=None, p=0.0, seed=0, offset=0, counter=None,
                       dtype=None, out=None, out8=None, pre8=None, stream=None):
    """out = drop(act(x w^T + b)) + residual for x [..., K] and w [N, K] in eight bits (w is output-major), b [N]
    or None, residual and out [..., N] of dtype (default: theirs, else bfloat16).  out8: an Mx8 (mx8_empty) that receives
    the result in eight bits; with it and without out, nothing is written in dtype and out8 is what the call
    returns.  pre8: an Mx8 that receives x w^T + b, which mx8_linear_backward takes where there is an
    activation.  activation and dropout as in linear_forward."""
    import torch
    *lead, K = _shape8("x", x)
    if w is None or len(_shape8("w", w)) != 2:
        raise ValueError("w must be an Mx8 of [N, K]")
    values, N = x.values, w.values.shape[0]
    shape, device = (*lead, N), values.device
    if not (_fit8(x, lead, K, device) and _fit8(w, (N,), K, device) and _fit8(out8, lead, N, device)
            and _fit8(pre8, lead, N, device)):
        _expect8("x", x, (*lead, K), device)
        _expect8("w", w, (N, K), device)
        for n, t in (("out8", out8), ("pre8", pre8)):
            if t is not None:
                _expect8(n, t, shape, device)
    if dtype is None:
        dtype = next((t.dtype for t in (out, b, residual) if t is not None), torch.bfloat16)
    code = _code(dtype)
    for n, t, s in (("b", b, (N,)), ("residual", residual, shape), ("out", out, shape)):
        if t is not None and (t.shape != s or t.dtype != dtype or t.device != device or not t.is_contiguous()):
            _expect(values, [(n, t, s, dtype)])
    act, drop = _activation(activation), _random(values, p, seed, offset, counter)
    M = x.scales.numel() // x.scales.shape[-1]

    def call(handle):
        y = values.new_empty(shape, dtype=dtype) if out is None and out8 is None else out
        ws, nbytes, _held = _workspace(values, _bytes(afno_mx8_linear_forward_workspace, M, K, N, code))
        _check(afno_mx8_linear_forward(*_addresses8(x), *_addresses8(w), _address(b), _address(residual), M, K, N, act,
                                       *drop, code, _address(y), *_addresses8(out8), *_addresses8(pre8), ws, nbytes,
                                       handle))
        return out8 if y is None else y

    return _launch(values, stream, (*_tensors8(x, w, out8, pre8), b, residual, out, counter), call)


def mx8_linear_backward(g, x: Mx8, w, *, pre8=None, activation="none", p=0.0, seed=0, offset=0, counter=None, bias=True,
                        need_dx=True, need_dw=True, stream=None):
    """Gradients of drop(act(x w + b)) for g = dL/dout [..., N] from x [..., K] and, where there is an activation,
    pre8 [..., N] = x w + b as they were kept in eight bits: a dict as linear_backward's, of the dtype of g and
    w [K, N] (as linear_forward's).  ReLU passes on 0 where pre8 is not above 0, whatever g is there."""
    *lead, K = _shape8("x", x)
    if w is None or w.dim() != 2:
        raise ValueError("w must be [K, N]")
    if g is None:
        raise ValueError("g is missing")
    code, N = _dtype_code(g), w.shape[1]
    act = _activation(activation)
    shape = (*lead, N)
    if act == AFNO_ACT_NONE:
        pre8 = None  # not read
    if N == 0:
        raise ValueError("w has no columns")
    if g.shape != shape or not _fit(g, (w, (K, N))):
        _expect(g, [("g", g, shape, None), ("w", w, (K, N), None)])
    if not _fit8(x, lead, K, g.device):
        _expect8("x", x, (*lead, K), g.device)
    if act and (pre8 is None or not _fit8(pre8, lead, N, g.device)):
        _expect8("pre8", pre8, shape, g.device)
    if not (bias or need_dx or need_dw):
        raise ValueError("no gradient is asked for")
    drop = _random(g, p, seed, offset, counter)
    M = x.scales.numel() // x.scales.shape[-1]

    def call(handle):
        dx = g.new_empty((*lead, K)) if need_dx else None
        dw = g.new_empty((K, N)) if need_dw else None
        db = g.new_empty(N) if bias else None
        pg, pw = _address(g), _address(w)
        ws, nbytes, _held = _workspace(g, _bytes(afno_mx8_linear_backward_workspace, M, K, N, code, _aligned(pg, pw)))
        _check(afno_mx8_linear_backward(pg, *_addresses8(x), pw, *_addresses8(pre8), M, K, N, act, *drop, code,
                                        _address(dx), _address(dw), _address(db), ws, nbytes, handle))
        return {"dx": dx, "dw": dw, "db": db}

    return _launch(g, stream, (g, w, counter, *_tensors8(x, pre8)), call)

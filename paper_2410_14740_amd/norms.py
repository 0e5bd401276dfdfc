"""The residual stream between a layer's blocks, on torch tensors.

`residual_norm` adds a block's output to the residual stream, normed before and
gated where the layer asks for it, and norms the result for the next block, in
one pass of libm2c.so (include/m2c.h has the definition). Calls enqueue on
`stream` (default: torch's current stream) and return, as those of attention.py."""
from __future__ import annotations

import torch

from . import m2c
from .attention import _address, _alloc, _bad, _check, _raw

_DTYPES = {torch.float16: m2c.DTYPE_FP16, torch.bfloat16: m2c.DTYPE_BF16, torch.float32: m2c.DTYPE_FP32}
_KINDS = {"rms": m2c.NORM_RMS, "layer": m2c.NORM_LAYER}


def _matrix(name, t, shape, device):
    """Row stride of t [rows][d] (a single row's is free)."""
    if t.shape != shape or t.dtype not in _DTYPES or t.device != device:
        _bad(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, need fp16, bf16 or fp32 {tuple(shape)} on {device}")
    a, b = t.stride()
    if b != 1 and shape[1] > 1:
        _bad(f"{name}: the elements of a row must be contiguous")
    return a if shape[0] > 1 else shape[1]


def _empty(x, dtype, stream):
    """Rows like x, contiguous (the usual case by the shorter call)."""
    if stream is None and x.is_contiguous():
        return torch.empty_like(x, dtype=dtype)
    return _alloc(stream, x.device, (x.shape, dtype))[0]


def _vector(name, t, d, dtype, device):
    if t is None:
        return None
    if (t.shape != (d,) or t.dtype != dtype or t.device != device or not t.is_contiguous()):
        _bad(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, need a contiguous {dtype} ({d},) on {device}")
    return t.data_ptr()


def residual_norm(x, y=None, weight=None, bias=None, *, post=False, post_weight=None, post_bias=None, gate=None,
                  scale=1.0, kind="rms", eps=1e-5, x_out=None, out=None, out_dtype=None, norm=True, stream=None):
    """x [rows, d]: the residual stream; y [rows, d]: a block's output, or None.

    t = N(y) post_weight + post_bias with `post`, y without; r = x + scale gate t;
    out = N(r) weight + bias, N the norm of `kind` ("rms" or "layer": mean taken
    off as well). Any row strides; x, y, out fp32 or one 16-bit type; weight, bias,
    post_weight, post_bias [d] and gate [d] or [rows, d] of one type, fp32 or that
    16-bit type; None for ones and zeros.
    Returns (r, out): r in x's type, in x_out (which may be x; allocated if not
    given; x itself where y is None), out in `out` (allocated if not given, in
    out_dtype, by default y's type, x's or, where those are fp32, fp16). norm False:
    out is None."""
    if x.dim() != 2 or x.dtype not in _DTYPES or not x.is_cuda:
        _bad("x: need an fp16, bf16 or fp32 GPU tensor [rows, d]")
    if kind not in _KINDS:
        _bad(f"kind {kind!r}: need 'rms' or 'layer'")
    dev, shape, d = x.device, x.shape, x.shape[1]
    wt = torch.float32
    for t in (weight, bias, post_weight, post_bias, gate):
        if t is not None:
            wt = t.dtype
            break
    if wt not in _DTYPES:
        _bad(f"weights: {wt}, need fp16, bf16 or fp32")
    xs, ys, gs = _matrix("x", x, shape, dev), 0, 0
    if y is not None:
        ys = _matrix("y", y, shape, dev)
    if gate is not None:
        if gate.dim() == 2:
            gs = _matrix("gate", gate, shape, dev)
            if gate.dtype != wt:
                _bad(f"gate: {gate.dtype}, the other weights are {wt}")
        else:
            _vector("gate", gate, d, wt, dev)
    if x_out is None:
        r = x if y is None else _empty(x, x.dtype, stream)
    else:
        r = x_out
        if r.dtype != x.dtype:
            _bad(f"x_out: {r.dtype}, x is {x.dtype}")
    rs = _matrix("x_out", r, shape, dev)
    if not norm:
        if out is not None or weight is not None or bias is not None:
            _bad("norm False: out, weight and bias have no use")
        if r is x and y is None:
            return x, None
    elif out is None:
        if out_dtype is None:
            out_dtype = y.dtype if y is not None and y.dtype != torch.float32 else x.dtype
            if out_dtype == torch.float32:
                out_dtype = torch.float16
        if out_dtype not in _DTYPES:
            _bad(f"out_dtype {out_dtype}: need fp16, bf16 or fp32")
        out = _empty(x, out_dtype, stream)
    elif out_dtype is not None and out.dtype != out_dtype:
        _bad(f"out: {out.dtype}, out_dtype is {out_dtype}")
    os = _matrix("out", out, shape, dev) if out is not None else 0
    desc = m2c.NormDesc(_KINDS[kind], 1 if post else 0, d, dev.index, _DTYPES[x.dtype],
                        _DTYPES[y.dtype] if y is not None else 0, _DTYPES[out.dtype] if out is not None else 0,
                        _DTYPES[wt], eps, scale, xs, ys, rs, os, gs, _vector("weight", weight, d, wt, dev),
                        _vector("bias", bias, d, wt, dev), _vector("post_weight", post_weight, d, wt, dev),
                        _vector("post_bias", post_bias, d, wt, dev), _address(gate))
    _check(m2c.load().m2c_residual_norm(desc, x.data_ptr(), _address(y), shape[0],
                                        None if r is x and y is None else r.data_ptr(), _address(out),
                                        _raw(stream, dev)))
    return r, out

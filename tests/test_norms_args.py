"""The residual norm's argument checks (no GPU is touched)."""
import os

import pytest
import torch

from paper_2410_14740_amd import m2c, norms

P = 1 << 20  # an aligned address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(m2c.LIB_PATH):
        from paper_2410_14740_amd import build
        build.build()
    return m2c.load()


def desc(**kw):
    d = m2c.NormDesc(m2c.NORM_RMS, 0, 64, 0, m2c.DTYPE_FP32, m2c.DTYPE_FP16, m2c.DTYPE_FP16, m2c.DTYPE_FP32,
                     1e-5, 1.0, 64, 64, 64, 64, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


REFUSED = [
    (dict(kind=2), {}, "kind"), (dict(post=2), {}, "post"), (dict(d=0), {}, "d 0"), (dict(d=65537), {}, "d 65537"),
    (dict(device=-1), {}, "device"), (dict(eps=-1.0), {}, "eps"), (dict(eps=float("nan")), {}, "eps"),
    (dict(eps=float("inf")), {}, "eps"), (dict(scale=float("nan")), {}, "scale"), (dict(scale=float("-inf")), {}, "scale"),
    ({}, dict(rows=-1), "rows"), ({}, dict(rows=(1 << 30) + 1), "rows"), ({}, dict(x=None), "x: NULL"),
    ({}, dict(x_out=None, out=None), "nothing"), (dict(post=1), dict(y=None), "y is NULL"),
    (dict(gate=P), dict(y=None), "y is NULL"), (dict(post_weight=P), {}, "need post"), (dict(post_bias=P), {}, "need post"),
    (dict(x_dtype=3), {}, "x: dtype"), (dict(y_dtype=-1), {}, "y: dtype"), (dict(out_dtype=m2c.DTYPE_BF16), {}, "16-bit"),
    (dict(weight_dtype=m2c.DTYPE_BF16, weight=P), {}, "16-bit"), (dict(weight_dtype=9, bias=P), {}, "bias: dtype"),
    ({}, dict(x=P + 2), "x: not aligned"), ({}, dict(y=P + 1), "y: not aligned"), (dict(weight=P + 2), {}, "weight: not"),
    (dict(x_stride=-64), {}, "x: stride"), (dict(y_stride=(1 << 40) + 1), {}, "y: stride"),
    (dict(x_out_stride=63), {}, "x_out: stride"), (dict(out_stride=0), {}, "out: stride"),
    (dict(gate=P, gate_stride=-1), {}, "gate: stride"), (dict(x_out_stride=72), dict(x_out=P), "other strides"),
]


@pytest.mark.parametrize("fields,args,needle", REFUSED)
def test_refusals(lib, fields, args, needle):
    a = dict(x=P, y=2 * P, rows=3, x_out=3 * P, out=4 * P) | args
    with pytest.raises(m2c.M2CError) as e:
        m2c.m2c_residual_norm(desc(**fields), a["x"], a["y"], a["rows"], a["x_out"], a["out"], 0)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_nothing_to_do(lib):
    m2c.m2c_residual_norm(desc(), None, None, 0, None, P, 0)
    assert lib.m2c_residual_norm(None, P, P, 1, P, P, None) == m2c.M2C_ERR_INVALID_ARG


def test_host_tensors_are_refused():
    x = torch.zeros((2, 8))
    with pytest.raises(m2c.M2CError) as e:
        norms.residual_norm(x)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "GPU" in str(e.value)

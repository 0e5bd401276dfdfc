"""Argument checks of the rotation and of the append that rotates (no GPU is touched)."""
import os

import pytest
import torch

from paper_2410_14740_amd import attention, m2c

P = 1 << 20  # an aligned address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(m2c.LIB_PATH):
        from paper_2410_14740_amd import build
        build.build()
    return m2c.load()


def rotary(**kw):
    r = m2c.RotaryDesc(64, 0, 2, (m2c.ctypes.c_int32 * 4)(20, 12, 0, 0), 1.0, P)
    for k, v in kw.items():
        setattr(r, k, (m2c.ctypes.c_int32 * 4)(*v) if k == "section" else v)
    return r


def cache(**kw):
    c = m2c.KvCacheDesc(m2c.DTYPE_BF16, 4, 2, 128, 64, 16, 0, 0, 128, *[P] * 11)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


ROTARIES = [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=24, section=(12, 0, 0, 0)), "rot_dim"), (dict(rot_dim=144, section=(60, 12, 0, 0)), "rot_dim"),
    (dict(interleaved=2), "interleaved"), (dict(n_axes=0), "n_axes"), (dict(n_axes=5), "n_axes"),
    (dict(section=(20, 13, 0, 0)), "section"), (dict(section=(40, -8, 0, 0)), "section[1]"), (dict(section=(20, 0, 12, 0)), "section[2]"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(freq=None), "NULL"),
]
S = (1024, 128)


def rotate(r=None, dtype=0, dim=128, device=0, total=4, positions=P, stride=4, hq=8, q=P, qs=S, qo=2 * P, qos=S, hk=2, k=3 * P,
           ks=S, ko=4 * P, kos=S):
    m2c.m2c_rotate(r or rotary(), dtype, dim, device, total, positions, stride, hq, q, qs, qo, qos, hk, k, ks, ko, kos, 0)


def append(c=None, r=None, n=2, cu=None, total=2, positions=P, stride=2, k=P, v=P, ks=S, ko=None, kos=(0, 0), hq=8, q=2 * P, qs=S,
           qo=3 * P, qos=S):
    m2c.m2c_kv_append_rotated(c or cache(), r or rotary(), None, n, cu, total, None, positions, stride, k, v, ks, S, ko, kos, hq, q, qs,
                              qo, qos, 0)


@pytest.mark.parametrize("fields,needle", ROTARIES)
@pytest.mark.parametrize("call", [rotate, append])
def test_rotary_refusals(lib, call, fields, needle):
    with pytest.raises(m2c.M2CError) as e:
        call(r=rotary(**fields))
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


@pytest.mark.parametrize("kw,needle", [
    (dict(dtype=2), "dtype"), (dict(dim=96), "head_dim"), (dict(device=-1), "device"), (dict(total=-1), "total"),
    (dict(total=(1 << 30) + 1), "total"), (dict(positions=None), "NULL"), (dict(stride=3), "pos_stride"), (dict(hq=0), "heads"),
    (dict(hq=1025), "heads"), (dict(q=None), "q: NULL"), (dict(q=P + 8), "q: not"), (dict(qs=(1024, 4)), "q: stride"), (dict(qs=(64, 8)), "q: token"),
    (dict(qo=None), "q_out: NULL"), (dict(qos=(512, 128)), "overlap"), (dict(qos=(1024, 64)), "head stride"),
    (dict(qo=P, qos=(2048, 128)), "other strides"), (dict(k=None), "n_kv_heads 2"), (dict(k=None, hk=0), "k_out"), (dict(hk=0), "k: 0 heads"),
    (dict(ko=3 * P, kos=(1024, 256)), "other strides"),
])
def test_rotate_refusals(lib, kw, needle):
    with pytest.raises(m2c.M2CError) as e:
        rotate(**kw)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


@pytest.mark.parametrize("kw,needle", [
    (dict(c=cache(block_tokens=16)), "block_tokens"), (dict(n=5, total=5), "n 5"), (dict(total=3, stride=3), "total"), (dict(total=-1), "total"),
    (dict(stride=1), "pos_stride"), (dict(k=None), "k: NULL"), (dict(v=P + 2), "v: not"), (dict(ks=(1024, 100)), "k: stride"),
    (dict(ko=P, kos=S), "k_out is k"), (dict(ko=5 * P, kos=(128, 128)), "k_out: rows overlap"), (dict(hq=0), "0 heads"),
    (dict(q=None), "n_heads 8"), (dict(q=None, hq=0), "q_out"), (dict(qo=None), "q_out: NULL"), (dict(qo=2 * P, qos=(4096, 128)), "other strides"),
])
def test_append_refusals(lib, kw, needle):
    with pytest.raises(m2c.M2CError) as e:
        append(**kw)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_nothing_to_do(lib):
    rotate(total=0, q=None, positions=None)
    append(cu=P, total=0, positions=None, k=None)
    assert lib.m2c_rotate(None, 0, 128, 0, 4, P, 4, 8, P, m2c._I64x2(*S), P, m2c._I64x2(*S), 0, None, m2c._I64x2(0, 0), None,
                          m2c._I64x2(0, 0), None) == m2c.M2C_ERR_INVALID_ARG


def test_frequencies_on_the_host_are_refused():
    with pytest.raises(m2c.M2CError) as e:
        attention.Rotary(torch.ones(32))
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "freq" in str(e.value)

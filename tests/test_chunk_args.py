"""Argument checks of the attention of chunks over the cache (no GPU is touched)."""
import os

import pytest

from paper_2410_14740_amd import m2c

P = 1 << 20  # an aligned address that no refused call reads
S, T = (1024, 128), (256, 128)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(m2c.LIB_PATH):
        from paper_2410_14740_amd import build
        build.build()
    return m2c.load()


def cache(**kw):
    c = m2c.KvCacheDesc(m2c.DTYPE_BF16, 4, 2, 128, 64, 16, 0, 0, 128, *[P] * 11)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def chunk(c=None, n=2, cu=P, total=6, hq=8, scale=0.0, q=P, qs=S, k=P, ks=T, v=P, vs=T, out=2 * P, os=S, max_q=0, max_len=0, ws=None, wsb=0):
    m2c.m2c_kv_attend_chunk(c or cache(), None, n, cu, total, hq, scale, q, qs, k, ks, v, vs, out, os, None, max_q, max_len, ws, wsb, 0)


@pytest.mark.parametrize("kw,needle", [
    (dict(c=cache(block_tokens=16)), "block_tokens"), (dict(c=cache(tail_k=None)), "NULL"), (dict(n=0), "n 0"), (dict(n=65536), "n 65536"),
    (dict(cu=None), "cu"), (dict(total=-1), "total"), (dict(total=(1 << 30) + 1), "total"), (dict(hq=7), "n_heads"), (dict(hq=2048), "n_heads"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(q=None), "q: NULL"), (dict(q=P + 2), "q: not"),
    (dict(qs=(1020, 128)), "q: stride"), (dict(k=None), "both"), (dict(v=None), "both"), (dict(ks=(64, 128)), "k: token"), (dict(v=P + 8), "v: not"),
    (dict(vs=(256, -8)), "v: stride"), (dict(out=None), "out: NULL"), (dict(os=(512, 128)), "overlap"), (dict(os=(1024, 64)), "head stride"),
    (dict(max_q=-1), "max_q -1"), (dict(max_len=-2), "max_len -2"), (dict(ws=P + 64, wsb=1 << 40), "aligned"),
])
def test_refusals(lib, kw, needle):
    with pytest.raises(m2c.M2CError) as e:
        chunk(**kw)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_nothing_to_do(lib):
    chunk(total=0, q=None, out=None)
    assert lib.m2c_kv_attend_chunk_workspace(None, 1, 1, 8, 0, 0) == -1


def test_workspace(lib):
    """Room for parts of rows where some may see many more keys than others."""
    need = lambda c, n, total, hq=8, q=0, most=0: m2c.m2c_kv_attend_chunk_workspace(c, n, total, hq, q, most)  # noqa: E731
    c = cache(max_blocks=2048, n_pages=1 << 14)
    assert need(c, 4, 40, q=10, most=300) == 0    # no row is long
    assert need(c, 65, 9000) == 0                 # more sequences than lanes
    assert need(c, 1, 0) == 0
    long = need(c, 2, 10, q=5, most=131072)
    assert long >= 2 * 8 * 128 * (128 + 2) * 4 and need(c, 2, 10) == long  # the capacity where no length is known
    assert need(c, 1, 60000, hq=64) == 0          # a single sequence of enough rows
    assert need(c, 60, 1 << 20, hq=64) <= (2 * 1024 * 128) * (128 * 4 + 8) + 512
    with pytest.raises(m2c.M2CError) as e:
        chunk(c=c, n=1, total=5, ws=P, wsb=4096)
    assert e.value.status == m2c.M2C_ERR_CAPACITY and "workspace" in str(e.value)
    with pytest.raises(m2c.M2CError) as e:
        need(c, 1, 5, q=-1)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "max_q" in str(e.value)

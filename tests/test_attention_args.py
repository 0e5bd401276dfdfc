"""The attention entry points' host-side argument checks (no GPU is touched)."""
import ctypes
import os

import pytest

from paper_2410_14740_amd import m2c

P = 1 << 20  # an aligned address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(m2c.LIB_PATH):
        from paper_2410_14740_amd import build
        build.build()
    return m2c.load()


def desc(**kw):
    d = m2c.AttnDesc(m2c.DTYPE_FP16, 8, 2, 128, 1, 0, 0.0, 0)
    for name in ("q_stride", "k_stride", "v_stride", "out_stride"):
        setattr(d, name, (1024, 128))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def prompt(d=None, q=P, k=P, v=P, cu_q=P, cu_k=P, n=1, tq=4, tk=4, out=P):
    m2c.m2c_prompt_attention(desc() if d is None else d, q, k, v, cu_q, cu_k, n, tq, tk, out, None, 0)


@pytest.mark.parametrize("kw,needle", [
    (dict(d=desc(dtype=2)), "dtype"), (dict(d=desc(n_heads=7)), "n_heads"), (dict(d=desc(n_kv_heads=0)), "n_kv_heads"),
    (dict(d=desc(n_heads=2048, n_kv_heads=2)), "n_heads"), (dict(d=desc(head_dim=96)), "head_dim"),
    (dict(d=desc(causal=2)), "causal"), (dict(d=desc(scale=-1.0)), "scale"), (dict(d=desc(scale=float("nan"))), "scale"),
    (dict(d=desc(scale=float("inf"))), "scale"), (dict(d=desc(device=-1)), "device"),
    (dict(d=desc(q_stride=(1020, 128))), "q: stride"), (dict(d=desc(k_stride=(1024, -128))), "k: stride"),
    (dict(d=desc(out_stride=(1024, 4))), "out: stride"), (dict(q=P + 8), "q: not"), (dict(v=P + 2), "v: not"),
    (dict(q=None), "q: NULL"), (dict(out=None), "out: NULL"), (dict(k=None), "k: NULL"),
    (dict(cu_q=None), "NULL"), (dict(cu_k=None), "NULL"), (dict(n=0), "n_seqs"), (dict(n=65536), "n_seqs"),
    (dict(tq=-1), "total_q"), (dict(tk=(1 << 30) + 1), "total_k"),
])
def test_prompt_refuses(lib, kw, needle):
    with pytest.raises(m2c.M2CError) as e:
        prompt(**kw)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_prompt_without_rows_is_nothing(lib):
    prompt(tq=0, q=None, out=None)


def cache(**kw):
    c = m2c.KvCacheDesc(m2c.DTYPE_BF16, 4, 2, 128, 64, 16, 0, 0, 128, *[P] * 11)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


CACHES = [
    (dict(dtype=5), "dtype"), (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=70000), "n_seqs"), (dict(n_kv_heads=0), "n_kv_heads"),
    (dict(head_dim=32), "head_dim"), (dict(block_tokens=16), "block_tokens"), (dict(block_tokens=96), "block_tokens"),
    (dict(max_blocks=0), "max_blocks"), (dict(max_blocks=16385), "max_blocks"), (dict(n_pages=0), "n_pages"),
    (dict(n_pages=1 << 31), "n_pages"), (dict(reserved=1), "reserved"), (dict(device=-2), "device"),
    (dict(k_codes=None), "NULL"), (dict(status=None), "NULL"), (dict(tail_v=P + 8), "alignment"),
]


@pytest.mark.parametrize("kw,needle", CACHES)
def test_cache_refusals(lib, kw, needle):
    c = cache(**kw)
    calls = [lambda: m2c.m2c_kv_reset(c, None, 1, 0),
             lambda: m2c.m2c_kv_append(c, None, 1, None, 1, None, P, P, (256, 128), (256, 128), 0),
             lambda: m2c.m2c_kv_read(c, None, 1, P, 1, P, P, (256, 128), (256, 128), 0),
             lambda: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 0, 64, P, 1 << 30, 0),
             lambda: m2c.m2c_kv_evict(c, None, 1, 1, 0, 0, None, None, None, 0),
             lambda: m2c.m2c_kv_status(c, 0),
             lambda: m2c.m2c_kv_attend_workspace(c, 1, 8, 0, 64)]
    for f in calls:
        with pytest.raises(m2c.M2CError) as e:
            f()
        assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


@pytest.mark.parametrize("call,status,needle", [
    (lambda c: m2c.m2c_kv_reset(c, None, 5, 0), m2c.M2C_ERR_INVALID_ARG, "n 5"),
    (lambda c: m2c.m2c_kv_append(c, None, 0, None, 0, None, P, P, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "n 0"),
    (lambda c: m2c.m2c_kv_append(c, None, 2, None, 3, None, P, P, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "total"),
    (lambda c: m2c.m2c_kv_append(c, None, 2, P, -1, None, P, P, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "total"),
    (lambda c: m2c.m2c_kv_append(c, None, 1, None, 1, None, P, P + 4, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "v: not"),
    (lambda c: m2c.m2c_kv_append(c, None, 1, None, 1, None, P, P, (256, 100), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "k: stride"),
    (lambda c: m2c.m2c_kv_read(c, None, 1, None, 1, P, P, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "cu"),
    (lambda c: m2c.m2c_kv_read(c, None, 1, P, 1, None, P, (256, 128), (256, 128), 0), m2c.M2C_ERR_INVALID_ARG, "k: NULL"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 7, 0.0, P, (1024, 128), P, (1024, 128), None, 0, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "n_heads"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, -0.5, P, (1024, 128), P, (1024, 128), None, 0, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "scale"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 2, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "track"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 0, -1, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "max_len"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 1, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "workspace"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 1, 64, P, 8, 0), m2c.M2C_ERR_CAPACITY, "workspace"),
    (lambda c: m2c.m2c_kv_attend(c, None, 1, 8, 0.0, P, (1024, 128), P, (1024, 128), None, 1, 64, P + 64, 1 << 30, 0), m2c.M2C_ERR_INVALID_ARG, "aligned"),
    (lambda c: m2c.m2c_kv_attend(c, None, 2, 8, 0.0, P, (1024, 128), P, (1024, 0), None, 0, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "out: "),
    (lambda c: m2c.m2c_kv_attend(c, None, 2, 8, 0.0, P, (1024, 128), P, (512, 128), None, 0, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "out: rows overlap"),
    (lambda c: m2c.m2c_kv_attend(c, None, 2, 8, 0.0, P, (1024, 128), P, (1024, 64), None, 0, 64, None, 0, 0), m2c.M2C_ERR_INVALID_ARG, "out: head stride"),
    (lambda c: m2c.m2c_kv_read(c, None, 1, P, 9, P, P, (256, 128), (128, 128), 0), m2c.M2C_ERR_INVALID_ARG, "v: rows overlap"),
    (lambda c: m2c.m2c_kv_attend_workspace(c, 1, 8, 0, -1), m2c.M2C_ERR_INVALID_ARG, "max_len -1"),
    (lambda c: m2c.m2c_kv_evict(c, None, 1, 3, 2, 2, None, None, None, 0), m2c.M2C_ERR_INVALID_ARG, "keep 3"),
    (lambda c: m2c.m2c_kv_evict(c, None, 1, 3, -1, 2, None, None, None, 0), m2c.M2C_ERR_INVALID_ARG, "first -1"),
    (lambda c: m2c.m2c_kv_evict(c, None, 1, 3, 1, 2, P, None, None, 0), m2c.M2C_ERR_INVALID_ARG, "all three"),
    (lambda c: m2c.m2c_kv_evict(c, None, 1, 3, 1, 2, P, P, P, 0), m2c.M2C_ERR_INVALID_ARG, "own arrays"),
    (lambda c: m2c.m2c_kv_attend_workspace(c, 9, 8, 0, 64), m2c.M2C_ERR_INVALID_ARG, "n 9"),
    (lambda c: m2c.m2c_kv_attend_workspace(c, 1, 3, 0, 64), m2c.M2C_ERR_INVALID_ARG, "n_heads"),
])
def test_call_refusals(lib, call, status, needle):
    with pytest.raises(m2c.M2CError) as e:
        call(cache())
    assert e.value.status == status and needle in str(e.value)


def test_null_cache(lib):
    assert lib.m2c_kv_reset(None, None, 1, None) == m2c.M2C_ERR_INVALID_ARG
    assert lib.m2c_kv_status(None, None) == m2c.M2C_ERR_INVALID_ARG
    assert lib.m2c_kv_attend_workspace(None, 1, 8, 0, 64) == -1
    assert lib.m2c_prompt_attention(None, P, P, P, P, P, 1, 1, 1, P, None, None) == m2c.M2C_ERR_INVALID_ARG


def test_workspace_sizes(lib):
    """Nothing for a sequence that one workgroup takes, partial results where it
    is split, one pair per unit of the capacity and query head where weights
    are tracked."""
    c = cache(max_blocks=16384, n_pages=1 << 20)
    ws = lambda n, track, most: m2c.m2c_kv_attend_workspace(c, n, 8, track, most)
    assert ws(1, 0, 64) == 0
    long = ws(1, 0, 16384 * 64)
    assert long >= 8 * 128 * 4 * 2 and ws(1, 0, 0) == long  # the capacity where no length is known
    assert ws(2, 0, 16384 * 64) >= long
    assert ws(1, 1, 64) >= 8 * 16384 * 8


@pytest.mark.parametrize("max_blocks", [300, 2048, 16384])
def test_workspace_of_many_sequences(lib, max_blocks):
    """Parts of rows, each 8 heads of 128 sums with m and l: at most 16 rounds of
    512 workgroups and two a row, however long a sequence may get."""
    for n in (64, 65, 128, 1000, 65535):
        c = cache(n_seqs=n, n_kv_heads=8, max_blocks=max_blocks)
        for most in (0, 5000):
            need = m2c.m2c_kv_attend_workspace(c, n, 64, 0, most)
            assert need <= (16 * 512 + 2 * 8 * n) * 8 * (128 * 4 + 8) + 512, (n, most)


def test_prompt_workspace(lib):
    """Room for parts of rows where some may see many more keys than others."""
    need = lambda d, same, n, tq, tk: m2c.m2c_prompt_attention_workspace(d, P, P if same else 2 * P, n, tq, tk)  # noqa: E731
    assert need(desc(), True, 1, 500, 500) == 0      # no row is long
    assert need(desc(), False, 65, 9000, 90000) == 0  # more sequences than lanes
    assert need(desc(n_heads=64, n_kv_heads=8, max_q=8192), True, 2, 10000, 10000) == 0  # enough rows
    assert need(desc(), False, 1, 1, 100000) >= 2 * 8 * 128 * (128 + 2) * 4
    assert need(desc(), True, 1, 0, 9000) == 0
    with pytest.raises(m2c.M2CError) as e:
        need(desc(max_q=-1), False, 1, 1, 100000)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "max_q" in str(e.value)
    for kw, status, needle in [(dict(workspace=P + 64, workspace_bytes=1 << 40), m2c.M2C_ERR_INVALID_ARG, "aligned"),
                               (dict(workspace=P, workspace_bytes=4096), m2c.M2C_ERR_CAPACITY, "workspace")]:
        with pytest.raises(m2c.M2CError) as e:
            prompt(d=desc(**kw), cu_k=2 * P, tq=1, tk=100000)
        assert e.value.status == status and needle in str(e.value)

"""Chunks over bf16 caches whose value blocks are of very different sizes, all of
them with weight: outputs are summed in units that follow the sizes. Tolerances are
those of test_gpu_chunk.py."""
import pytest
import torch

from helpers import say
from paper_2410_14740_amd.attention import KVCache
from test_gpu_chunk import check, held64, rand, starts

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
LOG2 = 0.6931471805599453


def cache(d, block, parts):
    """A sequence of `parts`: (blocks, size of the values, score in binary places)."""
    n = sum(p[0] for p in parts) * block
    k = torch.zeros((n, 1, d), dtype=BF16, device="cuda")
    v = rand((n, 1, d), BF16, 2).float().clamp(-1, 1)
    at = 0
    for blocks, size, score in parts:
        rows = slice(at, at + blocks * block)
        k[rows, 0, 0] = score
        v[rows] *= size
        at += blocks * block
    c = KVCache(1, 1, d, n // block + 1, block_tokens=block, dtype=BF16)
    c.append(k, v.to(BF16), cu=starts([n]))
    return c


def queries(m, d):
    q = torch.zeros((m, 1, d), dtype=BF16, device="cuda")
    q[:, 0, 0] = 1.0
    return q


def attend(c, m, d, own=None, **kw):
    """Rows of which each score is what its key's first element says, in binary places."""
    q, scale = queries(m, d), LOG2
    k, v = own if own else (None, None)
    out, lse = c.attend_chunk(q, starts([m]), k, v, scale=scale, return_lse=True, **kw)
    c.check()
    check(c, q, starts([m]), k, v, out, lse, scale=scale)


UP = [
    [(2, 1.0, 0), (2, 2.0 ** 39, 0), (2, 2.0 ** 42, 0)],   # a middle size that the first unit just holds
    [(2, 1.0, 44), (2, 2.0 ** 44, 0)],                     # a small block of large weight before a large one of little
    [(1, 2.0 ** -30, 60), (2, 2.0 ** 11, 19), (1, 2.0 ** 29, 1), (3, 2.0 ** 30, 0)],
    [(1, 2.0 ** -100, 3), (1, 2.0 ** -62, 3), (1, 2.0 ** -20, 3), (1, 2.0 ** 15, 3), (1, 2.0 ** 60, 2)],
    [(3, 0.0, 0), (1, 2.0 ** -40, 50), (1, 2.0 ** 9, 1), (2, 0.0, 7), (1, 2.0 ** 50, -40)],
]


@pytest.mark.parametrize("parts", UP)
@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("d,block", [(64, 32), (128, 64), (128, 128)])
def test_sizes_that_grow(parts, order, d, block):
    say(f"chunk units {parts} {order} {d} {block}")
    if order < 0 and parts is UP[-1]:
        # 2^-40 is less than 2^-80 of 2^50, after which it may count as larger
        parts = [p for p in parts if p[1] != 2.0 ** 50]
    c = cache(d, block, parts[::order])
    attend(c, 1, d)
    attend(c, 40, d)


@pytest.mark.parametrize("size,score", [(2.0 ** 60, 55.0), (2.0 ** 40, 38.0), (2.0 ** -50, -48.0), (2.0 ** 80, 20.0), (2.0 ** 20, 0.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_own_keys_beside_large_blocks(size, score, d):
    """The chunk's own values are about 1, their weights so large that both count."""
    say(f"chunk units beside own {size} {score} {d}")
    c = cache(d, 64, [(3, size, 0.0)])
    m = 33
    k = torch.zeros((m, 1, d), dtype=BF16, device="cuda")
    k[:, 0, 0] = score
    v = rand((m, 1, d), BF16, 9)
    attend(c, m, d, own=(k, v))
    # and with the weights that are subnormal in fp16 bounded by the largest w s of a
    # coded key, or the largest w of another, whose size counts as 1 at most
    q = queries(m, d)
    out = c.attend_chunk(q, starts([m]), k, v, scale=LOG2)
    kk, vv, sizes, codes = held64(c, 0, 0)
    n = kk.shape[0]
    kk, vv = torch.cat([kk, k[:, 0].double()]), torch.cat([vv, v[:, 0].double()])
    x = (q[:, 0].double() @ kk.t()) * LOG2
    x = x.masked_fill(torch.arange(n + m, device="cuda")[None] > n + torch.arange(m, device="cuda")[:, None], -float("inf"))
    w = torch.softmax(x, 1)
    e = 2.0 ** -16 * (1 + x.masked_fill(x.isinf(), 0).abs().amax(1, keepdim=True))
    want, far = w @ vv, torch.maximum((w[:, :n] * sizes).amax(1, keepdim=True), w[:, n:].amax(1, keepdim=True))
    tol = (2.0 ** -11 + e) * (w[:, :n] @ vv[:n].abs()) + (2.0 ** -8 + e) * (w[:, n:] @ vv[n:].abs())
    tol = tol + 2.0 ** -35 * codes * far + 2.0 ** -8 * want.abs()
    bad = float(((out[:, 0].double() - want).abs() / tol).max())
    assert bad <= 1, f"output off by {bad:.2f} of its bound"


@pytest.mark.parametrize("parts", [
    [(70, 1.0, 0), (70, 2.0 ** 39, 0), (70, 2.0 ** 42, 0)], [(100, 1.0, 44), (90, 2.0 ** 44, 0)]])
def test_rows_cut_along_the_keys(parts):
    say(f"chunk units cut {parts}")
    c = cache(64, 32, parts)
    attend(c, 3, 64, max_q=3, max_len=int(c.len[0]))


@pytest.mark.parametrize("parts", [
    [(1, 1.0, -30), (1, 2.0 ** 39, 0), (500, 0.0, -20)], [(1, 1.0, -30), (1, 2.0 ** 30, 0), (500, 0.0, -24)],
    [(1, 1.0, -30), (1, 2.0 ** 39, 0), (500, 2.0 ** -38, -20)]])
@pytest.mark.parametrize("d", [64, 128])
def test_many_small_weights_of_small_blocks(parts, d):
    """16000 keys of weights 2^-20 or 2^-24, whose values are zeros or small, after a
    large block that has the rest: they are 1.5% or 0.1% of the sum of weights."""
    say(f"chunk units small {parts} {d}")
    c = cache(d, 32, parts)
    attend(c, 1, d)
    attend(c, 2, d, max_q=2, max_len=int(c.len[0]))

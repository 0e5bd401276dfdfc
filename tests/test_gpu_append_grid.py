"""Appends of more blocks (tokens / 32 x heads) than one dimension of a grid takes:
2^24 workgroups of 256 threads would be 2^32 threads. All heads share one row of
keys and values, and the first sequence is far too long for the cache, so that
little memory is used."""
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import m2c
from paper_2410_14740_amd.attention import KVCache, Rotary

pytestmark = pytest.mark.gpu

HEADS, D, BLOCK, LAST = 1024, 64, 32, 57
F16 = torch.float16


def rand(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=F16, device="cuda").normal_(generator=g)


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("tokens", [(1 << 19) + 1000, (3 << 19) + 77])
def test_more_blocks_than_a_grid_has_threads(turned, tokens):
    say(f"append grid {turned} {tokens}")
    k, v = (rand((tokens, 1, D), i).expand(tokens, HEADS, D) for i in (1, 2))
    cu = torch.tensor([0, tokens - LAST, tokens], dtype=torch.int32, device="cuda")
    at = torch.arange(tokens, dtype=torch.int32, device="cuda")
    rotary = Rotary(torch.tensor([1e4 ** (-i / 32) for i in range(32)], dtype=torch.float32, device="cuda"))
    c, want = KVCache(2, HEADS, D, 2, BLOCK), KVCache(1, HEADS, D, 2, BLOCK)
    end, place = slice(tokens - LAST, tokens), torch.tensor([0, LAST], dtype=torch.int32, device="cuda")
    if turned:
        q = rand((tokens, 3, D), 3)
        got, _ = c.append_rotated(rotary, k, v, at, q=q, cu=cu)
        for part in (slice(0, 5000), slice(tokens // 2, tokens // 2 + 5000), slice(tokens - 5000, tokens)):
            assert torch.equal(got[part], rotary.rotate(q[part], at[part]))
        want.append_rotated(rotary, k[end], v[end], at[end], cu=place)
    else:
        c.append(k, v, cu=cu)
        want.append(k[end], v[end], cu=place)
    want.check()
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_CAPACITY  # the first sequence, which stays as it was
    assert c.len.tolist() == [0, LAST] and want.len.tolist() == [LAST]
    got = c.read(place, LAST, seqs=torch.tensor([1], dtype=torch.int32, device="cuda"))
    for a, b in zip(got, want.read(place, LAST)):
        assert torch.equal(a, b)

"""Edges of the attention calls. The bounds are those of test_gpu_attention.py."""
import pytest

from helpers import say
from paper_2410_14740_amd.attention import KVCache
from test_gpu_attention import BF16, check_attend, rand, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [192, 200])
@pytest.mark.parametrize("qs,ks,scale", [(1e-34, 1e34, 0.2), (1e-36, 1e36, 0.2), (1e-38, 2e37, 1.0)])
def test_attend_tiny_queries(qs, ks, scale, n):
    """bf16 queries down to the type's subnormal numbers, and keys that give
    them scores of some units."""
    say(f"attend tiny queries {qs} {n}")
    c = KVCache(1, 2, 64, 4, dtype=BF16)
    c.append(rand((n, 2, 64), BF16, 301, ks), rand((n, 2, 64), BF16, 302), cu=starts([n]))
    q = rand((1, 6, 64), BF16, 303, qs)
    out, lse = c.attend(q, scale=scale, return_lse=True)
    check_attend(c, q, out, lse, [0], scale=scale)

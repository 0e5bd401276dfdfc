"""A decoder layer's two ways to attend a later chunk, each against 64 bits.

Over a copy the keys and values are what the cache reads back as, so the reference
is over those. With A the sum of weight times |value|, an output is off by at most
2^-11 A (weights in fp16), 2^-16 (1 + largest |score|) A (scores and exponents in
fp32) and 2^-11 |out|, fp16's smallest number beside it."""
import numpy as np
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import decoder
from paper_2410_14740_amd.attention import KVCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,d,lens,before", [
    (8, 2, 64, [130, 0, 1, 77], [200, 64, 0, 63]), (4, 4, 128, [65, 300], [640, 31]), (16, 1, 64, [5], [1000])])
@pytest.mark.parametrize("back", [False, True])
def test_routes(hq, hk, d, lens, before, back, monkeypatch):
    say(f"chunk routes {hq}/{hk}x{d} {lens} {before} {back}")
    n, T = len(lens), sum(lens)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rand = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda").normal_(generator=g)  # noqa: E731
    layer = object.__new__(decoder.DecoderLayer)
    layer.budget, layer.n_heads, layer.n_kv_heads, layer.dim = 0, hq, hk, d
    layer.cache = c = KVCache(n, hk, d, 24)
    held = torch.tensor(np.cumsum([0, *before]), dtype=torch.int32, device="cuda")
    c.append(rand(sum(before), hk, d), rand(sum(before), hk, d), cu=held)
    k, v = c.read(held, sum(before))
    monkeypatch.setattr(decoder, "reads_back", lambda *a: back)
    calls = []
    read = c.read
    monkeypatch.setattr(c, "read", lambda *a: calls.append(a) or read(*a))
    x = rand(T, hq + 2 * hk, d)
    q, own_k, own_v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    out = layer.attend(q, own_k, own_v, decoder._starts(lens), lens, before)
    c.check()
    assert len(calls) == back and out.shape == q.shape
    at, a = np.cumsum([0, *before]), 0
    for b, m in enumerate(lens):
        kk = torch.cat([k[at[b]:at[b + 1]], own_k[a:a + m]]).double()
        vv = torch.cat([v[at[b]:at[b + 1]], own_v[a:a + m]]).double()
        hide = torch.arange(kk.shape[0], device="cuda")[None] > before[b] + torch.arange(m, device="cuda")[:, None]
        for h in range(hq if m else 0):
            s = ((q[a:a + m, h].double() @ kk[:, h * hk // hq].t()) * d ** -0.5).masked_fill(hide, -np.inf)
            w, vh = torch.softmax(s, 1), vv[:, h * hk // hq]
            o = w @ vh
            big = 1 + s.masked_fill(hide, 0).abs().amax(1, keepdim=True)
            # over codes: keys and values that are not rounded to fp16, 2^-11 of themselves; scores then
            # move by 2^-11 of the sum of |q k|, and weights by twice that
            move = 0.0 if back else 2.0 ** -11 + 2.0 ** -10 * ((q[a:a + m, h].double().abs() @ kk[:, h * hk // hq].abs().t()) * d ** -0.5).amax(1, keepdim=True)
            tol = (2.0 ** -11 + 2.0 ** -16 * big + move) * (w @ vh.abs()) + 2.0 ** -11 * o.abs() + 2.0 ** -24
            bad = float(((out[a:a + m, h].double() - o).abs() / tol).max())
            assert bad <= 1, f"sequence {b} head {h}: off by {bad:.2f} of its bound"
        a += m

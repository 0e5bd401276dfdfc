"""Prompt attention, the 8-bit key/value cache and its eviction against plain
implementations in 64 bits.

Tolerances. With w the exact softmax weights, A = sum w |v| and S the largest
|score| of a row, an output differs from the exact one by at most
  u_p A    each weight's rounding to the 16-bit type of the value product,
  u |out|  the output's own rounding,
  e A      e = 2^-16 (1 + S): scores are sums of 128 exact products in fp32
           (relative 128 * 2^-24 of sums of magnitude S at worst, taken for
           scores whose terms are no larger than eight times the sum), times
           ln-base factors and the running rescales, all fp32,
with u = 2^-11 (fp16) or 2^-8 (bf16), plus fp16's smallest subnormal.
ln-sum-exp and the accumulated weights carry the e part only."""
import math

import numpy as np
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import m2c
from paper_2410_14740_amd.attention import KVCache, prompt_attention

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F16, BF16 = torch.float16, torch.bfloat16


def rand(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def starts(lens):
    return torch.tensor(np.cumsum([0, *lens]), dtype=torch.int32, device="cuda")


def attention64(q, k, v, seen, scale):
    """q [m][d], k / v [l][d]: exact outputs, ln-sum-exp, weights, A and S."""
    x = (q.double() @ k.double().t()) * scale
    hide = torch.arange(k.shape[0], device=q.device)[None, :] >= seen[:, None]
    x = x.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(x, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    w = torch.exp(x - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[:, None])
    v = v.double()
    # values of keys that a row does not see do not enter it
    v = torch.where(hide.all(0)[:, None], torch.zeros_like(v), v)
    big = x.masked_fill(hide, 0).abs().amax(1) if k.shape[0] else torch.zeros(q.shape[0], dtype=torch.float64, device=q.device)
    return w @ v, lse, w, w @ v.abs(), big


def check_rows(out, lse, ref, u, u_p, what):
    o, e, _, A, S = ref
    eps = 2.0 ** -16 * (1 + S)
    tol = (u_p + eps[:, None]) * A + u * o.abs() + 2.0 ** -24
    err = (out.double() - o).abs()
    assert torch.isfinite(out.float()).all(), what
    assert bool((err <= tol).all()), f"{what}: output off by {float((err / tol).max()):.2f} of its bound"
    if lse is not None:
        fin = ~e.isinf()
        assert torch.equal(lse.isinf(), e.isinf()), what
        d = (lse.double() - e)[fin].abs()
        assert bool((d <= eps[fin]).all()), f"{what}: lse off by {float((d / eps[fin]).max()):.2f} of its bound"


def check_prompt(q, k, v, ql, kl, causal, out, lse, scale=None):
    hq, hk, d = q.shape[1], k.shape[1], q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    a = b = 0
    for i, (nq, nk) in enumerate(zip(ql, kl)):
        seen = torch.full((nq,), nk, device="cuda")
        if causal:
            seen = (nk - nq + 1 + torch.arange(nq, device="cuda")).clamp(min=0)
        for h in range(hq) if nq else ():
            g = h // (hq // hk)
            ref = attention64(q[a:a + nq, h], k[b:b + nk, g], v[b:b + nk, g], seen, scale)
            check_rows(out[a:a + nq, h], lse[a:a + nq, h] if lse is not None else None, ref,
                       U[q.dtype], U[q.dtype], f"sequence {i} head {h}")
        a, b = a + nq, b + nk


PROMPTS = [
    # heads, kv heads, width, type, query lengths, key lengths, causal
    (1, 1, 64, F16, [1], [1], True),
    (2, 1, 128, BF16, [1, 2, 3], [1, 2, 3], True),
    (4, 4, 64, F16, [33], [33], True),
    (4, 2, 128, F16, [63, 64, 65, 127, 128, 129], None, True),
    (8, 1, 128, BF16, [300, 1, 0, 257], None, True),
    (6, 2, 64, BF16, [5, 700, 31], None, False),
    (3, 3, 128, F16, [1, 64, 130], [200, 64, 1000], True),      # chunks against older keys
    (4, 2, 128, BF16, [70, 10, 200], [7, 0, 130], True),        # rows without keys
    (5, 1, 64, F16, [90, 3], [31, 0], True),
    (2, 2, 128, F16, [40, 9], [0, 77], False),
    (16, 2, 128, F16, [513, 1024], None, True),
    (40, 8, 64, BF16, [257, 255], None, True),
    (2, 1, 128, BF16, [3001], None, True),
]


@pytest.mark.parametrize("hq,hk,d,dt,ql,kl,causal", PROMPTS)
def test_prompt(hq, hk, d, dt, ql, kl, causal):
    kl = ql if kl is None else kl
    say(f"prompt {hq}/{hk}x{d} {dt} {ql} {kl} causal={causal}")
    q, k, v = rand((sum(ql), hq, d), dt, 1, 1.5), rand((sum(kl), hk, d), dt, 2), rand((sum(kl), hk, d), dt, 3)
    out, lse = prompt_attention(q, k, v, starts(ql), starts(kl), causal=causal, return_lse=True,
                                max_q=max(ql))
    check_prompt(q, k, v, ql, kl, causal, out, lse)
    # the hint changes no value's meaning: without it, and with a wrong one
    for hint in (0, 1, 1 << 20):
        again = prompt_attention(q, k, v, starts(ql), starts(kl), causal=causal, max_q=hint)
        check_prompt(q, k, v, ql, kl, causal, again, None)
    same = prompt_attention(q, k, v, starts(ql), starts(kl), causal=causal, max_q=max(ql))
    assert torch.equal(out, same)  # the same bits on every run


SPLITS = [
    # few rows and many keys: rows are cut along their keys
    (2, 1, 128, BF16, [1], [5000], True),
    (1, 1, 64, F16, [2], [769], True),                          # one part and a tile's first key
    (4, 2, 64, F16, [130, 17, 1], [4000, 900, 3000], True),
    (3, 3, 128, F16, [300, 0, 40], [4097, 2000, 1], False),
    (1, 1, 128, F16, [3000], [2000], True),                     # row tiles without keys before those that are cut
    (2, 2, 64, BF16, [1500, 700, 3000], [800, 2500, 3100], True),
    (8, 1, 128, F16, [129], [6000], True),                      # a tile of one row
    (64, 8, 64, BF16, [20, 5], [1500, 20000], True),
]


@pytest.mark.parametrize("hq,hk,d,dt,ql,kl,causal", SPLITS)
def test_prompt_cut_along_the_keys(hq, hk, d, dt, ql, kl, causal):
    say(f"prompt cut {hq}/{hk}x{d} {dt} {ql} {kl} causal={causal}")
    q, k, v = rand((sum(ql), hq, d), dt, 4, 1.5), rand((sum(kl), hk, d), dt, 5), rand((sum(kl), hk, d), dt, 6)
    cu, ck = starts(ql), starts(kl)
    args = dict(causal=causal, return_lse=True, max_q=max(ql))
    out, lse = prompt_attention(q, k, v, cu, ck, **args)
    check_prompt(q, k, v, ql, kl, causal, out, lse)
    assert all(map(torch.equal, (out, lse), prompt_attention(q, k, v, cu, ck, **args)))
    # the same call without room for parts
    desc = m2c.AttnDesc(m2c.DTYPE_BF16 if dt == BF16 else m2c.DTYPE_FP16, hq, hk, d, causal, 0, 0.0, 0)
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        setattr(desc, name + "_stride", t.stride()[:2])
    whole, wlse = torch.empty_like(out), torch.empty_like(lse)
    assert m2c.m2c_prompt_attention_workspace(desc, cu, ck, len(ql), sum(ql), sum(kl)) > 0
    m2c.m2c_prompt_attention(desc, q, k, v, cu, ck, len(ql), sum(ql), sum(kl), whole, wlse)
    check_prompt(q, k, v, ql, kl, causal, whole, wlse)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_prompt_cut_masked_values_do_not_enter(dt, what):
    """The keys that only some rows see lie in one part or in two."""
    say(f"prompt cut masked {dt} {what}")
    hq, hk, d, nq, nk = 2, 1, 64, 200, 3000
    q, k, v = rand((nq, hq, d), dt, 7), rand((nk, hk, d), dt, 8), rand((nk, hk, d), dt, 9)
    for at in (nk - 150, nk - 60, nk - 1):
        k2, v2 = k.clone(), v.clone()
        k2[at], v2[at] = what, what
        out, lse = prompt_attention(q, k2, v2, starts([nq]), starts([nk]), return_lse=True)
        blind = nq - (nk - at)  # the rows that do not see it
        check_prompt(q[:blind], k[:at], v[:at], [blind], [at], True, out[:blind], lse[:blind])
        assert not torch.isfinite(out[blind:].float()).any()


def test_prompt_cut_in_a_graph():
    say("prompt cut in a graph")
    q, k, v = rand((40, 4, 128), BF16, 11), rand((6000, 2, 128), BF16, 12), rand((6000, 2, 128), BF16, 13)
    cu, ck = starts([30, 10]), starts([2000, 4000])
    out = torch.empty_like(q)
    want = prompt_attention(q, k, v, cu, ck).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        prompt_attention(q, k, v, cu, ck, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prompt_attention(q, k, v, cu, ck, out=out)
    for i in range(4):
        q.copy_(rand(q.shape, BF16, 20 + i))
        cu.copy_(starts([30 - 7 * i, 10 + 7 * i]) if i else starts([30, 10]))
        cu[2] = 40
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, prompt_attention(q, k, v, cu, ck))
    assert want.shape == out.shape


@pytest.mark.parametrize("layout", ["fused", "head_major", "padded", "shared_row"])
def test_prompt_strides(layout):
    hq, hk, d, lens = 4, 2, 128, [130, 64, 3]
    T = sum(lens)
    say(f"prompt strides {layout}")
    if layout == "fused":
        x = rand((T, hq + 2 * hk, d), F16, 5)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        out = torch.zeros((T, hq + 3, d), dtype=F16, device="cuda")[:, 1:1 + hq]
    elif layout == "head_major":
        q, k, v = (rand((h, T, d), F16, 6 + i).transpose(0, 1) for i, h in enumerate((hq, hk, hk)))
        out = torch.zeros((hq, T, d), dtype=F16, device="cuda").transpose(0, 1)
    elif layout == "padded":
        q, k, v = (rand((T, h, d + 24), F16, 9 + i)[:, :, 8:8 + d] for i, h in enumerate((hq, hk, hk)))
        out = torch.zeros((T, hq, d + 8), dtype=F16, device="cuda")[:, :, :d]
    else:  # one key/value head for all, by a stride of 0
        q = rand((T, hq, d), F16, 12)
        k, v = (rand((T, 1, d), F16, 13 + i).expand(T, hk, d) for i in range(2))
        out = torch.zeros((T, hq, d), dtype=F16, device="cuda")
    whole = out._base if out._base is not None else out
    prompt_attention(q, k, v, starts(lens), out=out)
    check_prompt(q, k, v, lens, lens, True, out, None)
    mask = torch.ones_like(whole, dtype=torch.bool)
    mask.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((whole[mask] == 0).all())  # nothing written beside the rows


@pytest.mark.parametrize("dt,d", [(F16, 128), (BF16, 64)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_prompt_masked_values_do_not_enter(dt, d, what):
    hq, hk, lens = 4, 2, [200, 100]
    say(f"prompt masked {what}")
    q, k, v = rand((300, hq, d), dt, 21), rand((300, hk, d), dt, 22), rand((300, hk, d), dt, 23)
    clean = prompt_attention(q, k, v, starts(lens))
    at = 137  # of the first sequence: rows before it must not notice
    k2, v2 = k.clone(), v.clone()
    k2[at, :, 3], v2[at, :, 5] = what, what
    v2[at + 20] = what
    out = prompt_attention(q, k2, v2, starts(lens))
    check_prompt(q[:at], k[:at], v[:at], [at], [at], True, out[:at], None)
    assert torch.equal(out[200:], clean[200:])
    assert not torch.isfinite(out[at + 20:200].float()).any(dim=2).all()
    # rows of no sequence around the packed ones
    cu = starts([200, 100]) + 0
    k3 = torch.cat([k2.new_full((7, hk, d), what), k, k2.new_full((9, hk, d), what)])
    v3 = torch.cat([v2.new_full((7, hk, d), what), v, v2.new_full((9, hk, d), what)])
    out = prompt_attention(q, k3, v3, cu, cu + 7)
    assert torch.equal(out, clean)
    out = prompt_attention(q, k3, v3, cu, cu + 7, causal=False)
    assert torch.equal(out, prompt_attention(q, k, v, cu, causal=False))


def test_prompt_extreme_scores():
    say("prompt extreme scores")
    d, lens = 64, [150]
    q, k, v = rand((150, 2, d), F16, 31, 30.0), rand((150, 2, d), F16, 32, 30.0), rand((150, 2, d), F16, 33)
    out, lse = prompt_attention(q, k, v, starts(lens), return_lse=True)  # scores of some thousands
    check_prompt(q, k, v, lens, lens, True, out, lse)
    out, lse = prompt_attention(q, k, v, starts(lens), scale=1e-6, return_lse=True)
    check_prompt(q, k, v, lens, lens, True, out, lse, scale=1e-6)
    low = torch.finfo(F16).min  # one key at the type's lowest value for every query
    q1, k1 = torch.ones_like(q), k.clone()
    k1[0] = low
    out, lse = prompt_attention(q1, k1, v, starts(lens), scale=1.0, return_lse=True)
    check_prompt(q1, k1, v, lens, lens, True, out, lse, scale=1.0)


def test_prompt_without_keys():
    say("prompt without keys")
    q, k = rand((5, 2, 64), F16, 34), rand((0, 2, 64), F16, 35)
    for causal in (True, False):
        out, lse = prompt_attention(q, k, k, starts([3, 2]), starts([0, 0]), causal=causal, return_lse=True)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert prompt_attention(q[:0], k, k, starts([0, 0]), starts([0, 0])).shape == (0, 2, 64)


def test_prompt_many_sequences():
    """More sequences than a wave has lanes, empty ones among them."""
    say("prompt many sequences")
    ql = [(7 * i) % 150 if i % 5 else 0 for i in range(150)]
    kl = [(11 * i) % 190 for i in range(150)]
    q, k, v = rand((sum(ql), 2, 64), BF16, 36), rand((sum(kl), 1, 64), BF16, 37), rand((sum(kl), 1, 64), BF16, 38)
    out, lse = prompt_attention(q, k, v, starts(ql), starts(kl), return_lse=True)
    check_prompt(q, k, v, ql, kl, True, out, lse)
    c = KVCache(150, 1, 64, 4, dtype=BF16)
    shuffle_pages(c, 3)
    c.append(k, v, cu=starts(kl))
    check_cache(c, {b: (k[sum(kl[:b]):sum(kl[:b + 1])], v[sum(kl[:b]):sum(kl[:b + 1])]) for b in range(0, 150, 7)})
    kk, _ = c.read(starts(kl), sum(kl))
    assert float((kk.float() - k.float()).abs().max()) < 0.05
    x = rand((150, 2, 64), BF16, 39)
    o, e = c.attend(x, max_len=190, return_lse=True)
    check_attend(c, x, o, e, list(range(150)))


def test_prompt_offsets_past_32_bits():
    """Head strides past 2^31 elements, and token strides whose sum passes them."""
    say("prompt offsets past 32 bits")
    buf = torch.empty(2 ** 31 + 2 ** 24, dtype=F16, device="cuda")
    T, d = 100, 64
    far = [(T, 2, d), (d, 2 ** 31, 1)]
    x = rand((3, T, 2, d), F16, 44)
    k, v = (buf.as_strided(*far, 2 * i * T * d) for i in range(2))
    k.copy_(x[1]), v.copy_(x[2])
    out = buf.as_strided(*far, 4 * T * d)
    prompt_attention(x[0], k, v, starts([T]), out=out)
    check_prompt(x[0], x[1], x[2], [T], [T], True, out, None)
    wide = [(128, 1, d), (2 ** 24, d, 1)]
    x = rand((3, 128, 1, d), F16, 45)
    q, k, v = (buf.as_strided(*wide, i * d) for i in range(3))
    for a, b in zip((q, k, v), x):
        a.copy_(b)
    check_prompt(*x, [128], [128], True, prompt_attention(q, k, v, starts([128])), None)


@pytest.mark.parametrize("dt", [F16, BF16])
def test_small_weights_beside_a_large_one(dt):
    """One key takes almost all the weight, thousands of others 2^-20 .. 2^-30
    of it each, all with the same value: their sum is seen in the output."""
    say(f"small weights {dt}")
    d, L = 64, 8000
    k = torch.zeros((L, 1, d), dtype=dt, device="cuda")
    k[0, 0, 0] = 1.0
    v = torch.ones((L, 1, d), dtype=dt, device="cuda")
    v[0] = 0
    for lg in (20, 24, 26, 30):
        q = torch.zeros((1, 1, d), dtype=dt, device="cuda")
        q[0, 0, 0] = lg
        rest = (L - 1) * 2.0 ** -lg
        out = prompt_attention(q, k, v, starts([1]), starts([L]), scale=math.log(2.0))
        assert abs(float(out[0, 0, 0]) / (rest / (1 + rest)) - 1) <= 4 * U[dt], lg
        c = KVCache(1, 1, d, L // 64 + 1, dtype=dt)
        c.append(k, v, cu=starts([L]))
        out = c.attend(q, scale=math.log(2.0))
        assert abs(float(out[0, 0, 0]) / (rest / (1 + rest)) - 1) <= 4 * U[dt], lg


def test_prompt_stream_and_graph():
    say("prompt on another stream and in a graph")
    lens = [100, 300]
    q, k, v = rand((400, 4, 128), BF16, 41), rand((400, 2, 128), BF16, 42), rand((400, 2, 128), BF16, 43)
    cu = starts(lens)
    want = prompt_attention(q, k, v, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = prompt_attention(q, k, v, cu, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prompt_attention(q, k, v, cu, out=out)
    for i in range(3):
        q.copy_(rand(q.shape, BF16, 50 + i))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, prompt_attention(q, k, v, cu))


# ---------------------------------------------------------------------------
# the cache

def quantized(x):
    """Codes and scale of one block [tokens][d] by the definition (numpy, fp32)."""
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        amax = np.max(np.abs(x))
        if np.isnan(x).any():
            amax = np.float32(np.nan)
        s = np.float32(amax) / np.float32(127)
        if not (s > 0 and np.isfinite(s)):
            return np.zeros(x.shape, np.int8), s
        return np.clip(np.rint(x / s), -127, 127).astype(np.int8), s


def check_cache(c, tokens):
    """The cache holds exactly tokens = {sequence: (k, v)}."""
    B = c.block_tokens
    lens = c.len.cpu().tolist()
    table = c.table.cpu()
    for s, (k, v) in tokens.items():
        n = k.shape[0]
        assert lens[s] == n, (s, lens[s], n)
        last = (n - 1) // B if n else 0
        for h in range(c.n_kv_heads):
            for x, codes, scale, tail in ((k, c.k_codes, c.k_scale, c.tail_k), (v, c.v_codes, c.v_scale, c.tail_v)):
                for blk in range(n // B):
                    want, ws = quantized(x[blk * B:(blk + 1) * B, h])
                    page = int(table[s, h, blk])
                    got, gs = codes[page].cpu().numpy(), float(scale[page])
                    assert np.array_equal(np.float32(gs), ws, equal_nan=True), (s, h, blk, gs, ws)
                    assert np.array_equal(got, want), (s, h, blk)
                rest = n - last * B
                assert torch.equal(tail[s, h, :rest].view(torch.int16),
                                   x[last * B:n, h].contiguous().view(torch.int16)), (s, h)


def shuffle_pages(c, seed=0):
    g = torch.Generator().manual_seed(seed)
    c.table.copy_(torch.randperm(c.table.numel(), generator=g).int().view(c.table.shape))


@pytest.mark.parametrize("dt,d,B", [(F16, 128, 64), (BF16, 128, 128), (F16, 64, 32), (BF16, 64, 64),
                                    (BF16, 128, 32), (F16, 64, 128)])
def test_append_in_pieces(dt, d, B):
    say(f"append {dt} {d} {B}")
    H, lens = 3, [0, 1, B - 1, B, B + 1, 3 * B + 5]
    n = len(lens)
    k, v = ([rand((m, H, d), dt, 60 + 7 * i + j) for i, m in enumerate(lens)] for j in range(2))
    k[5][:B, 0] = 0  # a block of zeros
    whole = KVCache(n, H, d, 5, block_tokens=B, dtype=dt)
    shuffle_pages(whole)
    whole.weight.fill_(7.0)
    whole.append(torch.cat(k), torch.cat(v), cu=starts(lens))
    whole.check()
    check_cache(whole, {i: (k[i], v[i]) for i in range(n)})
    for i, m in enumerate(lens):  # the blocks that got tokens have no weight yet
        used = -(-m // B)
        assert bool((whole.weight[i, :, :used] == 0).all()) and bool((whole.weight[i, :, used:] == 7).all())
    # the same tokens in pieces of any size leave the same cache
    for piece in (1, 7, B, B + 3):
        c = KVCache(n, H, d, 5, block_tokens=B, dtype=dt)
        shuffle_pages(c)
        for a in range(0, max(lens), piece):
            part = [max(0, min(piece, m - a)) for m in lens]
            rows = [x[a:a + p] for x, p in zip(k, part)], [x[a:a + p] for x, p in zip(v, part)]
            if piece == 1:  # one token each, for the sequences that have one
                ids = [i for i, p in enumerate(part) if p]
                c.append(torch.cat(rows[0]), torch.cat(rows[1]),
                         seqs=torch.tensor(ids, dtype=torch.int32, device="cuda"))
            else:
                c.append(torch.cat(rows[0]), torch.cat(rows[1]), cu=starts(part))
        c.check()
        check_cache(c, {i: (k[i], v[i]) for i in range(n)})
        assert torch.equal(c.k_codes[c.table[5, :, :3].long()], whole.k_codes[whole.table[5, :, :3].long()])


@pytest.mark.parametrize("dt", [F16, BF16])
def test_codes_of_every_significand(dt):
    """Codes against an IEEE division for every significand of the block's
    largest magnitude with every significand of an element, over the exponents
    that give a code (keys: around 1; values: down among fp16's subnormals)."""
    say(f"codes of every significand {dt}")
    bits = 10 if dt == F16 else 7
    n, B, D = 1 << bits, 128, 128
    for top in (15, 10) if dt == F16 else (127, 20):  # exponent field of the largest
        sig = torch.arange(n, dtype=torch.int32)
        amax = (sig | top << bits)[:, None]
        x = torch.cat([sig | (top - e) << bits for e in range(9)])[None].expand(n, -1)
        x = torch.minimum(x, amax)
        x = torch.nn.functional.pad(torch.cat([amax, x], 1), (0, -(9 * n + 1) % (B * D)))
        x[:, 2::2] |= 0x8000  # half of them negative
        blocks = x.reshape(-1, B * D)
        if blocks.shape[0] > n:  # every block has its row's largest first
            blocks[:, 0] = amax.expand(-1, blocks.shape[0] // n).reshape(-1)
        vals = blocks.to(torch.int16).view(dt).view(-1, 1, D)
        T = vals.shape[0]
        c = KVCache(1, 1, D, T // B, block_tokens=B, dtype=dt)
        c.append(vals.cuda(), vals.cuda(), cu=starts([T]))
        c.check()
        f = vals.float().view(-1, B * D)
        s = f.abs().amax(1, keepdim=True).numpy() / np.float32(127)
        want = np.rint(f.numpy() / s).astype(np.int8)
        for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
            assert np.array_equal(scale.cpu().numpy(), s[:, 0])
            assert np.array_equal(codes.view(-1, B * D).cpu().numpy(), want)


def test_append_strides_seqs_and_places():
    say("append strides, seqs, pos")
    H, d, B = 2, 128, 64
    x = rand((400, 2 * H + 1, d), F16, 80)
    k, v = x[:, :H], x[:, H:2 * H]
    c = KVCache(6, H, d, 4, block_tokens=B)
    shuffle_pages(c, 1)
    seqs = torch.tensor([4, 1, 3], dtype=torch.int32, device="cuda")
    c.append(k[:300], v[:300], cu=starts([100, 150, 50]), seqs=seqs)
    c.check()
    check_cache(c, {4: (k[:100], v[:100]), 1: (k[100:250], v[100:250]), 3: (k[250:300], v[250:300]),
                    0: (k[:0], v[:0])})
    # over the last block from its middle, from a block's start, and at the end
    pos = torch.tensor([70, 64, 50], dtype=torch.int32, device="cuda")
    c.append(k[300:400], v[300:400], cu=starts([20, 70, 10]), seqs=seqs, pos=pos)
    c.check()
    cat = torch.cat
    check_cache(c, {4: (cat([k[:70], k[300:320]]), cat([v[:70], v[300:320]])),
                    1: (cat([k[100:164], k[320:390]]), cat([v[100:164], v[320:390]])),
                    3: (cat([k[250:300], k[390:400]]), cat([v[250:300], v[390:400]]))})
    # a block that was full is still the last one: its tokens can be written over
    one = torch.tensor([3], dtype=torch.int32, device="cuda")
    c.append(k[:4], v[:4], cu=starts([4]), seqs=one)
    c.append(k[4:5], v[4:5], seqs=one, pos=torch.tensor([60], dtype=torch.int32, device="cuda"))
    c.check()
    check_cache(c, {3: (cat([k[250:300], k[390:400], k[4:5]]), cat([v[250:300], v[390:400], v[4:5]]))})
    c.reset(one)
    assert c.len.cpu().tolist()[3] == 0 and c.len.cpu().tolist()[4] == 90


def test_append_non_finite_blocks():
    say("append non-finite blocks")
    for dt in (F16, BF16):
        for what in (math.inf, math.nan, -math.inf):
            k, v = rand((128, 2, 64), dt, 90), rand((128, 2, 64), dt, 91)
            k[5, 0, 9] = what
            v[70, 1, 0] = what
            c = KVCache(1, 2, 64, 4, dtype=dt)
            c.append(k, v, cu=starts([128]))
            check_cache(c, {0: (k, v)})
            rk, rv = c.read(starts([128]), 128)
            assert bool(rk[:64, 0].isnan().all()) and bool(rk[:, 1].isfinite().all()) and bool(rk[64:].isfinite().all())
            assert bool(rv[64:, 1].isnan().all()) and bool(rv[:, 0].isfinite().all())
    # the types' ends: the largest and the smallest magnitudes
    for dt in (F16, BF16):
        f = torch.finfo(dt)
        x = torch.zeros((64, 1, 64), dtype=dt, device="cuda")
        x[0, 0, 0], x[1, 0, 1] = f.max, f.min
        y = torch.full((64, 1, 64), f.smallest_normal, dtype=dt, device="cuda")
        c = KVCache(1, 1, 64, 2, dtype=dt)
        c.append(x, y, cu=starts([64]))
        check_cache(c, {0: (x, y)})
        rk, _ = c.read(starts([64]), 64)
        assert torch.equal(rk, x)


def test_append_errors_leave_the_sequence():
    say("append errors")
    H, d, B = 2, 64, 32
    k, v = rand((200, H, d), F16, 95), rand((200, H, d), F16, 96)
    c = KVCache(3, H, d, 2, block_tokens=B)
    c.append(k[:90], v[:90], cu=starts([40, 50, 0]))
    state = [t.clone() for t in (c.len, c.k_codes, c.tail_k, c.weight)]

    def same():
        return all(torch.equal(a, b) for a, b in zip(state, (c.len, c.k_codes, c.tail_k, c.weight)))

    def i32(*a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    c.append(k[:30], v[:30], cu=starts([30]))  # 70 of 64 tokens
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_CAPACITY and same()
    for pos in (41, 10, -1, 33 + 32):  # past the end, inside an earlier block, negative
        c.append(k[:2], v[:2], cu=starts([2]), pos=i32(pos))
        with pytest.raises(m2c.M2CError) as e:
            c.check()
        assert e.value.status == m2c.M2C_ERR_STATE and same(), pos
    for s in (3, -1):
        c.append(k[:2], v[:2], cu=starts([2]), seqs=i32(s))
        with pytest.raises(m2c.M2CError) as e:
            c.check()
        assert e.value.status == m2c.M2C_ERR_INVALID_ARG and same()
    c.table[2] = 1 << 20  # a page that does not exist
    c.append(k[:40], v[:40], cu=starts([40]), seqs=i32(2))
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG
    out = c.attend(rand((1, H, d), F16, 97), seqs=i32(2))
    assert bool(torch.isfinite(out.float()).all())
    with pytest.raises(m2c.M2CError):
        c.check()
    out = c.attend(rand((2, H, d), F16, 97), seqs=i32(-1, 7))
    assert bool((out == 0).all())
    with pytest.raises(m2c.M2CError):
        c.check()
    c.check()  # reported once
    c.append(k[:1], v[:1], seqs=i32(0))  # the others go on
    c.check()
    assert c.len.cpu().tolist()[0] == 41


@pytest.mark.parametrize("dt,d,B", [(F16, 128, 64), (BF16, 64, 32), (BF16, 128, 128), (F16, 64, 64)])
def test_read(dt, d, B):
    say(f"read {dt} {d} {B}")
    H, lens = 3, [0, 1, 2 * B, 3 * B + 7]
    k, v = rand((sum(lens), H, d), dt, 100), rand((sum(lens), H, d), dt, 101)
    c = KVCache(4, H, d, 4, block_tokens=B, dtype=dt)
    shuffle_pages(c, 2)
    c.append(k, v, cu=starts(lens))
    # room for 5 more tokens after each sequence, and the third only in part
    room = [5, 6, B + 3, 3 * B + 12]
    cu = starts(room)
    ko = torch.full((sum(room) + 2, 2 * H, d), 9.0, dtype=dt, device="cuda")
    kk, vv = c.read(cu, k=ko[:, :H], v=ko[:, H:])
    c.check()
    at = 0
    for i, (n, r) in enumerate(zip(lens, room)):
        got = min(n, r)
        lo = sum(lens[:i])
        for h in range(H):
            for x, y in ((k, kk), (v, vv)):
                for blk in range(-(-got // B)):
                    a, b = blk * B, min(got, blk * B + B)
                    if blk * B + B <= n:
                        codes, s = quantized(x[lo + a:lo + a + B, h])
                        want = torch.from_numpy(codes.astype(np.float32) * s).to(dt)[:b - a]
                    else:
                        want = x[lo + a:lo + b, h].cpu()
                    assert torch.equal(y[at + a:at + b, h].cpu(), want), (i, h, blk)
        assert bool((ko[at + got:at + r] == 9).all())
        at += r
    assert bool((ko[at:] == 9).all())


def dense_of(c, s, h):
    """What the cache says of one sequence and head, in 64 bits."""
    n, B = int(c.len[s]), c.block_tokens
    page = c.table[s, h, :n // B].long()
    res = []
    for codes, scale, tail in ((c.k_codes, c.k_scale, c.tail_k), (c.v_codes, c.v_scale, c.tail_v)):
        full = codes[page].double() * scale[page].double()[:, None, None]
        res.append(torch.cat([full.reshape(-1, c.head_dim), tail[s, h, :n % B].double()]))
    return res


def check_attend(c, q, out, lse, seqs, scale=None, before=None):
    n, hq, d = q.shape
    G = hq // c.n_kv_heads
    scale = d ** -0.5 if scale is None else scale
    for b, s in enumerate(seqs):
        L = int(c.len[s])
        for h in range(c.n_kv_heads):
            k, v = dense_of(c, s, h)
            ref = attention64(q[b, h * G:(h + 1) * G], k, v, torch.full((G,), L, device="cuda"), scale)
            u_p = U[F16]
            if c.dtype == BF16 and L % c.block_tokens:
                u_p = U[BF16]  # the open block's weights are rounded to bf16
            check_rows(out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] if lse is not None else None,
                       ref, U[c.dtype], u_p, f"row {b} (sequence {s}) kv head {h}")
            if before is not None:
                B = c.block_tokens
                w = torch.nn.functional.pad(ref[2].sum(0), (0, -L % B)).view(-1, B).sum(1)
                got = c.weight[s, h].double()
                want = before[s, h].double()
                want[:w.numel()] += w
                tol = 2.0 ** -16 * (1 + (float(ref[4].max()) if L else 0)) * (want - before[s, h].double()) + 2.0 ** -22 * want + 1e-9
                assert bool(((got - want).abs() <= tol).all()), (b, h)


def filled(lens, H, d, B, dt, max_blocks, seed, poison=True):
    c = KVCache(len(lens), H, d, max_blocks, block_tokens=B, dtype=dt)
    shuffle_pages(c, seed)
    if poison:  # whatever lies in unused pages and past the tails' ends must not matter
        c.k_codes.fill_(-128)
        c.v_codes.fill_(-128)
        c.k_scale.fill_(math.nan)
        c.v_scale.fill_(math.nan)
        c.tail_k.fill_(math.nan)
        c.tail_v.fill_(math.inf)
    k, v = rand((sum(lens), H, d), dt, seed + 1), rand((sum(lens), H, d), dt, seed + 2)
    if sum(lens):
        c.append(k, v, cu=starts(lens))
    return c


ATTENDS = [
    # heads, kv heads, width, block, type, lengths
    (1, 1, 64, 32, F16, [1]),
    (2, 2, 128, 64, F16, [0, 1, 63, 64, 65]),
    (8, 1, 128, 64, BF16, [127, 128, 300, 1]),
    (6, 2, 64, 64, F16, [700, 31, 64]),
    (16, 1, 128, 32, F16, [33, 32, 31, 250]),
    (24, 1, 128, 64, BF16, [100, 641]),      # two tiles of query heads
    (40, 2, 64, 128, BF16, [1, 127, 128, 129, 1000]),
    (64, 8, 128, 64, F16, [513, 2000]),
    (8, 8, 128, 128, F16, [127, 640, 64]),
    (10, 2, 128, 32, BF16, [5000]),          # split
    (5, 1, 64, 32, F16, [9001, 77]),
]


@pytest.mark.parametrize("hq,hk,d,B,dt,lens", ATTENDS)
def test_attend(hq, hk, d, B, dt, lens):
    say(f"attend {hq}/{hk}x{d} block {B} {dt} {lens}")
    c = filled(lens, hk, d, B, dt, max(lens) // B + 2, 110)
    q = rand((len(lens), hq, d), dt, 113, 1.5)
    seqs = list(range(len(lens)))
    out, lse = c.attend(q, max_len=max(lens), return_lse=True)
    c.check()
    check_attend(c, q, out, lse, seqs)
    assert torch.equal(out, c.attend(q, max_len=max(lens)))  # the same bits on every run
    for hint in (0, 1, 200):  # unknown, and far too short
        o, e = c.attend(q, max_len=hint, return_lse=True)
        check_attend(c, q, o, e, seqs)
    c.weight.copy_(rand(c.weight.shape, torch.float32, 114).abs())
    before = c.weight.clone()
    o, e = c.attend(q, max_len=max(lens), track=True, return_lse=True)
    assert torch.equal(o, out) and torch.equal(e, lse)
    check_attend(c, q, o, e, seqs, before=before)
    before = c.weight.clone()
    o = c.attend(q, track=True)
    check_attend(c, q, o, None, seqs, before=before)


@pytest.mark.parametrize("n", [64, 70])
def test_attend_many_ragged_sequences(n):
    """As many sequences as a wave has lanes, and more; the longest split, some empty, heads over two tiles."""
    say(f"attend {n} ragged sequences")
    lens = [(37 * i) % 400 if i % 6 else 0 for i in range(n)]
    lens[n // 2], lens[-1] = 3000, 1500
    c = filled(lens, 1, 64, 32, F16, 100, 115)
    q = rand((n, 20, 64), F16, 118, 1.5)
    before = c.weight.clone()
    out, lse = c.attend(q, max_len=3000, track=True, return_lse=True)
    c.check()
    check_attend(c, q, out, lse, list(range(n)), before=before)
    for hint in (0, 64, 500):
        o, e = c.attend(q, max_len=hint, return_lse=True)
        check_attend(c, q, o, e, list(range(n)))


@pytest.mark.parametrize("hq,hk,d,dt", [(16, 8, 128, BF16), (32, 8, 64, F16)])
def test_attend_however_it_is_split(hq, hk, d, dt):
    """Whole rows, chunks and even shares by the longest length the caller
    names: the same values and block weights; rows without tokens, of one and of
    many between long ones."""
    say(f"attend splits {hq}/{hk}x{d} {dt}")
    lens = [4000, 0, 1, 700, 64, 65, 0, 3333, 128, 2, 1999, 63]
    c = filled(lens, hk, d, 64, dt, 64, 119)
    q = rand((len(lens), hq, d), dt, 122, 1.5)
    for hint in (4000, 2000, 1500, 64, 0):
        before = c.weight.clone()
        out, lse = c.attend(q, max_len=hint, track=True, return_lse=True)
        c.check()
        check_attend(c, q, out, lse, list(range(len(lens))), before=before)
        assert bool((out[[1, 6]] == 0).all()) and bool((c.weight[[1, 6]] == before[[1, 6]]).all())


def test_attend_rows_strides_and_scale():
    say("attend subset, strides, scale")
    c = filled([70, 0, 500, 64, 129], 2, 128, 64, BF16, 9, 120)
    seqs = [3, 0, 4]
    ids = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    x = rand((3, 8, 128), BF16, 124)
    q = x[:, 1:7]
    room = torch.zeros((3, 9, 136), dtype=BF16, device="cuda")
    out, lse = c.attend(q, seqs=ids, scale=0.3, out=room[:, 2:8, :128], return_lse=True)
    check_attend(c, q, out, lse, seqs, scale=0.3)
    assert bool((room[:, :2] == 0).all()) and bool((room[:, 8:] == 0).all()) and bool((room[..., 128:] == 0).all())


@pytest.mark.parametrize("dt", [F16, BF16])
def test_attend_ranges(dt):
    """Queries and keys of very large and very small magnitude, one key far above the others."""
    say(f"attend ranges {dt}")
    for qs, ks in ((1e-4, 1e3), (2e3, 1e-3), (30.0, 30.0)) + (((1e30, 1e-30), (1e-30, 1e30)) if dt == BF16 else ()):
        c = KVCache(1, 2, 64, 8, block_tokens=32, dtype=dt)
        k, v = rand((200, 2, 64), dt, 130, ks), rand((200, 2, 64), dt, 131, 3.0)
        c.append(k, v, cu=starts([200]))
        q = rand((1, 6, 64), dt, 132, qs)
        q[:, 1] = 0
        out, lse = c.attend(q, return_lse=True)
        check_attend(c, q, out, lse, [0])


def test_attend_pages_past_32_bits():
    """Pages whose byte offsets do not fit 32 bits (and element offsets neither)."""
    say("attend pages past 32 bits")
    pages, H = 540_000, 2  # of 8192 codes: 4.4e9 bytes
    c = KVCache(1, H, 128, 8, n_pages=pages)
    c.table.copy_(torch.tensor([pages - 1 - 7 * i for i in range(16)], dtype=torch.int32).view(1, H, 8))
    k, v = rand((400, H, 128), F16, 140), rand((400, H, 128), F16, 141)
    c.append(k, v, cu=starts([400]))
    check_cache(c, {0: (k, v)})
    q = rand((1, 4, 128), F16, 142)
    out, lse = c.attend(q, return_lse=True)
    check_attend(c, q, out, lse, [0])
    rk, _ = c.read(starts([400]), 400)
    assert float((rk.float() - k.float()).abs().max()) < 0.05


def test_decode_graph():
    """Append and attend captured once, replayed for token after token."""
    say("decode graph")
    H, d = 2, 128
    c, e = (filled([60, 10, 130], H, d, 64, F16, 4, 150, poison=False) for _ in range(2))
    k, v, q = rand((3, H, d), F16, 151), rand((3, H, d), F16, 152), rand((3, 8, d), F16, 153)
    need = m2c.m2c_kv_attend_workspace(c.desc, 3, 8, 1, 0)
    assert need > 0
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.append(k, v)
        c.attend(q, track=True, out=out)
    for i in range(8):
        k.copy_(rand(k.shape, F16, 160 + i))
        v.copy_(rand(v.shape, F16, 170 + i))
        q.copy_(rand(q.shape, F16, 180 + i))
        g.replay()
        torch.cuda.synchronize()
        e.append(k, v)
        want = e.attend(q, track=True)
        assert torch.equal(out, want) and torch.equal(c.len, e.len) and torch.equal(c.weight, e.weight), i
    c.check()


def test_calls_on_another_stream():
    say("cache calls on another stream")
    side = torch.cuda.Stream()
    c = KVCache(2, 2, 64, 4)
    k, v, q = rand((150, 2, 64), F16, 190), rand((150, 2, 64), F16, 191), rand((2, 4, 64), F16, 192)
    cu = starts([100, 50])
    side.wait_stream(torch.cuda.current_stream())
    c.append(k, v, cu=cu, stream=side)
    out, lse = c.attend(q, track=True, return_lse=True, stream=side)
    rk, _ = c.read(cu, 150, stream=side)
    c.check(stream=side)
    check_attend(c, q, out, lse, [0, 1])
    assert float((rk.float() - k.float()).abs().max()) < 0.05


# ---------------------------------------------------------------------------
# eviction

def evicted(table, weight, n, B, keep, first, recent):
    """One row's (table, weight, length) after an eviction, by the definition."""
    m = (n - 1) // B if n else 0
    if m <= keep:
        return table, weight, n
    u = weight.view(np.uint32).astype(np.int64)
    key = np.where(u >> 31, ~u & 0xffffffff, u | 0x80000000)
    mid = list(range(first, m - recent))
    best = sorted(mid, key=lambda i: (-key[i], i))[:keep - first - recent]
    kept = sorted(set(range(first)) | set(range(m - recent, m)) | set(best))
    gone = [i for i in range(m) if i not in set(kept)]
    order = kept + list(range(m, len(table))) + gone
    w = weight.copy()
    w[gone] = 0
    return table[order], w[order], n - len(gone) * B


@pytest.mark.parametrize("mb,B,keep,first,recent", [
    (1, 64, 0, 0, 0), (8, 32, 3, 1, 1), (8, 64, 0, 0, 0), (40, 64, 16, 0, 16), (256, 32, 100, 4, 9),
    (257, 64, 200, 200, 0), (700, 64, 33, 0, 0), (1024, 128, 1000, 1, 2), (3000, 64, 700, 4, 64),
    (9000, 32, 4000, 0, 1),
])
def test_evict(mb, B, keep, first, recent):
    say(f"evict {mb} {B} {keep} {first} {recent}")
    n, H = 5, 2
    rng = np.random.default_rng(mb + keep)
    lens = [0, min(B, mb * B), (keep + 1) * B if keep + 1 <= mb else mb * B, mb * B, mb * B - B // 2]
    for kind in ("spread", "ties", "equal", "signs"):
        w = np.exp(rng.standard_normal((n, H, mb)) * 2).astype(np.float32)
        if kind == "ties":
            w = np.round(w).astype(np.float32)
        elif kind == "equal":
            w[:] = 0.5
        elif kind == "signs":
            w = rng.standard_normal((n, H, mb)).astype(np.float32)
            w[rng.random(w.shape) < 0.2] = 0.0
            w[rng.random(w.shape) < 0.2] = -0.0
            w[rng.random(w.shape) < 0.05] = np.inf
            w[rng.random(w.shape) < 0.05] = -np.inf
        c = KVCache(n, H, 64, mb, block_tokens=B, n_pages=1)
        c.table.copy_(torch.from_numpy(rng.permutation(n * H * mb).astype(np.int32).reshape(n, H, mb)))
        c.weight.copy_(torch.from_numpy(w))
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
        t0 = c.table.cpu().numpy()
        want = [[evicted(t0[s, h], w[s, h], lens[s], B, keep, first, recent) for h in range(H)] for s in range(n)]
        out = {k: torch.full_like(getattr(c, k), -7) for k in ("table", "weight", "len")}
        c.evict(keep, first, recent, out=out)
        assert torch.equal(c.table.cpu(), torch.from_numpy(t0)) and c.len.cpu().tolist() == lens
        sub = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
        c.evict(keep, first, recent, seqs=sub)
        assert c.len.cpu().tolist() == [want[s][0][2] if s in (1, 3) else lens[s] for s in range(n)]
        c.evict(keep, first, recent)
        c.check()
        for got in (out, {k: getattr(c, k) for k in out}):
            assert got["len"].cpu().tolist() == [want[s][0][2] for s in range(n)], kind
            t, x = got["table"].cpu().numpy(), got["weight"].cpu().numpy()
            for s in range(n):
                for h in range(H):
                    assert np.array_equal(t[s, h], want[s][h][0]), (kind, s, h)
                    assert np.array_equal(x[s, h].view(np.uint32), want[s][h][1].view(np.uint32)), (kind, s, h)


def test_evict_then_go_on():
    """After an eviction the sequences are their remaining tokens: attention, append and a second eviction."""
    say("evict then go on")
    H, d, B = 2, 64, 32
    c = filled([32 * 7 + 5, 32 * 9, 40], H, d, B, F16, 12, 200)
    q = rand((3, 4, d), F16, 201, 2.0)
    c.attend(q, track=True)
    w = c.weight.clone()
    c.evict(4, 1, 1)
    c.check()
    assert c.len.cpu().tolist() == [32 * 4 + 5, 32 * 5, 40]
    for s, m in ((0, 7), (1, 8)):
        for h in range(H):
            kept = c.weight[s, h, 1:3]
            assert float(kept.min()) >= float(torch.topk(w[s, h, 1:m - 1], 2).values.min())
    out, lse = c.attend(q, return_lse=True)
    check_attend(c, q, out, lse, [0, 1, 2])
    k, v = rand((150, H, d), F16, 202), rand((150, H, d), F16, 203)
    c.append(k, v, cu=starts([50, 50, 50]))
    c.check()
    before = c.weight.clone()
    out, lse = c.attend(q, track=True, return_lse=True)
    check_attend(c, q, out, lse, [0, 1, 2], before=before)
    c.evict(2, 0, 0)
    out, lse = c.attend(q, return_lse=True)
    check_attend(c, q, out, lse, [0, 1, 2])


# ---------------------------------------------------------------------------
# refusals on tensors (the C entry points' own are checked without a GPU)

def test_tensor_refusals():
    q, k, v = rand((4, 4, 64), F16, 1), rand((4, 2, 64), F16, 2), rand((4, 2, 64), F16, 3)
    cu = starts([4])
    bad = [
        lambda: prompt_attention(q.float(), k, v, cu), lambda: prompt_attention(q, k.bfloat16(), v, cu),
        lambda: prompt_attention(q, k, v[:3], cu), lambda: prompt_attention(q.cpu(), k, v, cu),
        lambda: prompt_attention(q, k, v, cu.long()), lambda: prompt_attention(q, k, v, cu[:1]),
        lambda: prompt_attention(q[:, :3], k, v, cu), lambda: prompt_attention(q[..., :48], k[..., :48], v[..., :48], cu),
        lambda: prompt_attention(q, k, v, cu, scale=-1.0), lambda: prompt_attention(q, k, v, cu, scale=math.nan),
        lambda: prompt_attention(q, k, v, cu, out=torch.empty((4, 4, 128), dtype=F16, device="cuda")),
        lambda: prompt_attention(rand((4, 4, 68), F16, 1)[..., 2:66], k, v, cu),
        lambda: KVCache(1, 2, 64, 2, dtype=torch.float32),
    ]
    c = KVCache(2, 2, 64, 2)
    bad += [
        lambda: c.append(k, v), lambda: c.append(k, v[:3], cu=cu), lambda: c.append(k.bfloat16(), v, cu=cu),
        lambda: c.append(k, v, cu=cu, pos=starts([1])), lambda: c.append(k, v, cu=cu, seqs=starts([1]).long()[:1]),
        lambda: c.read(cu), lambda: c.read(cu, k=k), lambda: c.attend(q), lambda: c.attend(q[:2, :3]),
        lambda: c.attend(q[:2], scale=-0.5), lambda: c.evict(1, 1, 1), lambda: c.evict(-1),
        lambda: c.evict(1, out={"table": c.table, "weight": c.weight, "len": c.len}),
        lambda: KVCache(2, 2, 64, 2, tensors={"k_codes": c.k_codes}),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(m2c.M2CError) as e:
            f()
        assert e.value.status == m2c.M2C_ERR_INVALID_ARG, i
    c.check()

"""Attention of chunks of tokens over the 8-bit cache against loops in 64 bits
over what the cache's own arrays say.

Tolerances. With w the exact softmax weights of a row, A8 and A16 its sums of w |v|
over the keys that are codes and over the others, and S its largest |score|, an
output differs from the exact one by at most
  2^-11 A8          each weight's rounding to fp16 (codes are exact in it),
  u A16             the others' to the 16-bit type, u = 2^-11 (fp16) or 2^-8 (bf16),
  e (A8 + A16)      e = 2^-16 (1 + S): scores are sums of 128 exact products in
                    fp32 (relative 128 * 2^-24 of sums of magnitude S at worst,
                    taken for scores whose terms are no larger than eight times
                    the sum), and exponents of up to 100 binary places, rounded
                    to 2^-17.4, all fp32,
  2^-35 C W         the weights of codes that are subnormal in fp16, off by 2^-25 of
                    what 2^m stands for: weights are 2^(x + g - m + 10), m at most
                    the row's largest x + g, 2^g a value block's scale s in the
                    call's unit, so 2^m over the sum of 2^x is at most W, the
                    largest w s of a coded key or the largest w of another times the
                    unit (2^-24 in fp16, at most 2^-20 of the largest s in bf16); C
                    is the sum of |code| over the keys,
  u |out|           the output's own rounding, and fp16's smallest number, 2^-24.
ln-sum-exp carries e alone."""
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


_made = []


@pytest.fixture(autouse=True)
def clean():
    """Poisoned memory does not go back to the allocator, which other tests take
    memory from without filling it."""
    yield
    for c in _made:
        for t in (c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.tail_k, c.tail_v):
            t.zero_()
    _made.clear()


def make(n, hk, d, block, dtype, lens, seed=1, sigma=1.0, spare=0):
    """A cache that holds `lens` tokens, its pages in no order, its unused places poisoned."""
    mb = max(-(-max(lens) // block), 1) + spare
    c = KVCache(n, hk, d, mb, block_tokens=block, dtype=dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c.table.copy_(torch.randperm(c.table.numel(), generator=g, device="cuda").int().view_as(c.table))
    c.k_codes.fill_(77), c.v_codes.fill_(-77)
    c.k_scale.fill_(math.nan), c.v_scale.fill_(math.inf)
    c.tail_k.fill_(math.nan), c.tail_v.fill_(math.inf)
    _made.append(c)
    if sum(lens):
        c.append(rand((sum(lens), hk, d), dtype, seed + 1, sigma), rand((sum(lens), hk, d), dtype, seed + 2, sigma), cu=starts(lens))
    c.check()
    return c


def held64(c, s, h):
    """Keys and values of a sequence and head in 64 bits, the value scales of those
    that are codes, and the sums of their |code| by dimension."""
    n, B = int(c.len[s]), c.block_tokens
    page = c.table[s, h, :n // B].long()
    size = c.v_scale[page].double()[:, None].expand(-1, B).reshape(-1)
    codes = c.v_codes[page].double().abs().sum((0, 1))
    kv = []
    for name in ("k", "v"):
        x = getattr(c, name + "_codes")[page].double() * getattr(c, name + "_scale")[page].double()[:, None, None]
        kv.append(torch.cat([x.reshape(-1, c.head_dim), getattr(c, "tail_" + name)[s, h, :n % B].double()]))
    return *kv, size, codes


def check(c, q, cu, k, v, out, lse, seqs=None, scale=None, what=""):
    scale = c.head_dim ** -0.5 if scale is None else scale
    G, cu = q.shape[1] // c.n_kv_heads, cu.tolist()
    u, worst = U[q.dtype], 0.0
    for b in range(len(cu) - 1):
        rows = slice(cu[b], cu[b + 1])
        m = cu[b + 1] - cu[b]
        if m == 0:
            continue
        s = b if seqs is None else int(seqs[b])
        for h in range(c.n_kv_heads):
            kk, vv, size, codes = held64(c, s, h)
            coded = size.shape[0]
            if k is not None:
                kk, vv = torch.cat([kk, k[rows, h].double()]), torch.cat([vv, v[rows, h].double()])
            hide = torch.arange(kk.shape[0], device="cuda")[None, :] >= (kk.shape[0] - m + 1 + torch.arange(m, device="cuda"))[:, None]
            vv = torch.where(hide.all(0)[:, None], torch.zeros_like(vv), vv)
            for g in range(h * G, (h + 1) * G):
                x = ((q[rows, g].double() @ kk.t()) * scale).masked_fill(hide, -math.inf)
                e = torch.logsumexp(x, 1) if kk.shape[0] else torch.full((m,), -math.inf, dtype=torch.float64, device="cuda")
                w = torch.exp(x - torch.where(e.isinf(), torch.zeros_like(e), e)[:, None])
                a = vv.abs()
                eps = 2.0 ** -16 * (1 + (x.masked_fill(hide, 0).abs().amax(1) if kk.shape[0] else torch.zeros_like(e)))
                o = w @ vv
                tol = (2.0 ** -11 + eps)[:, None] * (w[:, :coded] @ a[:coded]) + (u + eps)[:, None] * (w[:, coded:] @ a[coded:])
                if coded:
                    top = (w[:, :coded] * size).amax(1)
                    if kk.shape[0] > coded:
                        top = torch.maximum(top, w[:, coded:].amax(1) * (2.0 ** -24 if q.dtype == F16 else 2.0 ** -20 * size.amax()))
                    tol = tol + 2.0 ** -35 * codes * top[:, None]
                tol = tol + u * o.abs() + (2.0 ** -24 if q.dtype == F16 else 1e-38)
                assert torch.isfinite(out[rows, g].float()).all(), f"{what}: sequence {b} head {g}"
                bad = float(((out[rows, g].double() - o).abs() / tol).max())
                assert bad <= 1, f"{what}: sequence {b} head {g}: output off by {bad:.2f} of its bound"
                worst = max(worst, bad)
                if lse is not None:
                    fin = ~e.isinf()
                    assert torch.equal(lse[rows, g].isinf(), ~fin)
                    off = ((lse[rows, g].double() - e).abs() / eps)[fin]
                    assert bool((off <= 1).all()), f"{what}: sequence {b} head {g}: lse off by {float(off.max()):.2f}"
    return worst


CASES = [  # heads, kv heads, width, block, type, held, chunks
    (1, 1, 64, 64, F16, [0], [1]), (1, 1, 128, 64, BF16, [1], [1]), (2, 2, 64, 32, F16, [31, 32, 33, 64, 95, 96], [1, 2, 3, 1, 64, 65]),
    (4, 1, 128, 64, F16, [63, 64, 65, 127, 0], [33, 32, 31, 1, 130]), (8, 2, 128, 128, BF16, [127, 128, 129, 300], [5, 64, 1, 200]),
    (16, 16, 64, 64, F16, [100], [33]), (64, 8, 128, 64, BF16, [500, 77], [16, 3]), (40, 8, 64, 32, BF16, [160, 33, 1000], [7, 140, 1]),
    (3, 3, 128, 32, F16, [224, 32], [129, 256]), (6, 2, 64, 128, F16, [640, 50, 0, 383], [10, 0, 300, 1]), (32, 1, 128, 64, BF16, [192], [40]),
    (5, 1, 128, 64, F16, [4100], [9]), (12, 4, 64, 64, BF16, [2500, 10], [600, 70]),
]


@pytest.mark.parametrize("hq,hk,d,block,dt,lens,ql", CASES)
@pytest.mark.parametrize("how", ["new", "held"])
def test_chunk(hq, hk, d, block, dt, lens, ql, how):
    say(f"chunk {hq}/{hk}x{d} {block} {dt} {lens} {ql} {how}")
    n, T = len(lens), sum(ql)
    c = make(n, hk, d, block, dt, lens if how == "new" else [a + b for a, b in zip(lens, ql)])
    x = rand((T, hq + 2 * hk, d), dt, 7)
    q, k, v = x[:, :hq] * 1.5, x[:, hq:hq + hk], x[:, hq + hk:]
    k, v = (k, v) if how == "new" else (None, None)
    cu = starts(ql)
    out, lse = c.attend_chunk(q, cu, k, v, max_q=max(ql), max_len=int(c.len.max()), return_lse=True)
    c.check()
    check(c, q, cu, k, v, out, lse, what=f"{how}")
    for hint in (dict(), dict(max_q=1, max_len=1), dict(max_q=1 << 20, max_len=1 << 30)):  # hints change no value's meaning
        check(c, q, cu, k, v, c.attend_chunk(q, cu, k, v, **hint), None, what=f"{how} {hint}")
    again = c.attend_chunk(q, cu, k, v, max_q=max(ql), max_len=int(c.len.max()), return_lse=True)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)  # the same bits on every run


LONG = [  # few rows on many keys: rows are cut along them
    (2, 1, 128, 64, BF16, [5000], [1]), (64, 8, 128, 64, F16, [9000, 300, 2000], [5, 5, 5]), (8, 8, 64, 32, F16, [3000, 40], [70, 900]),
    # parts that are longer than what is looked up at a time, and begin anywhere in it
    (32, 32, 64, 64, F16, [30000, 21111, 17000, 26001], [2, 1, 3, 2]), (32, 16, 64, 32, BF16, [24000, 9111, 17007], [3, 2, 1]),
    (16, 16, 64, 128, BF16, [60000, 41111, 57000, 36001], [2, 1, 3, 2]),
    (4, 2, 128, 128, BF16, [6017, 0], [130, 20]), (1, 1, 128, 32, F16, [12345], [300]), (8, 1, 64, 64, BF16, [20000, 1], [17, 200]),
]


@pytest.mark.parametrize("hq,hk,d,block,dt,lens,ql", LONG)
@pytest.mark.parametrize("how", ["new", "held"])
def test_cut_along_the_keys(hq, hk, d, block, dt, lens, ql, how):
    say(f"chunk cut {hq}/{hk}x{d} {block} {dt} {lens} {ql} {how}")
    c = make(len(lens), hk, d, block, dt, lens if how == "new" else [a + b for a, b in zip(lens, ql)])
    T, cu = sum(ql), starts(ql)
    q, k, v = rand((T, hq, d), dt, 4, 1.5), rand((T, hk, d), dt, 5), rand((T, hk, d), dt, 6)
    k, v = (k, v) if how == "new" else (None, None)
    most = int(c.len.max())
    assert m2c.m2c_kv_attend_chunk_workspace(c.desc, len(lens), T, hq, max(ql), most) > 0
    out, lse = c.attend_chunk(q, cu, k, v, max_q=max(ql), max_len=most, return_lse=True)
    check(c, q, cu, k, v, out, lse, what="cut")
    again = c.attend_chunk(q, cu, k, v, max_q=max(ql), max_len=most, return_lse=True)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    whole, wl = torch.empty_like(out), torch.empty_like(lse)  # without room for parts
    m2c.m2c_kv_attend_chunk(c.desc, None, len(lens), cu, T, hq, 0.0, q, q.stride()[:2], k, k.stride()[:2] if how == "new" else (0, 0), v,
                            v.stride()[:2] if how == "new" else (0, 0), whole, out.stride()[:2], wl)
    check(c, q, cu, k, v, whole, wl, what="whole")


def test_rows_without_keys():
    """A chunk of more tokens than the cache holds: its first see nothing."""
    say("chunk rows without keys")
    c = make(3, 2, 64, 32, F16, [40, 0, 3])
    cu = starts([100, 5, 3])
    q = rand((108, 4, 64), F16, 2)
    out, lse = c.attend_chunk(q, cu, return_lse=True)
    check(c, q, cu, None, None, out, lse)
    assert not out[:60].any() and bool((lse[:60] == -math.inf).all()) and not out[100:105].any()


def test_one_token_as_attend():
    """Of one token a chunk is what attend computes, and of a cache without tokens a prompt."""
    say("chunk as attend")
    c = make(5, 4, 128, 64, F16, [1, 64, 200, 639, 3000])
    q = rand((5, 16, 128), F16, 3)
    want, wl = c.attend(q, max_len=3000, return_lse=True)
    got, gl = c.attend_chunk(q, starts([1] * 5), max_q=1, max_len=3000, return_lse=True)
    check(c, q, starts([1] * 5), None, None, got, gl)
    assert float((gl - wl).abs().max()) <= 1e-5
    lens = [130, 1, 64]
    c = make(3, 2, 64, 64, BF16, [0, 0, 0])
    q, k, v = rand((195, 4, 64), BF16, 4), rand((195, 2, 64), BF16, 5), rand((195, 2, 64), BF16, 6)
    got = c.attend_chunk(q, starts(lens), k, v, max_q=130)
    assert torch.equal(got, prompt_attention(q, k, v, starts(lens), max_q=130)) or \
        float((got.float() - prompt_attention(q, k, v, starts(lens), max_q=130).float()).abs().max()) <= 2.0 ** -6
    check(c, q, starts(lens), k, v, got, None)


def test_lists_of_sequences():
    """In any order, some twice, rows of no sequence around them."""
    say("chunk lists")
    c = make(6, 2, 64, 32, BF16, [40, 0, 333, 64, 5, 130])
    seqs = torch.tensor([4, 2, 2, 0, 1], dtype=torch.int32, device="cuda")
    ql = [3, 40, 7, 0, 60]
    cu = starts(ql) + 11
    T = sum(ql) + 30
    q, k, v = rand((T, 4, 64), BF16, 2), rand((T, 2, 64), BF16, 3), rand((T, 2, 64), BF16, 4)
    out = torch.full_like(q, 9.0)
    got, lse = c.attend_chunk(q, cu, k, v, seqs=seqs, out=out, return_lse=True)
    assert got is out
    check(c, q, cu, k, v, out, lse, seqs=seqs)
    assert bool((out[:11] == 9).all()) and bool((out[11 + sum(ql):] == 9).all())


def test_many_sequences():
    say("chunk many sequences")
    lens, ql = [(37 * i) % 200 for i in range(150)], [(11 * i) % 9 for i in range(150)]
    c = make(150, 2, 64, 64, F16, lens)
    q, k, v = rand((sum(ql), 4, 64), F16, 2), rand((sum(ql), 2, 64), F16, 3), rand((sum(ql), 2, 64), F16, 4)
    out, lse = c.attend_chunk(q, starts(ql), k, v, return_lse=True)
    check(c, q, starts(ql), k, v, out, lse)


@pytest.mark.parametrize("layout", ["fused", "head_major", "padded", "shared_row"])
def test_strides(layout):
    hq, hk, d, ql = 4, 2, 128, [70, 64, 3]
    say(f"chunk strides {layout}")
    c = make(3, hk, d, 64, F16, [100, 0, 64])
    T = sum(ql)
    out = None
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
    else:
        q = rand((T, hq, d), F16, 12)
        k, v = (rand((T, 1, d), F16, 13 + i).expand(T, hk, d) for i in range(2))
        out = torch.zeros((T, hq, d), dtype=F16, device="cuda")
    whole = out._base if out._base is not None else out
    c.attend_chunk(q, starts(ql), k, v, out=out)
    check(c, q, starts(ql), k, v, out, None)
    mask = torch.ones_like(whole, dtype=torch.bool)
    mask.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((whole[mask] == 0).all())


@pytest.mark.parametrize("dt,d", [(F16, 128), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("long", [False, True])
def test_masked_values_do_not_enter(dt, d, what, long):
    """Of keys that some rows of the chunk see and some do not."""
    hq, hk, lens, ql = 4, 2, ([6000, 64] if long else [80, 64]), [150, 100]
    say(f"chunk masked {what} {long}")
    c = make(2, hk, d, 64, dt, lens)
    q, k, v = rand((250, hq, d), dt, 21), rand((250, hk, d), dt, 22), rand((250, hk, d), dt, 23)
    cu = starts(ql)
    clean = c.attend_chunk(q, cu, k, v)
    at = 77
    k2, v2 = k.clone(), v.clone()
    k2[at, :, 3], v2[at, :, 5], v2[at + 20] = what, what, what
    out = c.attend_chunk(q, cu, k2, v2)
    k3, v3 = k.clone(), v.clone()
    k3[at:150], v3[at:150] = 0, 0
    check(c, q[:at], starts([at]), k[:at], v[:at], out[:at], None)
    assert torch.equal(out[150:], clean[150:])
    assert not torch.isfinite(out[at + 20:150].float()).any()
    # values alone: rows that see it have it in its own place only
    v2 = v.clone()
    v2[at, 0, 5] = what
    out = c.attend_chunk(q, cu, k, v2)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[at:150, :hq // hk, 5] = False
    off = (out.float() - clean.float()).abs()[keep]
    assert not torch.isfinite(out[~keep].float()).any()
    assert float((off / (4 * U[dt] * (1 + clean.float().abs()[keep]))).max()) <= 1


@pytest.mark.parametrize("dt", [F16, BF16])
def test_blocks_that_are_no_numbers(dt):
    """A block with an infinity reads back as NaN: rows that see any of it are NaN,
    those before it are not, and nor are other heads and sequences."""
    say(f"chunk nan blocks {dt}")
    block, hk, d = 32, 2, 64
    c = KVCache(2, hk, d, 16, block_tokens=block, dtype=dt)
    k, v = rand((500, hk, d), dt, 1), rand((500, hk, d), dt, 2)
    k2, v2 = k.clone(), v.clone()
    k2[130, 0, 3], v2[300, 1, 9] = math.inf, math.nan
    cu = starts([400, 100])
    c.append(k2, v2, cu=cu)
    q = rand((500, 4, d), dt, 3)
    out, lse = c.attend_chunk(q, cu, return_lse=True)
    clean = KVCache(2, hk, d, 16, block_tokens=block, dtype=dt)
    clean.append(k, v, cu=cu)
    want = clean.attend_chunk(q, cu)
    check(clean, q, cu, None, None, want, None)
    same = torch.ones(500, 4, dtype=torch.bool, device="cuda")
    same[128:400, :2], same[288:400, 2:] = False, False
    assert bool(out[~same].isnan().all())
    assert torch.equal(out[same], want[same])


@pytest.mark.parametrize("dt,sizes", [(F16, (2e-7, 1e-4, 1.0, 60000.0)), (BF16, (1e-11, 1e-6, 1.0, 1e6, 1e11)), (BF16, (1e-36, 1e-37)), (BF16, (1e10, 1e30))])
@pytest.mark.parametrize("order", [1, -1])
def test_far_scales(dt, sizes, order):
    """Blocks of very different sizes, each with a row that sees little else."""
    say(f"chunk far scales {dt} {sizes} {order}")
    block, d, per = 32, 64, 2
    sizes = sizes[::order]
    n = block * per * len(sizes)
    c = KVCache(1, 1, d, 64, block_tokens=block, dtype=dt)
    k, v = torch.zeros((n, 1, d), dtype=dt, device="cuda"), rand((n, 1, d), F32, 2).clamp(-1, 1)
    for i, z in enumerate(sizes):
        part = slice(i * block * per, (i + 1) * block * per)
        k[part, 0, i] = 8.0
        v[part] *= z
    c.append(k, v.to(dt), cu=starts([n]))
    q = torch.zeros((len(sizes) + 1, 1, d), dtype=dt, device="cuda")
    for i in range(len(sizes)):
        q[i, 0, i] = 200.0  # scores of 200: other blocks have weights of e^-200
    # the chunk's own have no weight but for the last row, whose weights are all alike
    cu = starts([q.shape[0]])
    new_k, new_v = torch.zeros((q.shape[0], 1, d), dtype=dt, device="cuda"), (rand((q.shape[0], 1, d), F32, 3).clamp(-1, 1) * sizes[0]).to(dt)
    out, lse = c.attend_chunk(q, cu, new_k, new_v, return_lse=True)
    check(c, q, cu, new_k, new_v, out, lse, what=f"{sizes}")
    # the last row beside values of a size of their own, 2^-80 of which are the least that count apart
    new_v = rand((q.shape[0], 1, d), dt, 4)
    out, lse = c.attend_chunk(q, cu, new_k, new_v, return_lse=True)
    assert bool(torch.isfinite(out.float()).all())
    got, lg = c.attend_chunk(q[-1:], starts([1]), new_k[-1:], new_v[-1:], return_lse=True)
    check(c, q[-1:], starts([1]), new_k[-1:], new_v[-1:], got, lg, what=f"{sizes} beside 1")


F32 = torch.float32


def test_blocks_of_zeros_and_small_weights():
    say("chunk zeros")
    c = KVCache(1, 1, 64, 64, block_tokens=32, dtype=F16)
    k, v = rand((1000, 1, 64), F16, 1), rand((1000, 1, 64), F16, 2)
    k[32:96], v[64:128], v[0:32], k[320:352], v[320:352] = 0, 0, 0, 0, 0
    c.append(k, v, cu=starts([1000]))
    q = rand((30, 2, 64), F16, 3)
    out, lse = c.attend_chunk(q, starts([30]), return_lse=True)
    check(c, q, starts([30]), None, None, out, lse)
    # 20000 weights of 2^-20 beside one of 1
    n = 20000
    c = KVCache(1, 1, 64, 640, block_tokens=32, dtype=F16)
    k, v = torch.zeros((n, 1, 64), dtype=F16, device="cuda"), torch.ones((n, 1, 64), dtype=F16, device="cuda")
    k[5, 0, 0], v[5] = 13.86 * 8, -1.0
    c.append(k, v, cu=starts([n]))
    q = torch.zeros((1, 1, 64), dtype=F16, device="cuda")
    q[0, 0, 0] = 1.0
    out, lse = c.attend_chunk(q, starts([1]), return_lse=True)
    check(c, q, starts([1]), None, None, out, lse)


@pytest.mark.parametrize("dt,scale", [(F16, 1e-6), (F16, 3.0), (BF16, 1.0)])
def test_extreme_scores(dt, scale):
    say(f"chunk extreme scores {dt} {scale}")
    c = make(1, 2, 64, 64, dt, [400], sigma=20.0)
    q, k, v = rand((60, 2, 64), dt, 2, 20.0), rand((60, 2, 64), dt, 3, 20.0), rand((60, 2, 64), dt, 4)
    out, lse = c.attend_chunk(q, starts([60]), k, v, scale=scale, return_lse=True)
    check(c, q, starts([60]), k, v, out, lse, scale=scale)
    if dt == BF16:  # queries of any size of bf16
        for size, s in ((1e-30, 1e28), (1e20, 1e-21), (3e-38, 1e30)):
            q2 = (q.float() * size).to(dt)
            out, lse = c.attend_chunk(q2, starts([60]), k, v, scale=s, return_lse=True)
            check(c, q2, starts([60]), k, v, out, lse, scale=s, what=f"{size}")


def test_bad_indices():
    """Reported, and nothing else is touched."""
    say("chunk bad indices")
    c = make(4, 2, 64, 32, F16, [100, 70, 200, 0])
    q, k, v = rand((40, 4, 64), F16, 2), rand((40, 2, 64), F16, 3), rand((40, 2, 64), F16, 4)
    cu = starts([10, 10, 10, 10])
    want = c.attend_chunk(q, cu, k, v)
    c.check()
    seqs = torch.tensor([0, 4, 2, -1], dtype=torch.int32, device="cuda")
    out, lse = c.attend_chunk(q, cu, k, v, seqs=seqs, return_lse=True)
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG
    assert torch.equal(out[:10], want[:10]) and torch.equal(out[20:30], want[20:30])
    assert not out[10:20].any() and not out[30:].any() and bool((lse[30:] == -math.inf).all())
    # a page out of range is attended as zeros
    own = c.table[0, 0, 1:3].clone()
    c.table[0, 0, 1], c.table[0, 0, 2] = 1 << 30, -7
    out, lse = c.attend_chunk(q[:10], starts([10]), k[:10], v[:10], return_lse=True)
    with pytest.raises(m2c.M2CError):
        c.check()
    c.table[0, 0, 1:3] = own
    for n in ("k_codes", "v_codes"):
        getattr(c, n)[own.long()] = 0
    check(c, q[:10], starts([10]), k[:10], v[:10], out, lse)
    # starts that do not ascend
    bad = torch.tensor([0, 30, 12, 40, 5], dtype=torch.int32, device="cuda")
    out = torch.full((60, 4, 64), 3.0, dtype=F16, device="cuda")
    c.attend_chunk(q, bad, k, v, out=out[10:50])
    with pytest.raises(m2c.M2CError):
        c.check()
    assert bool((out[:10] == 3).all()) and bool((out[50:] == 3).all())


@pytest.mark.parametrize("long", [False, True])
def test_a_graph_and_another_stream(long):
    say(f"chunk graph {long}")
    lens, ql = ([4000, 900] if long else [70, 33]), [20, 9]
    c = make(2, 2, 128, 64, BF16, lens, spare=2)
    q, k, v = rand((29, 8, 128), BF16, 2), rand((29, 2, 128), BF16, 3), rand((29, 2, 128), BF16, 4)
    cu = starts(ql)
    out, lse = torch.empty_like(q), None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.attend_chunk(q, cu, k, v, stream=side)
    side.synchronize()
    check(c, q, cu, k, v, got, None)
    with torch.cuda.stream(side):
        c.attend_chunk(q, cu, k, v, out=out, max_len=max(lens))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend_chunk(q, cu, k, v, out=out, max_len=max(lens) + 100)
    for i in range(4):
        q.copy_(rand(q.shape, BF16, 20 + i))
        cu.copy_(torch.tensor([0, 20 - 5 * i, 29], dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = c.attend_chunk(q, cu, k, v, max_len=max(lens) + 100)
        assert torch.equal(out, want)
        c.append(k, v, cu=cu)  # the sequences grow between the replays
    c.check()


def test_a_run_of_them():
    """A prompt in chunks, turned, attended and appended, and then tokens: the rows
    that one prompt's attention over the same keys and values gives, but for what 8
    bits take from those before."""
    from paper_2410_14740_amd.attention import Rotary
    say("chunk run")
    hq, hk, d, n, block = 8, 2, 64, 700, 64
    f = torch.tensor([1e4 ** (-i / 32) for i in range(32)], dtype=torch.float32, device="cuda")
    r = Rotary(f)
    x = rand((n, hq + 2 * hk, d), F16, 1)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    qr, kr = r.rotate(q, at, k=k)
    want = prompt_attention(qr, kr, v, starts([n]))
    c = KVCache(1, hk, d, 16, block_tokens=block, dtype=F16)
    got, done = [], 0
    for m in (200, 1, 63, 300, 100, 30):
        part = slice(done, done + m)
        qq, kk = r.rotate(q[part], at[part], k=k[part])
        out = c.attend_chunk(qq, starts([m]), kk, v[part], max_q=m, max_len=done)
        check(c, qq, starts([m]), kk, v[part], out, None, what=f"chunk of {m}")
        c.append(kk, v[part], cu=starts([m]))
        got.append(out)
        done += m
    for t in range(done, n):
        qq, _ = c.append_rotated(r, k[t:t + 1], v[t:t + 1], at[t:t + 1], q=q[t:t + 1])
        got.append(c.attend(qq, max_len=t + 1))
    c.check()
    off = (torch.cat(got).float() - want.float()).square().mean().sqrt() / want.float().square().mean().sqrt()
    assert float(off) <= 0.02  # codes are off by half a 254th of a block's largest: rms 0.9% of the keys' and values'


@pytest.mark.parametrize("call,needle", [
    (lambda c, q, cu: c.attend_chunk(q, cu, k=q[:, :2]), "k and v"), (lambda c, q, cu: c.attend_chunk(q, cu, q[:, :2], q[:4, :2]), "k, v"),
    (lambda c, q, cu: c.attend_chunk(q, cu, q[:, :1], q[:, :1]), "k:"), (lambda c, q, cu: c.attend_chunk(q, cu.long()), "cu"),
    (lambda c, q, cu: c.attend_chunk(q, cu, seqs=cu), "seqs"), (lambda c, q, cu: c.attend_chunk(q.float(), cu), "q:"),
    (lambda c, q, cu: c.attend_chunk(q[:, :3], cu), "n_heads"), (lambda c, q, cu: c.attend_chunk(q, cu, out=q[:5]), "out"),
    (lambda c, q, cu: c.attend_chunk(q, cu, max_q=-1), "max_q"), (lambda c, q, cu: c.attend_chunk(q[0], cu), "q:"),
])
def test_refusals(call, needle):
    c = KVCache(2, 2, 64, 4)
    with pytest.raises(m2c.M2CError) as e:
        call(c, torch.zeros((6, 4, 64), dtype=F16, device="cuda"), starts([2, 4]))
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


@pytest.mark.parametrize("new", [False, True])
def test_pages_past_32_bits(new):
    """Pages whose byte offsets do not fit 32 bits."""
    say(f"chunk pages past 32 bits {new}")
    hk, d, n_pages = 2, 128, (1 << 19) + 64  # 8 KB of codes a page
    c = KVCache(1, hk, d, 8, n_pages=n_pages, dtype=F16)
    c.table.copy_(torch.arange(n_pages - 16, n_pages, dtype=torch.int32, device="cuda").flip(0).view_as(c.table))
    c.append(rand((500, hk, d), F16, 2), rand((500, hk, d), F16, 3), cu=starts([500]))
    q, k, v = rand((37, 4, d), F16, 4), rand((37, hk, d), F16, 5), rand((37, hk, d), F16, 6)
    if not new:
        k = v = None
    out, lse = c.attend_chunk(q, starts([37]), k, v, return_lse=True)
    c.check()
    check(c, q, starts([37]), k, v, out, lse)


def test_a_full_cache():
    """A sequence at the end of its blocks, and a chunk behind it that would not fit."""
    say("chunk full cache")
    c = make(2, 2, 64, 64, BF16, [256, 255])
    q, k, v = rand((80, 4, 64), BF16, 2), rand((80, 2, 64), BF16, 3), rand((80, 2, 64), BF16, 4)
    cu = starts([70, 10])
    for kv in ((k, v), (None, None)):
        out, lse = c.attend_chunk(q, cu, *kv, return_lse=True)
        check(c, q, cu, *kv, out, lse)
    c.check()


def test_two_calls_at_once():
    """Calls on two streams, whose rows are cut, over one cache, as one after another."""
    say("chunk two at once")
    c = make(2, 2, 128, 64, F16, [6000, 900])
    cu, calls = starts([20, 9]), []
    for i in range(2):
        q, k, v = (rand((29, h, 128), F16, 10 * i + j) for j, h in enumerate((8, 2, 2)))
        calls.append((q, k, v, c.attend_chunk(q, cu, k, v)))
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[c.attend_chunk(*call[:1], cu, *call[1:3], stream=s) for s, call in zip(sides, calls)] for _ in range(20)]
    torch.cuda.synchronize()
    for pair in got:
        for out, call in zip(pair, calls):
            assert torch.equal(out, call[3])
    check(c, calls[0][0], cu, calls[0][1], calls[0][2], calls[0][3], None)

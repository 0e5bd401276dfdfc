"""Rotation by positions, and the append that rotates, against complex products
in 64 bits.

Tolerances. A cosine or sine: the fraction of a turn rounded to fp32 (2^-25 of a
turn, 2^-22.3 radians) and the hardware's function (2^-22.9), together 2^-21.6; the
scale and each product and sum a unit of 2^-24 more: 2^-21 (|a| + |b|) for a pair
(a, b). The angle itself is taken in 64 bits, three roundings: |angle| 2^-51 (|a| +
|b|). The output's own rounding adds 2^-11 (fp16, whose smallest number is 2^-24)
or 2^-8 (bf16) of its value."""
import math

import numpy as np
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import m2c
from paper_2410_14740_amd.attention import KVCache, Rotary

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8}


def rand(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def freqs(rot, base=1e4):
    return torch.tensor([base ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float32, device="cuda")


def starts(lens):
    return torch.tensor(np.cumsum([0, *lens]), dtype=torch.int32, device="cuda")


def turned64(x, freq, positions, sections, inter, scale=1.0):
    """Rows turned, in 64 bits, and how far ours may be off."""
    rot = 2 * freq.shape[0]
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = positions.view(len(sections), -1)[torch.from_numpy(axis).cuda()].double().t() * freq.double()
    turn = torch.complex(angle.cos(), angle.sin())[:, None]
    y, off = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    a = slice(0, rot, 2) if inter else slice(0, rot // 2)
    b = slice(1, rot, 2) if inter else slice(rot // 2, rot)
    z = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * turn * scale
    size = (y[..., a].abs() + y[..., b].abs()) * abs(scale) * (2.0 ** -21 + angle.abs()[:, None] * 2.0 ** -51)
    y[..., a], y[..., b] = z.real, z.imag
    off[..., a], off[..., b] = size, size
    return y, off


def check(got, x, freq, positions, sections, inter, scale=1.0, what=""):
    want, off = turned64(x, freq, positions, sections, inter, scale)
    bound = off + U[x.dtype] * want.abs() + (2.0 ** -24 if x.dtype == F16 else 0.0)
    bad = (got.double() - want).abs() / bound.clamp(min=1e-300)
    assert bool((bad <= 1).all()), f"{what}: off by {float(bad.max()):.2f} of its bound"
    rot = 2 * freq.shape[0]
    assert torch.equal(got[..., rot:], x[..., rot:])


CASES = [  # heads, kv heads, width, rotated, sections, interleaved, tokens
    (1, 1, 64, 16, [8], False, 1), (1, 1, 64, 16, [8], True, 1), (2, 1, 64, 64, [32], False, 3), (3, 3, 128, 128, [64], True, 4),
    (64, 8, 128, 128, [16, 24, 24], False, 5), (64, 8, 128, 128, [16, 24, 24], True, 33), (8, 8, 128, 48, [1, 22, 0, 1], False, 130),
    (5, 1, 64, 48, [7, 17], True, 1000), (40, 40, 128, 112, [56], False, 77), (7, 1, 128, 96, [0, 48], False, 2049),
    (1024, 1, 64, 32, [16], False, 2), (16, 2, 128, 80, [13, 14, 13], True, 515),
]


@pytest.mark.parametrize("hq,hk,d,rot,sections,inter,n", CASES)
@pytest.mark.parametrize("dt", [F16, BF16])
def test_rotate(hq, hk, d, rot, sections, inter, n, dt):
    say(f"rotate {hq}/{hk}x{d} {rot} {sections} {inter} {n} {dt}")
    q, k = rand((n, hq, d), dt, 1, 2.0), rand((n, hk, d), dt, 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    pos = torch.randint(-5, 4000, (len(sections), n), generator=g, device="cuda", dtype=torch.int32)
    f = freqs(rot)
    r = Rotary(f, sections=sections, interleaved=inter)
    qo, ko = r.rotate(q, pos, k=k)
    check(qo, q, f, pos, sections, inter, what="q")
    check(ko, k, f, pos, sections, inter, what="k")
    assert torch.equal(r.rotate(q, pos), qo)  # queries alone, the same bits
    q2, k2 = q.clone(), k.clone()
    r.rotate(q2, pos, k=k2, q_out=q2, k_out=k2)  # in place
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    if len(sections) == 1:
        assert torch.equal(r.rotate(q, pos[0]), qo)


@pytest.mark.parametrize("far", [1 << 17, 1 << 24, (1 << 31) - 3000])
@pytest.mark.parametrize("inter", [False, True])
def test_far_positions(far, inter):
    say(f"rotate far {far}")
    q = rand((200, 4, 128), F16, 1)
    for at in (far, -far):
        pos = (torch.arange(200, device="cuda") + at).int()
        f = freqs(128)
        check(Rotary(f, interleaved=inter).rotate(q, pos), q, f, pos, [64], inter, what=f"{at}")


def test_scale_and_frequencies():
    say("rotate scale")
    q, pos = rand((50, 3, 64), BF16, 1), torch.arange(50, dtype=torch.int32, device="cuda")
    for scale in (0.5, -2.25, 1e-3):
        f = freqs(64, 1e6) * 8.0
        check(Rotary(f, scale=scale).rotate(q, pos), q, f, pos, [32], False, scale)
    f = torch.zeros(32, device="cuda")
    assert torch.equal(Rotary(f).rotate(q, pos), q)  # no angle: the same bits
    one = rand((50, 3, 64), F16, 2)
    one[7, 1, 3], one[7, 1, 40] = math.inf, math.nan
    f = freqs(64)
    got, want = Rotary(f).rotate(one, pos), Rotary(f).rotate(torch.nan_to_num(one, 0, 0, 0), pos)
    hit = torch.zeros_like(one, dtype=torch.bool)
    hit[7, 1, [3, 35, 8, 40]] = True
    assert torch.equal(got[~hit], want[~hit]) and not torch.isfinite(got[hit]).any()


@pytest.mark.parametrize("inter", [False, True])
def test_strides(inter):
    say(f"rotate strides {inter}")
    n, hq, hk, d = 37, 6, 2, 64
    f, pos = freqs(64), torch.arange(n, dtype=torch.int32, device="cuda").repeat(2, 1)
    pos[1] *= 3
    wide = torch.zeros((2, n + 9), dtype=torch.int32, device="cuda")
    wide[:, 4:4 + n] = pos
    pos = wide[:, 4:4 + n]
    r = Rotary(f, sections=[20, 12], interleaved=inter)
    x = rand((n, hq + 2 * hk, d), F16, 1)  # rows of a fused projection, in place
    q, k = x[:, :hq], x[:, hq:hq + hk]
    before = x.clone()
    want = r.rotate(q, pos, k=k)
    r.rotate(q, pos, k=k, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, hq + hk:], before[:, hq + hk:])
    check(q, before[:, :hq], f, pos, [20, 12], inter)
    t = rand((hq, n, d + 24), F16, 2)[:, :, 8:8 + d].transpose(0, 1)  # head major, padded
    out = torch.zeros((n, hq + 3, d + 8), dtype=F16, device="cuda")[:, 1:1 + hq, :d]
    r.rotate(t, pos, q_out=out)
    check(out, t, f, pos, [20, 12], inter)
    base = out._base
    base[:, 1:1 + hq, :d] = 0
    assert not base.any()
    shared = rand((n, 1, d), F16, 3).expand(n, hk, d)  # one key for all heads
    check(r.rotate(q, pos, k=shared)[1], shared, f, pos, [20, 12], inter)


def state(c):
    return {n: getattr(c, n).clone() for n in ("k_codes", "v_codes", "k_scale", "v_scale", "tail_k", "tail_v", "len", "weight")}


def fill(c, lens, seed):
    """A cache with some tokens in it, its unused places with something known."""
    for i, n in enumerate(("k_codes", "v_codes", "tail_k", "tail_v")):
        getattr(c, n).fill_(7)
    for n in ("k_scale", "v_scale", "weight"):
        getattr(c, n).fill_(3.0)
    k = rand((sum(lens), c.n_kv_heads, c.head_dim), c.dtype, seed)
    if k.shape[0]:
        c.append(k, -k, cu=starts(lens))


APPENDS = [  # kv heads, heads, width, rotated, sections, interleaved, block, type, lengths held, new ones
    (2, 4, 64, 64, [32], False, 64, F16, [0, 0, 0], [1, 64, 130]),
    (1, 1, 128, 128, [64], False, 32, BF16, [5, 31, 32, 33], [27, 1, 0, 95]),
    (8, 64, 128, 128, [16, 24, 24], False, 64, BF16, [100, 0], [300, 63]),
    (3, 6, 128, 96, [20, 28], True, 128, F16, [127, 128, 1], [1, 128, 300]),
    (2, 2, 64, 16, [8], True, 32, F16, [10], [500]),
    (4, 8, 128, 48, [24], False, 64, F16, [63, 64, 65, 0], [1, 1, 1, 1]),
    (40, 40, 128, 128, [64], True, 64, BF16, [0], [70]),
]


@pytest.mark.parametrize("hk,hq,d,rot,sections,inter,block,dt,held,new", APPENDS)
@pytest.mark.parametrize("with_q,with_k", [(True, True), (False, False)])
def test_append_rotated(hk, hq, d, rot, sections, inter, block, dt, held, new, with_q, with_k):
    """To the bit what rotating first and appending then leaves."""
    say(f"append rotated {hk}/{hq}x{d} {rot} {sections} {inter} {block} {dt} {held} {new} {with_q}")
    n, T = len(held), sum(new)
    caches = [KVCache(n, hk, d, 16, block_tokens=block, dtype=dt) for _ in range(2)]
    for c in caches:
        fill(c, held, 5)
    x = rand((T, hq + 2 * hk, d), dt, 6, 2.0)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    pos = torch.randint(0, 5000, (len(sections), T), generator=g, device="cuda", dtype=torch.int32)
    f = freqs(rot)
    r = Rotary(f, sections=sections, interleaved=inter)
    qr, kr = r.rotate(q, pos, k=k)
    caches[0].append(kr, v, cu=starts(new))
    qo, ko = caches[1].append_rotated(r, k, v, pos, q=q if with_q else None, cu=starts(new), k_out=True if with_k else None)
    caches[1].check()
    a, b = state(caches[0]), state(caches[1])
    for name in a:
        assert torch.equal(a[name], b[name]), name
    assert torch.equal(qo, qr) if with_q else qo is None
    assert torch.equal(ko, kr) if with_k else ko is None
    check(kr, k, f, pos, sections, inter)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("inter", [False, True])
def test_append_rotated_token_by_token(block, inter):
    say(f"append rotated tokens {block} {inter}")
    n, hk, hq, d = 5, 2, 8, 64
    caches = [KVCache(n, hk, d, 8, block_tokens=block, dtype=F16) for _ in range(3)]
    r = Rotary(freqs(64), interleaved=inter)
    for c in caches:
        fill(c, [0, 3, block - 2, block - 1, 2 * block - 3], 1)
    steps = 6
    x = rand((steps, n, hq + 2 * hk, d), F16, 2)
    at = torch.tensor([0, 3, block - 2, block - 1, 2 * block - 3], device="cuda").int()
    for t in range(steps):
        q, k, v = x[t, :, :hq], x[t, :, hq:hq + hk], x[t, :, hq + hk:]
        qr, kr = r.rotate(q, at + t, k=k)
        caches[0].append(kr, v)
        q1, k1 = caches[1].append_rotated(r, k, v, at + t, q=q, k_out=True)
        own = q.clone()
        q2, k2 = caches[2].append_rotated(r, k, v, at + t, q=own, q_out=own, pos=caches[2].len.clone())
        assert q2 is own and k2 is None and torch.equal(own, qr) and torch.equal(q1, qr) and torch.equal(k1, kr)
    for c in caches[1:]:
        c.check()
        for name, t in state(caches[0]).items():
            assert torch.equal(t, state(c)[name]), name


def test_append_rotated_lists_places_and_refusals():
    """Sequences out of order, rewinds, a full one and one at no place of its
    own; rows of no sequence."""
    say("append rotated lists")
    n, hk, hq, d, block = 6, 2, 4, 64, 32
    held = [40, 70, 64, 0, 100, 128]
    caches = [KVCache(n, hk, d, 4, block_tokens=block, dtype=BF16) for _ in range(2)]
    for c in caches:
        fill(c, held, 1)
    new = [30, 0, 7, 40, 3]
    seqs = torch.tensor([4, 0, 1, 3, 5], dtype=torch.int32, device="cuda")
    pos = torch.tensor([96, 9, 20, 0, 128], dtype=torch.int32, device="cuda")  # the third at no place, the last is full
    T = sum(new)
    q, k, v = (rand((T + 9, h, d), BF16, 2 + i) for i, h in enumerate((hq, hk, hk)))
    cu = starts(new) + 4  # four rows before and five behind belong to nobody
    at = torch.arange(T + 9, dtype=torch.int32, device="cuda")
    r = Rotary(freqs(32))
    qr, kr = r.rotate(q, at, k=k)
    caches[0].append(kr, v, cu=cu, seqs=seqs, pos=pos)
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    caches[1].append_rotated(r, k, v, at, q=q, cu=cu, seqs=seqs, pos=pos, q_out=qo, k_out=ko)
    statuses = []
    for c in caches:
        with pytest.raises(m2c.M2CError) as e:
            c.check()
        statuses.append(str(e.value))
    assert statuses[0] == statuses[1]
    for name, t in state(caches[0]).items():
        assert torch.equal(t, state(caches[1])[name]), name
    inside = slice(4, 4 + T)
    assert torch.equal(qo[inside], qr[inside]) and bool((qo[:4] == 5).all()) and bool((qo[4 + T:] == 5).all())
    written = torch.zeros(T + 9, dtype=torch.bool, device="cuda")
    written[4:34] = True
    written[41:81] = True  # the refused ones' rows stay
    assert torch.equal(ko[written], kr[written]) and bool((ko[~written] == 5).all())


def test_append_rotated_in_a_graph():
    say("append rotated graph")
    n, hk, hq, d = 4, 2, 8, 128
    c, other = (KVCache(n, hk, d, 8, block_tokens=32, dtype=F16) for _ in range(2))
    for x in (c, other):
        fill(x, [5, 31, 40, 63], 1)
    r = Rotary(freqs(128))
    x = rand((n, hq + 2 * hk, d), F16, 2)
    at = torch.tensor([5, 31, 40, 63], dtype=torch.int32, device="cuda")
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    out = torch.empty((n, hq, d), dtype=F16, device="cuda")
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r.rotate(q, at)  # torch's first use of the stream outside the capture
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.append_rotated(r, k, v, at, q=q, q_out=out)
        at += 1
    for t in range(70):
        x.copy_(rand(x.shape, F16, 50 + t))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want, _ = other.append_rotated(r, k, v, at - 1, q=q)
        assert torch.equal(out, want)
    c.check()
    for name, t in state(other).items():
        assert torch.equal(t, state(c)[name]), name


@pytest.mark.parametrize("call,needle", [
    (lambda r, c, q, p: r.rotate(q, p[:1]), "positions"), (lambda r, c, q, p: r.rotate(q, p.long()), "positions"),
    (lambda r, c, q, p: r.rotate(q, p.cpu()), "positions"), (lambda r, c, q, p: r.rotate(q, p[:, :3]), "positions"),
    (lambda r, c, q, p: r.rotate(q, p.t().contiguous().t()), "positions"),
    (lambda r, c, q, p: r.rotate(q, p, k=q[:3]), "k:"), (lambda r, c, q, p: r.rotate(q, p, k_out=q), "k_out"),
    (lambda r, c, q, p: r.rotate(q, p, q_out=q[:, :1]), "q_out"), (lambda r, c, q, p: r.rotate(q[..., :32], p), "head_dim"),
    (lambda r, c, q, p: r.rotate(q.float(), p), "q:"), (lambda r, c, q, p: r.rotate(q, p, k=q.bfloat16()), "k:"),
    (lambda r, c, q, p: c.append_rotated(r, q, q, p, k_out=q), "k_out is k"), (lambda r, c, q, p: c.append_rotated(r, q, q, p, q_out=q), "q_out"),
    (lambda r, c, q, p: c.append_rotated(r, q, q[:3], p), "v:"), (lambda r, c, q, p: c.append_rotated(r, q, q, p, q=q[:3]), "q:"),
    (lambda r, c, q, p: Rotary(r.freq[:20]), "pairs"), (lambda r, c, q, p: Rotary(r.freq, sections=[30]), "sections"),
    (lambda r, c, q, p: Rotary(r.freq, scale=0.0), "scale"), (lambda r, c, q, p: Rotary(r.freq.half()), "freq"),
])
def test_refusals(call, needle):
    r = Rotary(freqs(64), sections=[20, 12])
    c = KVCache(4, 2, 64, 4)
    q, p = torch.zeros((4, 2, 64), dtype=F16, device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(m2c.M2CError) as e:
        call(r, c, q, p)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_more_tokens_than_a_grid_has_threads():
    """2^26 tokens and some: a workgroup of 256 threads for every four would be 2^32."""
    n, R = (1 << 26) + 5, Rotary(freqs(16))
    q = torch.empty(n, 1, 64, dtype=F16, device="cuda")
    q[:-4096] = 1.0
    q[-4096:] = rand((4096, 1, 64), F16, 92)
    p = torch.zeros(n, dtype=torch.int32, device="cuda")
    p[-4096:] = torch.arange(4096, dtype=torch.int32, device="cuda")
    want = R.rotate(q[-4096:], p[-4096:])
    R.rotate(q, p, q_out=q)
    assert torch.equal(q[-4096:], want)
    assert q[:-4096].min().item() == 1.0 == q[:-4096].max().item()


def test_heads_far_apart():
    """Heads whose byte offsets do not fit 32 bits, turned in place."""
    n, R, step = 9, Rotary(freqs(64)), (1 << 30) + 64
    buf = torch.empty(2 * step + n * 64, dtype=F16, device="cuda")
    q = buf.as_strided((n, 3, 64), (64, step, 1))
    q.copy_(rand((n, 3, 64), F16, 93))
    p = torch.arange(n, dtype=torch.int32, device="cuda")
    want = R.rotate(q.contiguous(), p)
    assert torch.equal(R.rotate(q, p, q_out=q), want)

"""The residual stream's norms against a plain implementation in 64 bits.

Tolerances. All arithmetic is fp32 (unit 2^-24). With up to 64 elements of a row
in a thread and 22 steps of joining, a sum of like terms is off by at most 86
units, 2^-17.5 of the sum of magnitudes; a factor 1 / sqrt by half of its sum's and
a unit or two. So N(z), with a = 1 / sqrt(mean square + eps) and M = a mean |z|
(of the mean that "layer" takes off), is off by at most e (1 + |N(z)| + M), e =
2^-16, and by a (dz + mean dz + |N(z)| rms dz) for errors dz of z itself. r is off by
2^-22 (|x| + |s g t|), and by |s g| times the error of t. An output's own rounding
adds u |value|: 2^-24, 2^-11 (fp16, whose smallest number is 2^-24) or 2^-8 (bf16)."""
import math

import pytest
import torch

from helpers import say
from paper_2410_14740_amd import m2c
from paper_2410_14740_amd.norms import residual_norm

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
E = 2.0 ** -16


def rand(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def normed64(z, dz, w, b, kind, eps):
    """N(z) w + b in 64 bits, and how far it may be off where z is by dz."""
    mean = z.mean(1, keepdim=True) if kind == "layer" else 0.0
    a = 1.0 / ((z - mean).square().mean(1, keepdim=True) + eps).sqrt()
    n = (z - mean) * a
    off = E * (1 + n.abs() + (a * z.abs().mean(1, keepdim=True) if kind == "layer" else 0.0))
    off = off + a * (dz + dz.mean(1, keepdim=True) + n.abs() * dz.square().mean(1, keepdim=True).sqrt())
    w = torch.ones_like(z) if w is None else w.double().expand_as(z)
    b = torch.zeros_like(z) if b is None else b.double().expand_as(z)
    return n * w + b, off * w.abs() + 2.0 ** -23 * b.abs()


def check(x, y, r, out, weight=None, bias=None, post=False, post_weight=None, post_bias=None, gate=None,
          scale=1.0, kind="rms", eps=1e-5, what=""):
    want, dr = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    if y is not None:
        t, dt = y.double(), torch.zeros_like(want)
        if post:
            t, dt = normed64(t, dt, post_weight, post_bias, kind, eps)
        sg = (scale * (gate.double() if gate is not None else 1.0) * torch.ones_like(want))
        want = want + sg * t
        dr = 2.0 ** -22 * (x.double().abs() + (sg * t).abs()) + sg.abs() * dt
    tiny = lambda t: 2.0 ** -24 if t.dtype == F16 else 0.0  # noqa: E731
    if r is not None:
        bound = dr + U[r.dtype] * want.abs() + tiny(r)
        bad = (r.double() - want).abs() / bound.clamp(min=1e-300)
        assert bool((bad <= 1).all()), f"{what}: stream off by {float(bad.max()):.2f} of its bound"
    if out is not None:
        o, do = normed64(want, dr, weight, bias, kind, eps)
        bound = do + U[out.dtype] * o.abs() + tiny(out)
        bad = (out.double() - o).abs() / bound.clamp(min=1e-300)
        assert bool((bad <= 1).all()), f"{what}: norm off by {float(bad.max()):.2f} of its bound"


WIDTHS = [1, 2, 7, 8, 63, 64, 65, 511, 512, 520, 1000, 1024, 1032, 2047, 4096, 5120, 8192, 10000, 16384, 16392, 20001,
          32768, 65528, 65535, 65536]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_widths(d, kind):
    say(f"norm width {d} {kind}")
    x, y = rand((3, d), F32, d, 2.0) + 0.5, rand((3, d), F16, d + 1)
    w, pw, b, pb = (1 + rand((d,), F32, i, 0.2) for i in range(4))
    args = dict(kind=kind, weight=w, bias=b, post=True, post_weight=pw, post_bias=pb, scale=0.7)
    r, out = residual_norm(x, y, **args)
    assert r.dtype == F32 and out.dtype == F16
    check(x, y, r, out, what=f"{d}", **args)
    again = residual_norm(x, y, **args)
    assert torch.equal(again[0], r) and torch.equal(again[1], out)


TYPES = [(x, y, o, w) for h in (F16, BF16) for x in (F32, h) for y in (F32, h) for o in (F32, h) for w in (F32, h)]


@pytest.mark.parametrize("xt,yt,ot,wt", TYPES)
@pytest.mark.parametrize("d", [96, 1032, 17000, 301])
def test_types(xt, yt, ot, wt, d):
    say(f"norm types {xt} {yt} {ot} {wt} {d}")
    x, y = rand((5, d), xt, 1, 3.0), rand((5, d), yt, 2)
    w, g, pb = 1 + rand((d,), wt, 3, 0.2), rand((5, d), wt, 4), rand((d,), wt, 5)
    args = dict(weight=w, gate=g, post=True, post_bias=pb, kind="layer")
    r, out = residual_norm(x, y, out_dtype=ot, **args)
    assert r.dtype == xt and out.dtype == ot
    check(x, y, r, out, what=f"{xt} {yt} {ot} {wt} {d}", **args)


@pytest.mark.parametrize("rows,d", [(1, 1024), (1, 8192), (1023, 512), (1024, 512), (1027, 512), (1030, 40), (300, 8192), (5000, 33)])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
def test_rows_and_gates(rows, d, gate):
    say(f"norm rows {rows} {d} {gate}")
    x, y = rand((rows, d), BF16, 1), rand((rows, d), BF16, 2)
    g = {"none": None, "channel": rand((d,), BF16, 3), "row": rand((rows, d), BF16, 4)}[gate]
    r, out = residual_norm(x, y, gate=g, scale=-1.5)
    check(x, y, r, out, gate=g, scale=-1.5, what=f"{rows} {d} {gate}")


def test_parts_of_the_call():
    say("norm parts")
    x, y, w = rand((9, 264), F32, 1), rand((9, 264), F16, 2), rand((264,), F32, 3)
    r, out = residual_norm(x, weight=w)  # the norm alone
    assert r is x and out.dtype == F16
    check(x, None, None, out, weight=w)
    r, out = residual_norm(x, y, norm=False)  # the stream alone
    assert out is None
    check(x, y, r, None)
    copy = torch.empty_like(x)
    r, out = residual_norm(x, x_out=copy)  # a copy beside the norm
    assert r is copy and torch.equal(copy, x)
    assert residual_norm(x, norm=False) == (x, None)
    assert residual_norm(x.half())[1].dtype == F16 and residual_norm(x, out_dtype=F32)[1].dtype == F32
    assert residual_norm(x[:0], y[:0])[1].shape == (0, 264)
    for zero in (0.0, -0.0):
        r, _ = residual_norm(x, y, scale=zero)
        assert torch.equal(r, x)


@pytest.mark.parametrize("d", [264, 261])
def test_in_place(d):
    say(f"norm in place {d}")
    x, y = rand((33, d), F32, 1), rand((33, d), F16, 2)
    want = residual_norm(x, y)
    own = x.clone()
    r, out = residual_norm(own, y, x_out=own)
    assert r is own and torch.equal(own, want[0]) and torch.equal(out, want[1])


@pytest.mark.parametrize("d", [128, 4096, 77])
def test_strides(d):
    """Rows of wider arrays, on starts that are and are not 16-byte aligned, and
    one row for all."""
    say(f"norm strides {d}")
    for shift, pad in ((8, 24), (1, 3), (0, 5), (4, 64)):
        big = [rand((6, d + shift + pad), t, i) for i, t in enumerate((F16, F16, F16, F16, F16))]
        x, y, g, ro, oo = (t[:, shift:shift + d] for t in big)
        before = [t.clone() for t in big]
        w = rand((d + 8,), F16, 9)[shift % 8:shift % 8 + d]
        r, out = residual_norm(x, y, weight=w, gate=g, x_out=ro, out=oo)
        assert r is ro and out is oo
        check(x, y, r, out, weight=w, gate=g, what=f"{shift} {pad}")
        for i in (0, 1, 2):
            assert torch.equal(big[i], before[i])
        for t, b in ((big[3], before[3]), (big[4], before[4])):  # nothing beside the rows
            assert torch.equal(t[:, :shift], b[:, :shift]) and torch.equal(t[:, shift + d:], b[:, shift + d:])
    one = rand((1, d), F16, 11).expand(6, d)
    r, out = residual_norm(rand((6, d), F16, 12), one)
    check(rand((6, d), F16, 12), one, r, out)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", [1e30, 1e25, 1e18, 1e-18, 1e-25, 1e-37])
def test_far_sizes(kind, size):
    """Squares that leave fp32's range, both ways, without eps."""
    say(f"norm size {size} {kind}")
    for d in (72, 3000):
        x = rand((4, d), F32, 1) * size
        _, out = residual_norm(x, kind=kind, eps=0.0, out_dtype=F32)
        check(x, None, None, out, kind=kind, eps=0.0, what=f"{size}")
        y = rand((4, d), BF16, 2) * size
        r, out = residual_norm(torch.zeros_like(x), y, post=True, kind=kind, eps=0.0)
        check(torch.zeros_like(x), y, r, out, post=True, kind=kind, eps=0.0, what=f"post {size}")


def test_rows_that_are_no_numbers_stay_alone():
    say("norm nan rows")
    x, y = rand((1500, 320), F32, 1), rand((1500, 320), F16, 2)
    want, wn = residual_norm(x, y, post=True)
    x2, y2 = x.clone(), y.clone()
    x2[3, 5], y2[700, 0], x2[1499, 319], y2[8] = math.nan, math.inf, -math.inf, 0
    r, out = residual_norm(x2, y2, post=True)
    keep = torch.ones(1500, dtype=torch.bool, device="cuda")
    keep[torch.tensor([3, 700, 1499, 8], device="cuda")] = False
    assert torch.equal(r[keep], want[keep]) and torch.equal(out[keep], wn[keep])
    assert torch.equal(r[8], x[8]) and bool(torch.isfinite(out[8]).all())  # a row of zeros is normed to zeros
    assert bool(out[3].isnan().all())
    # 1 / sqrt(inf) is 0: the infinity itself becomes NaN, the rest zeros
    assert bool(r[700, 0].isnan()) and bool(out[700].isnan().all())
    assert bool(out[1499, 319].isnan()) and bool((out[1499, :319] == 0).all())


def test_layer_of_a_constant_row():
    say("norm constant row")
    x = torch.full((2, 777), 3.0, device="cuda")
    _, out = residual_norm(x, kind="layer", out_dtype=F32)
    check(x, None, None, out, kind="layer")


def test_another_stream_and_a_graph():
    say("norm graph")
    x, y, w = rand((70, 1032), F32, 1), rand((70, 1032), F16, 2), rand((1032,), F32, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r, out = residual_norm(x, y, weight=w, post=True, stream=side)
    side.synchronize()
    check(x, y, r, out, weight=w, post=True)
    with torch.cuda.stream(side):
        residual_norm(x, y, weight=w, post=True, x_out=r, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        residual_norm(x, y, weight=w, post=True, x_out=r, out=out)
    for i in range(4):
        x.copy_(rand(x.shape, F32, 20 + i))
        r.zero_(), out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = residual_norm(x, y, weight=w, post=True)
        assert torch.equal(r, want[0]) and torch.equal(out, want[1])


@pytest.mark.parametrize("kw,needle", [
    (dict(y=(4, 63)), "y:"), (dict(weight=(63,)), "weight:"), (dict(gate=(3, 64)), "gate:"), (dict(kind="max"), "kind"),
    (dict(post=True), "y is NULL"), (dict(weight=(64,), bias=(64,), bias_type=F16), "bias:"), (dict(out=(4, 32)), "out:"),
    (dict(out_dtype=torch.int32), "out_dtype"), (dict(eps=-1.0), "eps"), (dict(norm=False, weight=(64,)), "norm False"),
    (dict(y=(4, 64), y_type=BF16, out_dtype=F16), "16-bit"), (dict(x_out=(4, 64), x_out_type=F16), "x_out"),
])
def test_refusals(kw, needle):
    args = {}
    for name, v in kw.items():
        if not name.endswith("_type"):
            args[name] = torch.zeros(v, dtype=kw.get(name + "_type", F32), device="cuda") if isinstance(v, tuple) else v
    with pytest.raises(m2c.M2CError) as e:
        residual_norm(torch.zeros((4, 64), device="cuda"), **args)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and needle in str(e.value)


def test_more_rows_than_a_grid_has_threads():
    """2^26 rows and some: 64 threads for each would be 2^32."""
    n, d = (1 << 26) + 3, 8
    x = torch.empty(n, d, dtype=F16, device="cuda")
    x[:4096] = rand((4096, d), F16, 90)
    x[4096:] = 1.0
    x[-4096:] = rand((4096, d), F16, 91)
    x_out, out = torch.empty_like(x), torch.zeros_like(x)
    residual_norm(x, weight=None, x_out=x_out, out=out)
    assert torch.equal(x_out, x)
    for rows in (slice(0, 4096), slice(n - 4096, n)):
        assert torch.equal(out[rows], residual_norm(x[rows])[1])
    mid = out[4096:-4096]
    assert torch.equal(mid, mid[:1].expand_as(mid)) and mid[0, 0].item() == 1.0


def test_rows_far_apart():
    """Rows whose byte offsets do not fit 32 bits."""
    d, step = 264, (1 << 30) + 8
    buf = torch.empty(2 * step + d, dtype=F16, device="cuda")
    x, y = buf.as_strided((3, d), (step, 1)), rand((3, d), F16, 95)
    x.copy_(rand((3, d), F16, 94))
    want = residual_norm(x.contiguous(), y)
    out = torch.empty_like(buf).as_strided((3, d), (step, 1))
    got = residual_norm(x, y, x_out=x, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

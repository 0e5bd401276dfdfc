"""Calls of a decoder layer's parts: positions of any integer type, with and without
rotation, and the FFN alone. Tolerances: norms and angles in fp32, each output
rounded to fp16 once, so two forms of one value are a step of fp16 apart at most:
2^-10 of it (2^-24 near zero). A rotated element is a sum of two products: a step of
each and of the sum, and angles of up to 300 in fp32, off by 2^-16."""
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import decoder

D, DFF, RANK, HEADS, KV = 512, 640, 32, 8, 2


def make(n_seqs):
    return decoder.random_layer(5, 0, D, DFF, RANK, DFF, DFF, 0, DFF, n_seqs, HEADS, KV, 512, max_batch=8)


def rows(n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((n, D), generator=g, device="cuda")


def test_plain_forms_of_any_width():
    """On the CPU, rows of 6 elements: pairs turn by pos 10000^(-i / 3)."""
    x = torch.arange(24, dtype=torch.float64).view(2, 2, 6)
    got = decoder.rotate(x.float(), torch.tensor([0, 3]))
    a = 3.0 * 10000.0 ** (-torch.arange(3, dtype=torch.float64) / 3)
    lo, hi = x[1, :, :3], x[1, :, 3:]
    want = torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)
    assert torch.equal(got[0], x[0].float()) and float((got[1] - want).abs().max()) <= 2.0 ** -17  # 24 elements of 2^-22
    z = torch.tensor([[3.0, 4.0], [0.0, 0.0]])
    want = torch.tensor([[3.0, 4.0], [0.0, 0.0]], dtype=torch.float64) / (12.5 + 1e-5) ** 0.5
    assert decoder.norm(z).dtype == torch.float16 and float((decoder.norm(z) - want).abs().max()) <= 2.0 ** -10


@pytest.mark.gpu
def test_projected_rows():
    say("decoder project")
    layer, x = make(1), rows(37, 2)
    q, k, v = layer.project(x)
    for dtype in (torch.int32, torch.int64):
        pos = torch.arange(40, 77, dtype=dtype, device="cuda") * 4
        for got, plain in zip(layer.project(x, pos), (decoder.rotate(q, pos), decoder.rotate(k, pos), v)):
            size = torch.maximum(*(t.float().abs() for t in (plain, plain.roll(32, -1))))
            off = (got.float() - plain.float()).abs()
            assert bool((off <= 2.0 ** -9 * size + 2.0 ** -14 * plain.float().abs().amax() + 2.0 ** -24).all())


@pytest.mark.gpu
def test_feed_forward_alone():
    """Beside a block's output of zeros: the same rows, bit by bit but for the order of the FFN's sums."""
    say("decoder feed forward")
    layer, x = make(1), rows(19, 3)
    a, b = x.clone(), x.clone()
    layer.feed_forward(a)
    layer.feed_forward(b, torch.zeros((19, HEADS, D // HEADS), dtype=torch.float16, device="cuda"))
    assert not torch.equal(a, x) and float((a - b).abs().max()) <= 2.0 ** -14 * float(a.abs().max())


@pytest.mark.gpu
def test_positions_of_64_bits():
    say("decoder int64 positions")
    out = []
    for dtype in (torch.int32, torch.int64):
        layer, x = make(2), rows(2, 4)
        for step in range(3):
            layer.decode(x, torch.tensor([step, step], dtype=dtype, device="cuda"), step + 1)
        out.append(layer.cache.tail_k[:, :, :3].clone())
    # the same rows go in first; later ones follow the FFN, whose sums have no fixed order
    assert torch.equal(out[0][:, :, 0], out[1][:, :, 0])
    assert float((out[0].float() - out[1].float()).abs().max()) <= 2.0 ** -8 * float(out[0].float().abs().max())

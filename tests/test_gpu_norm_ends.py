"""Norms of rows at both ends of the types' ranges, with the bounds of test_gpu_norms.py."""
import pytest
import torch

from helpers import say
from paper_2410_14740_amd.norms import residual_norm
from test_gpu_norms import BF16, F16, F32, check, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [72, 128, 301, 3000, 9000, 20000, 40000])
def test_subnormal_rows(kind, d):
    """Without eps: rows whose factor 1 / sqrt is no fp32 number."""
    say(f"norm subnormal rows {kind} {d}")
    for size in (1e-39, 3e-42, 2e-44):
        x = rand((3, d), F32, 1) * size
        _, out = residual_norm(x, kind=kind, eps=0.0, out_dtype=F32)
        check(x, None, None, out, kind=kind, eps=0.0, what=f"{size}")
        y = (rand((3, d), F32, 2) * max(size, 1e-39)).to(BF16)
        zero = torch.zeros_like(x)
        r, out = residual_norm(zero, y, post=True, kind=kind, eps=0.0)
        check(zero, y, r, out, post=True, kind=kind, eps=0.0, what=f"post {size}")


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [128, 301, 3000, 9000, 20000, 40000])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_the_largest_rows(kind, d, dt):
    """Numbers whose difference from the mean leaves fp32."""
    say(f"norm largest rows {kind} {d} {dt}")
    sign = torch.where(torch.arange(d, device="cuda") % 4 == 0, 1.0, -1.0)
    x = torch.stack([3e38 * sign, 3.3e38 * sign.roll(1), 1e38 * rand((d,), F32, 3).clamp(-3, 3)]).to(dt)
    _, out = residual_norm(x, kind=kind, out_dtype=F32)
    check(x, None, None, out, kind=kind)
    r, out = residual_norm(torch.ones_like(x), x, kind=kind, post=True, out_dtype=dt)
    check(torch.ones_like(x), x, r, out, kind=kind, post=True)


def test_rows_of_zeros_between():
    """Zero rows, which are summed in 64 bits too, beside ordinary ones."""
    say("norm zero rows")
    x = rand((64, 1000), F32, 1)
    x[::3] = 0
    for kind in ("rms", "layer"):
        _, out = residual_norm(x, kind=kind, out_dtype=F16)
        check(x, None, None, out, kind=kind)
        assert not out[::3].any()

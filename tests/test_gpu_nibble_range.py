"""4-bit weights at both ends of fp32's range, by the header's rule: a scale is the group's
largest size over 7, or its span over 15, in bfloat16; codes are rounded to nearest."""
import pytest
import torch

from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


@pytest.mark.parametrize("inner_rows", [False, True])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tiny_weights(dtype, zeros, inner_rows):
    """Whole multiples of a power of two whose quotient is that power: kept exactly, down to
    scales that fp32 has no inverse of, zeros among them."""
    hd = hd_gpu()
    announce(f"quantize tiny {dtype} zeros {zeros} rows {inner_rows}")
    powers = (-20, -125, -126, -127, -128, -129, -130, -131, -132, -133)
    g = torch.Generator().manual_seed(3)
    for group in (32, 64, 128):
        inner = 3 * group - 5
        k = torch.randint(-5, 11, (len(powers), inner), generator=g) if zeros else \
            torch.randint(-7, 8, (len(powers), inner), generator=g)
        for g0 in range(0, inner, group):
            k[:, g0], k[:, g0 + 1], k[:, g0 + 2] = (-5, 10, 0) if zeros else (-7, 7, 0)
        W = (k.double() * torch.tensor([2.0 ** p for p in powers])[:, None].double()).to(dtype)
        assert torch.equal(W.double() * torch.tensor([2.0 ** -p for p in powers],
                                                     dtype=torch.float64)[:, None], k.double())
        w = hd.nibble_quantize((W.t().contiguous() if inner_rows else W).cuda(), group=group,
                               inner_rows=inner_rows, zeros=zeros)
        assert torch.equal(hd.nibble_unpack(w).cpu(), W.float())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_too_small_for_any_scale(dtype):
    """A quotient below half of bfloat16's least value rounds to 0: the group stands for 0."""
    hd = hd_gpu()
    W = torch.zeros(4, 64)
    W[1] = 2.0 ** -133
    W[2, 3], W[3, 40] = 1e-45, -2.0 ** -133
    for zeros in (False, True):
        got = hd.nibble_unpack(hd.nibble_quantize(W.to(dtype).cuda(), group=32, zeros=zeros))
        assert bool((got == 0).all())


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_widest_weights(dtype, zeros):
    """Finite groups stay finite, whatever they span: within half a step (with zero points
    a rounded one more), the scale rounded by 2^-8 under up to 15 steps."""
    hd = hd_gpu()
    big = float(torch.finfo(dtype).max)
    W = torch.linspace(-1, 1, 64)[None].repeat(3, 1) * big
    W[1, 32:] = 0
    W[2, :32] = 3e38
    W[2, 32:] = -3e38
    W = W.to(dtype)
    got = hd.nibble_unpack(hd.nibble_quantize(W.cuda(), group=64, zeros=zeros)).cpu().double()
    x = W.double()
    lo, hi = x.amin(1).clamp(max=0), x.amax(1).clamp(min=0)
    s = (hi - lo) / 15 if zeros else torch.maximum(hi, -lo) / 7
    allowed = s * (1 + 2.0 ** -8) * ((0.5 + (0.5 if zeros else 0) + 15 * 2.0 ** -8) + 1e-5)
    # (a weight at the range's end may stand for one past it)
    past = (got.abs() == float("inf")) & (x.abs() + allowed[:, None] > 3.4e38)
    assert not bool(torch.isnan(got).any())
    assert bool((((got - x).abs() <= allowed[:, None]) | past).all())

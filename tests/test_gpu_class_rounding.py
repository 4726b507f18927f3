"""bf16 gradients of the cross entropy where what dS is rounded to does not average out: class vectors
that are equal (as before the first refining step) give every row the same dS, and the gradients
cancel whatever the encodings, or the class vectors, have in common. The scores' gradient may be
off by 2^-16 of itself, two roundings to bf16, and the result is rounded once."""
import math

import pytest
import torch

import learn_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# N, K, D: narrow tiles on either side, 128 and 256 wide ones, classes in pieces, of 256 at last
SIZES = [(300, 3, 64), (31, 700, 130), (520, 26, 200), (1000, 100, 136), (129, 129, 129),
         (3601, 3600, 72), (3601, 3600, 3599), (8200, 4900, 24), (140000, 600, 16)]


def make(N, K, D, kind, seed):
    g = torch.Generator().manual_seed(seed)
    H = (torch.randn(N, D, generator=g) + 3.0 * torch.randn(D, generator=g)).to(BF16)
    if kind == "zero":
        C = torch.zeros(K, D, dtype=BF16)
    else:
        C = torch.randn(D, generator=g).to(BF16).repeat(K, 1)
    y = torch.arange(N, dtype=torch.int32) % K
    return H, C, y, torch.full((N,), 1.0 / N), 0.7 / math.sqrt(D)


def bounds(dS, t, d, up, scale, H, C):
    """Of the errors of dH and dC before their own rounding: fp32's, and dS's two roundings."""
    eH, eC = P.grad_bounds(dS, t, d, up, scale, H, C, F32)
    return eH + 2.0 ** -16 * (dS.abs() @ C.abs()), eC + 2.0 ** -16 * (dS.abs().t() @ H.abs())


@pytest.mark.parametrize("kind", ["zero", "equal"])
@pytest.mark.parametrize("N,K,D", SIZES)
def test_equal_classes(N, K, D, kind):
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class gradient of {kind} classes, {N} rows, {K} classes, D {D}")
    H, C, y, up, scale = make(N, K, D, kind, seed=N + K + D)
    H, C, y, up = H.cuda(), C.cuda(), y.cuda(), up.cuda()
    cl = hd.class_loss(H, C, y, scale=scale)
    dH, dC = hd.class_loss_grad(H, C, y, cl, up, scale=scale)
    _, _, t, d, _ = P.class_loss(H, C, y, scale, None)
    dS, rH, rC, H0, C0 = P.class_grad(H, C, y, t, up, scale, None)
    eH, eC = bounds(dS, t, d, up, scale, H0, C0)
    for got, ref, e in ((dH, rH, eH), (dC, rC, eC)):
        off = (got.double() - ref).abs() - (e + 2.0 ** -8 * (ref.abs() + e))
        assert float(off.max()) <= 0, (float((got.double() - ref).norm() / ref.norm()),
                                       float(off.max()))


@pytest.mark.parametrize("N,K,D", [(20, 30, 64), (200, 150, 100), (3601, 3600, 72)])
def test_an_infinite_upstream_gradient(N, K, D):
    """A row whose upstream gradient overflowed: infinities of the formula's signs in dC, and NaN only
    where the formula has it (the row's own dH, a sum of both signs)."""
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class gradient, infinite upstream, {N} rows, {K} classes, D {D}")
    g = torch.Generator().manual_seed(N)
    H, C = (torch.randn(n, D, generator=g).to(BF16) for n in (N, K))
    H[H == 0] = 1.0
    y = torch.arange(N, dtype=torch.int32) % K
    up = torch.rand(N, generator=g)
    up[5] = math.inf
    scale = 0.3 / math.sqrt(D)
    cl = hd.class_loss(H.cuda(), C.cuda(), y.cuda(), scale=scale)
    dH, dC = hd.class_loss_grad(H.cuda(), C.cuda(), y.cuda(), cl, up.cuda(), scale=scale)
    sign = -torch.sign(H[5].double()).repeat(K, 1)
    sign[torch.arange(K) != y[5]] *= -1
    assert torch.equal(dC.cpu().double(), sign * math.inf)
    rest = torch.arange(N) != 5
    assert bool(torch.isnan(dH.cpu()[5]).all()) and bool(torch.isfinite(dH.cpu()[rest]).all())

"""Products with 4-bit weights where the codes' offset could weigh more than the weights: an X
of one sign (pixels, spectra, counts), most codes at their zero point. What a code at its zero
point meets adds exactly 0, so results follow from the few others, in fp32's every bit."""
import pytest
import torch

import ops_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def packed(q):
    """[outer, ceil(inner/2)] bytes from codes [outer, inner]."""
    if q.shape[1] % 2:
        q = torch.nn.functional.pad(q, (0, 1))
    return (q[:, ::2] | q[:, 1::2] << 4).to(torch.uint8)


# X in LDS: one row, a few, in more of the LDS, of more rows than a tile; X laid out in memory:
# a tile of rows past the LDS, more rows, many outputs, four output tiles
FORMS = [(1, 40, 561, F32), (9, 333, 784, F32), (1, 150, 16384, F32), (3, 4010, 4000, F32),
         (20, 64, 617, F32), (16, 50, 16384, F32), (40, 4130, 1300, F32), (64, 8210, 1200, F32),
         (16, 8300, 1100, F32), (1, 40, 561, BF16), (5, 333, 784, BF16), (40, 200, 617, BF16),
         (16, 50, 16384, BF16), (40, 4130, 1300, BF16), (130, 5770, 1100, BF16)]


def inputs(N, outer, inner, group, zeros, dtype):
    g = torch.Generator(device="cuda").manual_seed(N + outer + inner + group)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    groups = -(-inner // group)
    z = (torch.randint(1, 15, (outer, groups), generator=g, device="cuda") if zeros
         else torch.full((outer, groups), 8, device="cuda"))
    q = z.repeat_interleave(group, 1)[:, :inner].clone()
    X = (255 * rand(N, inner)).to(dtype)      # pixels, in all bits of the type
    scales = torch.tensor([0.5, 1.0, 2.0], device="cuda")[
        torch.randint(0, 3, (outer, groups), generator=g, device="cuda")]
    return q, z, X, scales, torch.arange(outer, device="cuda")


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,outer,inner,dtype", FORMS)
def test_one_code_off_its_zero_point(N, outer, inner, group, zeros, dtype):
    """The result is X's value at that code, times a power of two: all its bits."""
    hd = hd_gpu()
    announce(f"nibble one code {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
    q, z, X, scales, o = inputs(N, outer, inner, group, zeros, dtype)
    at = (o * 37 + 11) % inner
    step = torch.where(o % 2 == 0, 1, -1)
    q[o, at] += step
    w = hd.nibble_pack(packed(q), scales.to(BF16), z.to(torch.uint8) if zeros else None,
                       inner=inner, group=group)
    want = X.float()[:, at] * (scales[o, at // group] * step)
    assert torch.equal(hd.nibble_product(X, w, dtype=F32), want)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,outer,inner,dtype", FORMS)
def test_sums_that_cancel(N, outer, inner, group, zeros, dtype):
    """Two codes of one group, off to either side, over equal values of X: 0, and HardSign's 1."""
    hd = hd_gpu()
    announce(f"nibble cancel {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
    q, z, X, scales, o = inputs(N, outer, inner, group, zeros, dtype)
    X[:, 1::2] = X[:, :inner // 2 * 2:2]      # neighbours are equal
    at = (o * 19 + 5) % (inner // 2) * 2      # (groups begin at even inputs)
    q[o, at] += 1
    q[o, at + 1] -= 1
    w = hd.nibble_pack(packed(q), scales.to(BF16), z.to(torch.uint8) if zeros else None,
                       inner=inner, group=group)
    assert bool((hd.nibble_product(X, w, dtype=F32) == 0).all())
    for y_dt in (F32, BF16):
        assert bool((hd.nibble_product(X, w, act="hardsign", dtype=y_dt) == 1).all())


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,outer,inner,dtype", [
    (1, 40, 561, F32), (5, 333, 784, F32), (16, 50, 3000, F32), (40, 200, 617, F32),
    (5, 333, 784, BF16), (40, 200, 617, BF16)])
def test_readings_of_one_sign(N, outer, inner, group, zeros, dtype):
    """Any codes: every sum of the products themselves, (q - z) s x, in any order, is within I + 8
    roundings of their sizes."""
    hd = hd_gpu()
    codes, scales, z = P.random_nibble(outer, inner, group, zeros, seed=inner)
    X = torch.rand(N, inner, generator=torch.Generator().manual_seed(N)).to(dtype)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), z.cuda() if zeros else None, inner=inner,
                       group=group)
    W, _ = P.nibble_weights(codes, scales, z, inner, group)
    ref = X.double() @ W.t()
    for y_dt in (F32, BF16):
        Y = hd.nibble_product(X.cuda(), w, dtype=y_dt).cpu().double()
        if y_dt == F32 or dtype == F32:
            bound = P.nibble_bound(X, W.abs(), ref, y_dt)
        else:                                 # (bf16 of bf16: the zero point leaves the sums)
            bound = P.nibble_bound(X, P.nibble_weights(codes, scales, z, inner, group)[1], ref,
                                   y_dt)
        assert bool(((Y - ref).abs() <= bound).all())


# the kernels whose results are rounded to bf16 from bf16 X: rows, sizes, groups, zero points
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,outer,inner", [
    (1, 50, 4500), (20, 35, 2560), (40, 20, 1100), (16, 50, 16384), (40, 4130, 1300),
    (16, 28690, 2600), (130, 5770, 1100), (20, 28700, 1030), (3, 28690, 16384), (2, 30011, 16384),
    (16, 30011, 16384)])
def test_bf16_results(N, outer, inner, group, zeros):
    """Whole numbers: every order of the sums is exact, one rounding is left."""
    hd = hd_gpu()
    announce(f"nibble bf16 {N}x{outer}x{inner} group {group} zeros {zeros}")
    g = torch.Generator(device="cuda").manual_seed(N + inner)
    codes = torch.randint(0, 256, (outer, inner // 2), dtype=torch.uint8, generator=g,
                          device="cuda")
    ngroups = -(-inner // group)
    scales = torch.ones(outer, ngroups, dtype=BF16, device="cuda")
    z = torch.randint(0, 16, (outer, ngroups), dtype=torch.uint8, generator=g,
                      device="cuda") if zeros else None
    X = torch.randint(-8, 9, (N, inner), generator=g, device="cuda").to(BF16)
    Y = hd.nibble_product(X, hd.nibble_pack(codes, scales, z, inner=inner, group=group))
    H = hd.nibble_product(X, hd.nibble_pack(codes, scales, z, inner=inner, group=group),
                          act="hardsign")
    assert Y.dtype == BF16
    for o in range(0, outer, 4096):
        part = hd.nibble_pack(codes[o:o + 4096].contiguous(), scales[o:o + 4096].contiguous(),
                              None if z is None else z[o:o + 4096].contiguous(), inner=inner,
                              group=group)
        ref = X.float() @ hd.nibble_unpack(part).t()
        assert torch.equal(Y[:, o:o + 4096], ref.to(BF16))
        assert torch.equal(H[:, o:o + 4096], torch.where(ref >= 0, 1.0, -1.0).to(BF16))

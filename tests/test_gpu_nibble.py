"""Products with 4-bit weights and group scales against the formula in 64 bits."""
import math

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


def cuda(t):
    return None if t is None else t.cuda()


# N, outer, inner, group, zeros, dtype
SHAPES = [
    (1, 1, 1, 32, False, F32),
    (1, 16, 128, 128, False, BF16),
    (1, 17, 129, 64, True, F32),
    (2, 15, 127, 32, True, BF16),
    (1, 100, 10240, 128, False, F32),
    (3, 640, 561, 32, False, F32),
    (5, 333, 561, 64, True, BF16),
    (16, 31, 1000, 32, True, F32),
    (17, 64, 257, 64, False, BF16),
    (32, 130, 617, 128, True, F32),
    (33, 48, 300, 32, False, BF16),
    (33, 48, 300, 32, False, F32),
    (64, 200, 784, 64, True, BF16),
    (65, 77, 130, 128, True, F32),
    (131, 40, 96, 32, True, BF16),
    (4, 7, 16384, 64, False, BF16),
    (8, 4099, 256, 128, False, BF16),
    (64, 50, 2000, 32, True, F32),
]


@pytest.mark.parametrize("N,outer,inner,group,zeros,dtype", SHAPES)
def test_product(N, outer, inner, group, zeros, dtype):
    hd = hd_gpu()
    announce(f"nibble {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
    codes, scales, z = P.random_nibble(outer, inner, group, zeros, seed=N + outer + inner)
    X = torch.randn(N, inner, generator=torch.Generator().manual_seed(7)).to(dtype)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), cuda(z), inner=inner, group=group)
    W, size = P.nibble_weights(codes, scales, z, inner, group)
    assert torch.equal(hd.nibble_unpack(w).cpu().double(), W)  # 4 and 8 bits: exact in fp32
    ref = X.double() @ W.t()
    for y_dt in (F32, BF16):
        Y = hd.nibble_product(X.cuda(), w, dtype=y_dt)
        assert Y.dtype == y_dt and Y.shape == (N, outer)
        assert bool(((Y.cpu().double() - ref).abs() <= P.nibble_bound(X, size, ref, y_dt)).all())
    again = hd.nibble_product(X.cuda(), w, dtype=BF16)
    assert torch.equal(again, Y)


@pytest.mark.parametrize("N,outer,inner,group,zeros,dtype", SHAPES)
def test_product_exact_on_integers(N, outer, inner, group, zeros, dtype):
    """X of small integers and scales of powers of two: every order of the sums is exact."""
    hd = hd_gpu()
    announce(f"nibble integers {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
    codes, _, z = P.random_nibble(outer, inner, group, zeros, seed=3)
    g = torch.Generator().manual_seed(5)
    scales = torch.tensor([0.5, 1.0, 2.0])[
        torch.randint(0, 3, (outer, -(-inner // group)), generator=g)].to(BF16)
    X = torch.randint(-8, 9, (N, inner), generator=g).to(dtype)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), cuda(z), inner=inner, group=group)
    W, _ = P.nibble_weights(codes, scales, z, inner, group)
    Y = hd.nibble_product(X.cuda(), w, dtype=F32).cpu().double()
    ref = X.double() @ W.t()
    assert torch.equal(Y, ref)
    H = hd.nibble_product(X.cuda(), w, act="hardsign", dtype=F32).cpu().double()
    assert torch.equal(H, torch.where(ref >= 0, 1.0, -1.0).double())


# every kernel there is: rows, type, group, zero points; several tiles to a wave and one
# that ends inside
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [1, 20, 40])
def test_every_kernel(N, dtype, group, zeros):
    hd = hd_gpu()
    for outer, inner in ((50, 4500), (35, 2560), (20, 1100)):
        announce(f"nibble every {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
        codes, scales, z = P.random_nibble(outer, inner, group, zeros, seed=inner)
        X = torch.randn(N, inner, generator=torch.Generator().manual_seed(N)).to(dtype)
        w = hd.nibble_pack(codes.cuda(), scales.cuda(), cuda(z), inner=inner, group=group)
        W, size = P.nibble_weights(codes, scales, z, inner, group)
        ref = X.double() @ W.t()
        Y = hd.nibble_product(X.cuda(), w, dtype=F32).cpu().double()
        assert bool(((Y - ref).abs() <= P.nibble_bound(X, size, ref, F32)).all())


# 4-bit weights past the caches take loads of their own
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_weights(dtype, group, zeros):
    hd = hd_gpu()
    outer, inner, rows = 30011, 16384, 64
    announce(f"nibble large group {group} zeros {zeros} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (outer, inner // 2), dtype=torch.uint8, generator=g,
                          device="cuda")
    scales = (torch.rand(outer, inner // group, generator=g, device="cuda") + 0.25).to(BF16)
    z = torch.randint(0, 16, (outer, inner // group), dtype=torch.uint8, generator=g,
                      device="cuda") if zeros else None
    X = torch.randn(2, inner, generator=torch.Generator().manual_seed(2)).to(dtype)
    Y = hd.nibble_product(X.cuda(), hd.nibble_pack(codes, scales, z, group=group),
                          dtype=F32).cpu().double()
    pick = torch.linspace(0, outer - 1, rows).long()
    W, size = P.nibble_weights(codes[pick.cuda()].cpu(), scales[pick.cuda()].cpu(),
                               None if z is None else z[pick.cuda()].cpu(), inner, group)
    ref = X.double() @ W.t()
    assert bool(((Y[:, pick] - ref).abs() <= P.nibble_bound(X, size, ref, F32)).all())


# many outputs: workgroups of more output tiles, the last ones past the end
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,outer,inner,dtype", [
    (16, 8300, 1100, F32), (40, 4130, 1300, F32), (16, 28690, 2600, BF16),
    (130, 5770, 1100, BF16), (20, 28700, 1030, BF16), (3, 28690, 16384, BF16),
    # X of fp32 in more of the LDS: two, three, four output tiles
    (1, 150, 16384, F32), (4, 10230, 4096, F32), (3, 16010, 4000, F32), (1, 20010, 16384, F32),
    (1, 28690, 16384, F32)])
def test_many_outputs(N, outer, inner, dtype, group, zeros):
    hd = hd_gpu()
    announce(f"nibble many outputs {N}x{outer}x{inner} group {group} zeros {zeros} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(N + inner)
    codes = torch.randint(0, 256, (outer, inner // 2), dtype=torch.uint8, generator=g,
                          device="cuda")
    ngroups = -(-inner // group)
    scales = (torch.rand(outer, ngroups, generator=g, device="cuda") + 0.25).to(BF16)
    z = torch.randint(0, 16, (outer, ngroups), dtype=torch.uint8, generator=g,
                      device="cuda") if zeros else None
    X = torch.randn(N, inner, generator=torch.Generator().manual_seed(2)).to(dtype)
    w = hd.nibble_pack(codes, scales, z, inner=inner, group=group)
    Y = hd.nibble_product(X.cuda(), w, dtype=F32)
    pick = torch.cat([torch.arange(70), torch.arange(outer - 70, outer)])
    W, size = P.nibble_weights(codes[pick.cuda()].cpu(), scales[pick.cuda()].cpu(),
                               None if z is None else z[pick.cuda()].cpu(), inner, group)
    ref = X.double() @ W.t()
    bound = P.nibble_bound(X, size, ref, F32)
    assert bool(((Y[:, pick.cuda()].cpu().double() - ref).abs() <= bound).all())
    # the outputs between: whole numbers, exact in every order of the sums
    ones = torch.ones_like(scales)
    w = hd.nibble_pack(codes, ones, z, inner=inner, group=group)
    X = torch.randint(-8, 9, (N, inner), generator=torch.Generator().manual_seed(3)).to(dtype)
    Y = hd.nibble_product(X.cuda(), w, dtype=F32)
    for o in range(0, outer, 4096):
        part = hd.nibble_pack(codes[o:o + 4096].contiguous(), ones[o:o + 4096].contiguous(),
                              None if z is None else z[o:o + 4096].contiguous(), inner=inner,
                              group=group)
        assert torch.equal(Y[:, o:o + 4096], X.cuda().float() @ hd.nibble_unpack(part).t())


@pytest.mark.parametrize("inner", [64, 70, 200])
def test_codes_at_any_address(inner):
    hd = hd_gpu()
    codes, scales, z = P.random_nibble(37, inner, 32, True, seed=inner)
    want = hd.nibble_pack(codes.cuda(), scales.cuda(), z.cuda(), inner=inner, group=32)
    room = torch.empty(codes.numel() + 8, dtype=torch.uint8, device="cuda")
    for off in (1, 2, 4):
        there = room[off:off + codes.numel()].view(codes.shape)
        there.copy_(codes)
        got = hd.nibble_pack(there, scales.cuda(), z.cuda(), inner=inner, group=32)
        assert torch.equal(hd.nibble_unpack(got), hd.nibble_unpack(want))
    W, _ = P.nibble_weights(codes, scales, z, inner, 32)
    assert torch.equal(hd.nibble_unpack(want).cpu().double(), W)


def test_fp32_x_in_full():
    """Weight 1 (code 1, zero point 0) on one input: the three parts of an fp32 X add
    up to every bit of it."""
    hd = hd_gpu()
    inner = 192
    codes = torch.zeros((inner, -(-inner // 2)), dtype=torch.uint8)
    for o in range(inner):
        codes[o, o // 2] = 16 if o % 2 else 1
    ones = torch.ones(inner, inner // 64, dtype=BF16)
    w = hd.nibble_pack(codes.cuda(), ones.cuda(), torch.zeros_like(ones).to(torch.uint8).cuda(),
                       group=64)
    X = torch.randn(9, inner, generator=torch.Generator().manual_seed(6))
    X[0], X[1], X[2] = 1.0 + 2.0 ** -23, 16777215.0, -2.0 ** -100 * (2 - 2.0 ** -23)
    X[3] *= 1e30
    assert torch.equal(hd.nibble_product(X.cuda(), w).cpu(), X)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("zeros", [False, True])
def test_infinities_and_nan_in_x(dtype, zeros):
    hd = hd_gpu()
    N, outer, inner, group = 6, 40, 200, 32
    codes, scales, z = P.random_nibble(outer, inner, group, zeros, seed=11)
    X = torch.randn(N, inner, generator=torch.Generator().manual_seed(1))
    X[1, 17], X[2, 3], X[2, 190], X[3, 5] = math.inf, -math.inf, 2.0, math.nan
    X[4, 0], X[4, 1] = 3e38, -3e38
    X = X.to(dtype)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), cuda(z), inner=inner, group=group)
    W, _ = P.nibble_weights(codes, scales, z, inner, group)
    Y = hd.nibble_product(X.cuda(), w, dtype=F32).cpu().double()
    ref = torch.stack([(X[n].double()[None, :] * W).sum(1) for n in range(N)])
    for n in (0, 5):  # untouched by their neighbours
        alone = hd.nibble_product(X[n:n + 1].cuda(), w, dtype=F32).cpu().double()
        assert torch.equal(Y[n], alone[0]) and bool(torch.isfinite(Y[n]).all())
    for n in (1, 2, 3):
        assert torch.equal(torch.isnan(Y[n]), torch.isnan(ref[n]))
        ok = ~torch.isnan(ref[n])
        assert torch.equal(Y[n][ok], ref[n][ok])
    small = ref[4].abs() < 1e38  # where no partial sum of one order leaves fp32's range
    big = ref[4].abs() > 3.4e38 * 2
    assert bool((Y[4][big].abs() == math.inf).all())
    assert not bool(torch.isnan(Y[4][small]).any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_offsets(dtype):
    """Rows inside wider matrices, from any element on; nothing outside is written."""
    hd = hd_gpu()
    N, outer, inner, group = 19, 70, 203, 64
    codes, scales, _ = P.random_nibble(outer, inner, group, False, seed=2)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), inner=inner, group=group)
    wide = torch.randn(N, inner + 6, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    for off in (0, 1, 3, 5):
        X = wide[:, off:off + inner]
        ref = hd.nibble_product(X.contiguous(), w)
        out = torch.full((N, outer + 9), 7.0, dtype=dtype, device="cuda")
        hd.nibble_product(X, w, out=out[:, 4:4 + outer])
        assert torch.equal(out[:, 4:4 + outer], ref)
        assert bool((out[:, :4] == 7).all()) and bool((out[:, 4 + outer:] == 7).all())


def test_rows_do_not_depend_on_the_batch():
    hd = hd_gpu()
    codes, scales, z = P.random_nibble(90, 700, 64, True, seed=4)
    w = hd.nibble_pack(codes.cuda(), scales.cuda(), z.cuda(), inner=700, group=64)
    X = torch.randn(70, 700, generator=torch.Generator().manual_seed(8)).cuda()
    Y = hd.nibble_product(X, w)
    bound = P.nibble_bound(X.cpu(), P.nibble_weights(codes, scales, z, 700, 64)[1],
                           Y.cpu().double(), F32)
    for n in (0, 15, 16, 63, 69):
        one = hd.nibble_product(X[n:n + 1], w)
        assert bool(((one[0] - Y[n]).abs().cpu() <= 2 * bound[n]).all())


@pytest.mark.parametrize("outer,inner,group,inner_rows,zeros,dtype", [
    (40, 561, 32, False, False, F32), (40, 561, 64, True, True, F32),
    (33, 300, 128, False, True, BF16), (128, 617, 64, True, False, BF16),
    (1, 1, 32, True, True, F32),
])
def test_quantize(outer, inner, group, inner_rows, zeros, dtype):
    hd = hd_gpu()
    announce(f"quantize {outer}x{inner} group {group} {inner_rows} {zeros} {dtype}")
    g = torch.Generator().manual_seed(outer + inner)
    W = (torch.randn(outer, inner, generator=g) * 0.1 + 0.03).to(dtype)
    W[0, :] = 0  # groups of zeros
    V = W.t().contiguous() if inner_rows else W
    wide = torch.zeros(V.shape[0], V.shape[1] + 3, dtype=dtype)
    wide[:, 2:2 + V.shape[1]] = V
    w = hd.nibble_quantize(wide.cuda()[:, 2:2 + V.shape[1]], group=group, inner_rows=inner_rows,
                           zeros=zeros)
    got = hd.nibble_unpack(w).cpu().double()
    Wd = W.double()
    for g0 in range(0, inner, group):
        x = Wd[:, g0:g0 + group]
        lo, hi = x.amin(1).clamp(max=0), x.amax(1).clamp(min=0)
        s = (hi - lo) / 15 if zeros else torch.maximum(hi, -lo) / 7
        # half a step, a zero point rounded by up to half, the scale by 2^-8 of up to 15 steps
        step = s * (1 + 2.0 ** -8)
        allowed = step * ((0.5 + (0.5 if zeros else 0) + 15 * 2.0 ** -8) + 1e-5)
        assert bool(((got[:, g0:g0 + group] - x).abs() <= allowed[:, None]).all())
    X = torch.randn(2, inner, generator=g)
    Y = hd.nibble_product(X.cuda(), w).cpu().double()
    ref = X.double() @ got.t()
    # |code| + zero is at most 30 steps
    size = torch.zeros_like(got)
    for g0 in range(0, inner, group):
        x = Wd[:, g0:g0 + group]
        size[:, g0:g0 + group] = ((x.amax(1).clamp(min=0) - x.amin(1).clamp(max=0)) * 5)[:, None]
    assert bool(((Y - ref).abs() <= P.nibble_bound(X, size, ref, F32)).all())


def test_quantize_not_finite():
    hd = hd_gpu()
    W = torch.randn(20, 256, generator=torch.Generator().manual_seed(0))
    W[3, 70], W[5, 200] = math.inf, math.nan
    for zeros in (False, True):
        got = hd.nibble_unpack(hd.nibble_quantize(W.cuda(), group=64, zeros=zeros)).cpu()
        bad = torch.zeros(20, 256, dtype=torch.bool)
        bad[3, 64:128], bad[5, 192:] = True, True
        assert torch.equal(torch.isnan(got), bad)


def test_other_stream_and_empty():
    hd = hd_gpu()
    codes, scales, _ = P.random_nibble(30, 100, 32, False, seed=1)
    codes, scales = codes.cuda(), scales.cuda()
    X = torch.randn(3, 100).cuda()
    ref = hd.nibble_product(X, hd.nibble_pack(codes, scales, inner=100, group=32))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        w = hd.nibble_pack(codes, scales, inner=100, group=32)
        Y = hd.nibble_product(X, w)
    s.synchronize()
    assert torch.equal(Y, ref)
    assert hd.nibble_product(X[:0], w).shape == (0, 30)


def test_refusals():
    hd = hd_gpu()
    codes, scales, z = (t.cuda() for t in P.random_nibble(8, 64, 32, True, seed=0))
    w = hd.nibble_pack(codes, scales, z, inner=64, group=32)
    X = torch.zeros(2, 64, device="cuda")
    for bad in (lambda: hd.nibble_pack(codes, scales, inner=66, group=32),
                lambda: hd.nibble_pack(codes, scales, group=48),
                lambda: hd.nibble_pack(codes, scales, z[:, :1], inner=64, group=32),
                lambda: hd.nibble_product(X[:, :63], w),
                lambda: hd.nibble_product(X.cpu(), w),
                lambda: hd.nibble_product(X.t().contiguous().t(), w),
                lambda: hd.nibble_product(X, w, out=torch.zeros(2, 9, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: hd.nibble_pack(codes.float(), scales, inner=64, group=32),
                lambda: hd.nibble_pack(codes, scales.float(), inner=64, group=32),
                lambda: hd.nibble_product(X.half(), w),
                lambda: hd.nibble_product(X, w, dtype=torch.float16)):
        with pytest.raises(TypeError):
            bad()

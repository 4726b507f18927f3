"""Activations kept in 8 bits and the class vectors' gradient read from them."""
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


def activations(N, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    H = torch.randn(N, D, generator=g) * torch.exp(2 * torch.randn(D, generator=g))
    if D > 2:
        H[:, 1] = 0.0                              # a column of zeros
        H[:, 2] = torch.where(H[:, 2] > 0, 1.0, -1.0)  # an encoding
    return H.to(dtype)


SHAPES = [(1, 1), (1, 64), (63, 5), (64, 256), (65, 257), (130, 31), (200, 513), (7, 4097),
          (1000, 100)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D", SHAPES)
def test_store_and_load(N, D, dtype):
    hd = hd_gpu()
    announce(f"ckpt {N}x{D} {dtype}")
    H = activations(N, D, dtype, N + D)
    q, s = P.ckpt(H)
    kept = hd.ckpt_store(H.cuda())
    ref = P.ckpt_values(q, s)
    back = hd.ckpt_load(kept)
    assert back.dtype == F32
    assert torch.equal(back.cpu(), ref.float())   # the rule, step for step: one rounding of q s
    assert torch.equal(hd.ckpt_load(kept, dtype=BF16).cpu(), ref.float().to(BF16))
    # within half a step (a step is at most 1/127 of the group's largest)
    err = (back.cpu().double() - H.double()).abs()
    step = s.double().repeat_interleave(64, 0)[:N]
    assert bool((err <= step * (0.5 + 1e-4)).all())


def test_encodings_are_kept_exactly():
    hd = hd_gpu()
    H = torch.where(torch.randn(300, 700, generator=torch.Generator().manual_seed(1)) > 0, 1.0, -1.0)
    back = hd.ckpt_load(hd.ckpt_store(H.cuda())).cpu()
    one = torch.tensor(127.0) * (torch.tensor(1.0) / torch.tensor(127.0))
    assert torch.equal(back, H * one)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_not_finite_and_tiny(dtype):
    hd = hd_gpu()
    H = activations(200, 40, dtype, 3)
    H[70, 4], H[10, 5], H[199, 6] = math.nan, math.inf, -math.inf
    H[:, 7] = 1e-39
    H[:64, 8] = torch.finfo(dtype).max
    back = hd.ckpt_load(hd.ckpt_store(H.cuda())).cpu()
    bad = torch.zeros(200, 40, dtype=torch.bool)
    bad[64:128, 4], bad[:64, 5], bad[192:, 6] = True, True, True
    assert torch.equal(torch.isnan(back), bad)
    ok = ~bad
    ref = P.ckpt_values(*P.ckpt(H)).float()
    assert torch.equal(back[ok], ref[ok])
    assert bool((back[:, 7] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    hd = hd_gpu()
    N, D = 100, 301
    wide = activations(N, D + 5, dtype, 4).cuda()
    for off in (0, 1, 2, 5):
        H = wide[:, off:off + D]
        kept = hd.ckpt_store(H)
        ref = hd.ckpt_store(H.contiguous())
        assert torch.equal(hd.ckpt_load(kept), hd.ckpt_load(ref))
        out = torch.full((N, D + 3), 5.0, dtype=dtype, device="cuda")
        hd.ckpt_load(kept, out=out[:, 2:2 + D])
        assert torch.equal(out[:, 2:2 + D], hd.ckpt_load(kept, dtype=dtype))
        assert bool((out[:, :2] == 5).all()) and bool((out[:, 2 + D:] == 5).all())


GRADS = [(1, 1, 1), (1, 300, 26), (64, 32, 6), (65, 257, 33), (500, 100, 100), (1000, 513, 10),
         (3000, 1000, 26), (700, 129, 128), (129, 40, 200), (20000, 64, 2)]


def grad_bound(dS, ref_abs, N):
    """Products are exact. 64 terms of a group are added one after another by the matrix
    instruction's chain (three parts: 192), groups one after another, then slices."""
    return (192 + N / 64 + 64) * P.U32 * ref_abs


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D,K", GRADS)
def test_class_grad(N, D, K, dtype):
    hd = hd_gpu()
    announce(f"class grad {N}x{D}x{K} {dtype}")
    H = activations(N, D, F32, N + D + K)
    g = torch.Generator().manual_seed(K)
    dS = (torch.randn(N, K, generator=g) / N).to(dtype)
    v = P.ckpt_values(*P.ckpt(H))
    ref = dS.double().t() @ v
    bound = grad_bound(dS, dS.double().abs().t() @ v.abs(), N)
    kept = hd.ckpt_store(H.cuda())
    got = hd.ckpt_class_grad(dS.cuda(), kept)
    assert got.dtype == F32
    assert bool(((got.cpu().double() - ref).abs() <= bound).all())
    assert torch.equal(hd.ckpt_class_grad(dS.cuda(), kept), got)  # the same bits
    base = torch.randn(K, D, generator=g)
    acc = base.cuda()
    hd.ckpt_class_grad(dS.cuda(), kept, out=acc, accumulate=True)
    assert torch.equal(acc.cpu(), base + got.cpu())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D,K", GRADS)
def test_class_grad_exact_on_integers(N, D, K, dtype):
    """Encodings times a power of two, and small whole gradients: exact in any order."""
    hd = hd_gpu()
    g = torch.Generator().manual_seed(N + K)
    H = torch.where(torch.randn(N, D, generator=g) > 0, 127.0, -127.0)
    dS = torch.randint(-3, 4, (N, K), generator=g).to(dtype)
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H.cuda()))
    s = P.ckpt(H)[1][0, 0].double()  # one scale for all groups, about 1
    assert float(s) == 1.0
    assert torch.equal(got.cpu().double(), dS.double().t() @ H.double())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [1, 2, 6, 10, 11, 16, 21, 22, 31, 32, 33, 42, 43, 64, 65, 96, 97, 129])
def test_class_grad_every_count_of_classes(K, dtype):
    """Each layout of the classes in tiles, exact on integers."""
    hd = hd_gpu()
    N, D = 700, 300
    g = torch.Generator().manual_seed(K)
    H = torch.where(torch.randn(N, D, generator=g) > 0, 127.0, -127.0)
    dS = torch.randint(-3, 4, (N, K), generator=g).to(dtype)
    dS[5:9] *= 0.015625  # (and parts of dS beyond the first eight bits)
    dS[5:9] += 3.0
    ref = dS.double().t() @ H.double()
    kept = hd.ckpt_store(H.cuda())
    got = hd.ckpt_class_grad(dS.cuda(), kept)
    assert torch.equal(got.cpu().double(), ref)
    acc = torch.ones(K, D, device="cuda")
    hd.ckpt_class_grad(dS.cuda(), kept, out=acc, accumulate=True)
    assert torch.equal(acc.cpu().double(), ref + 1.0)


def test_fp32_gradients_in_full():
    """Every bit of an fp32 dS counts: one row, one group, q s = 1."""
    hd = hd_gpu()
    H = torch.full((1, 40), 127.0)
    dS = torch.randn(1, 64, generator=torch.Generator().manual_seed(2))
    dS[0, 0], dS[0, 1], dS[0, 2] = 1.0 + 2.0 ** -23, 16777215.0, -1e-30
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H.cuda())).cpu()
    # q = 127, so each part times 127 is exact and the sum of three parts is rounded twice
    ref = dS.double().t() * 127.0
    assert bool(((got.double() - ref).abs() <= 2 * P.U32 * ref.abs()).all())


@pytest.mark.parametrize("K", [3, 26])
def test_fp32_gradients_of_few_classes_in_full(K):
    """As above, where the workgroups cut dS by themselves."""
    hd = hd_gpu()
    H = torch.full((1, 40), 127.0)
    dS = torch.randn(1, K, generator=torch.Generator().manual_seed(2))
    dS[0, 0], dS[0, 1], dS[0, 2] = 1.0 + 2.0 ** -23, 16777215.0, -1e-30
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H.cuda())).cpu()
    ref = dS.double().t() * 127.0
    assert bool(((got.double() - ref).abs() <= 2 * P.U32 * ref.abs()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [6, 26])
def test_class_grad_short_and_long_calls_agree(K, dtype):
    """Few classes: a long call lays dS out first, a short one does not. Exact on integers."""
    hd = hd_gpu()
    N, D = 4300, 8200
    announce(f"class grad {N}x{D}x{K} {dtype}")
    g = torch.Generator().manual_seed(K)
    H = torch.where(torch.randn(N, D, generator=g) > 0, 127.0, -127.0).cuda()
    dS = torch.randint(-3, 4, (N, K), generator=g).to(dtype).cuda()
    whole = hd.ckpt_class_grad(dS, hd.ckpt_store(H))
    parts = torch.zeros(K, D, device="cuda")
    for n0 in range(0, N, 800):
        hd.ckpt_class_grad(dS[n0:n0 + 800], hd.ckpt_store(H[n0:n0 + 800]), out=parts,
                           accumulate=True)
    assert torch.equal(whole, parts)
    at = [0, 1, 63, 4095, D - 1]
    ref = dS.cpu().double().t() @ H[:, at].cpu().double()
    assert torch.equal(whole[:, at].cpu().double(), ref)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [5, 26])
def test_class_grad_of_few_classes_not_finite_and_strided(K, dtype):
    hd = hd_gpu()
    N, D = 150, 70
    kept = hd.ckpt_store(activations(N, D, F32, 1).cuda())
    wide = torch.randn(N, K + 3, generator=torch.Generator().manual_seed(3)).to(dtype)
    clean = hd.ckpt_class_grad(wide[:, 1:1 + K].contiguous().cuda(), kept).cpu()
    assert torch.equal(hd.ckpt_class_grad(wide.cuda()[:, 1:1 + K], kept).cpu(), clean)
    wide[5, 1 + 2], wide[140, 1 + 4] = math.nan, -math.inf
    wide[:, 0] = wide[:, 1 + K] = math.nan  # (not read)
    got = hd.ckpt_class_grad(wide.cuda()[:, 1:1 + K], kept).cpu()
    assert bool(torch.isnan(got[2]).all()) and not bool(torch.isfinite(got[4]).any())
    rest = [k for k in range(K) if k not in (2, 4)]
    assert torch.equal(got[rest], clean[rest])


def test_class_grad_not_finite():
    """NaN and infinities of dS stay in their class, those of H in their column."""
    hd = hd_gpu()
    N, D, K = 150, 70, 40
    H = activations(N, D, F32, 1)
    H[:, 1] = 1.0
    dS = torch.randn(N, K, generator=torch.Generator().manual_seed(3))
    clean = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H.cuda())).cpu()
    dS[5, 7], dS[140, 33] = math.nan, math.inf
    H[100, 9] = math.nan
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H.cuda())).cpu()
    assert bool(torch.isnan(got[7]).all()) and bool(torch.isnan(got[:, 9]).all())
    assert not bool(torch.isfinite(got[33]).any())
    keep_k = [k for k in range(K) if k not in (7, 33)]
    keep_d = [d for d in range(D) if d != 9]
    assert torch.equal(got[keep_k][:, keep_d], clean[keep_k][:, keep_d])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_class_grad_strided(dtype):
    hd = hd_gpu()
    N, D, K = 333, 90, 37
    kept = hd.ckpt_store(activations(N, D, F32, 8).cuda())
    wide = torch.randn(N, K + 3, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    for off in (0, 1, 3):
        dS = wide[:, off:off + K]
        assert torch.equal(hd.ckpt_class_grad(dS, kept),
                           hd.ckpt_class_grad(dS.contiguous(), kept))


def test_gradient_against_differences():
    """The scores are linear in C: for any change E of C, sum dS (Hq (C + E)^T - Hq C^T)
    = <dC, E>, with Hq what the checkpoint gives back."""
    hd = hd_gpu()
    N, D, K = 260, 150, 11
    H = activations(N, D, F32, 21).clamp(-50, 50)
    g = torch.Generator().manual_seed(4)
    dS, C, E = torch.randn(N, K, generator=g), torch.randn(K, D, generator=g), torch.randn(K, D, generator=g)
    kept = hd.ckpt_store(H.cuda())
    back = hd.ckpt_load(kept).cpu().double()
    dC = hd.ckpt_class_grad(dS.cuda(), kept).cpu().double()

    def value(c):
        return float((dS.double() * (back @ c.t())).sum())

    change = value(C.double() + E.double()) - value(C.double())
    bound = float((grad_bound(dS, dS.double().abs().t() @ back.abs(), N) * E.double().abs()).sum())
    # (q s was rounded once to fp32 on the way back)
    bound += float(P.U32 * ((dS.double().abs().t() @ back.abs()) * E.double().abs()).sum())
    assert abs(change - float((dC * E.double()).sum())) <= bound + 1e-9 * abs(change)


def test_other_stream_and_empty():
    hd = hd_gpu()
    H = activations(400, 300, BF16, 2).cuda()
    dS = torch.randn(400, 12, generator=torch.Generator().manual_seed(0)).cuda()
    ref = hd.ckpt_class_grad(dS, hd.ckpt_store(H))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = hd.ckpt_class_grad(dS, hd.ckpt_store(H))
    st.synchronize()
    assert torch.equal(got, ref)
    none = hd.ckpt_store(H[:0])
    assert hd.ckpt_load(none).shape == (0, 300)
    assert bool((hd.ckpt_class_grad(dS[:0], none) == 0).all())
    acc = ref.clone()
    hd.ckpt_class_grad(dS[:0], none, out=acc, accumulate=True)
    assert torch.equal(acc, ref)


def test_refusals():
    hd = hd_gpu()
    H = torch.zeros(10, 20, device="cuda")
    kept = hd.ckpt_store(H)
    dS = torch.zeros(10, 3, device="cuda")
    for bad in (lambda: hd.ckpt_store(H.t()), lambda: hd.ckpt_store(H.cpu()),
                lambda: hd.ckpt_store(H[:9], out=kept),
                lambda: hd.ckpt_load(kept, out=torch.zeros(10, 21, device="cuda")),
                lambda: hd.ckpt_class_grad(dS[:9], kept),
                lambda: hd.ckpt_class_grad(dS, kept, accumulate=True),
                lambda: hd.ckpt_class_grad(dS, kept, out=torch.zeros(3, 19, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: hd.ckpt_store(H.half()), lambda: hd.ckpt_load(kept, dtype=torch.float16),
                lambda: hd.ckpt_class_grad(dS.int(), kept)):
        with pytest.raises(TypeError):
            bad()


# the three parts of fp32 as rows of their own, laid out in memory: four row tiles, and few
# classes in a call that is too large for the workgroups to cut dS themselves
@pytest.mark.parametrize("D,K", [(40, 33), (40, 37), (40, 42), (300, 42), ((1 << 24) + 70, 3),
                                 ((1 << 24) + 70, 10), ((1 << 25) + 70, 26)])
def test_fp32_gradients_laid_out_in_full(D, K):
    """Every bit of an fp32 dS counts there too: one row, one group, q s = 127."""
    hd = hd_gpu()
    announce(f"class grad in full 1x{D}x{K}")
    dS = torch.randn(1, K, generator=torch.Generator().manual_seed(K))
    dS[0, 0], dS[0, 1], dS[0, 2] = 1.0 + 2.0 ** -23, 16777215.0, -1e-30
    H = torch.full((1, D), 127.0, device="cuda")
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(H))
    # as above: each part times 127 is exact and the sum of three parts is rounded twice
    ref = dS.double().t().cuda() * 127.0
    assert bool(((got.double() - ref).abs() <= 2 * P.U32 * ref.abs()).all())


@pytest.mark.parametrize("K", [3, 10, 26, 33, 42, 64])
def test_fp32_gradients_of_whole_groups_in_full(K):
    """One row of 64 holds something: the others add exact zeros, wherever it lies."""
    hd = hd_gpu()
    N, D = 200, 70
    dS = torch.zeros(N, K)
    at = (torch.arange(K) * 29 + 3) % N
    v = torch.randn(K, generator=torch.Generator().manual_seed(K))
    v[0], v[1], v[2] = 1.0 + 2.0 ** -23, 16777215.0, -1e-30
    dS[at, torch.arange(K)] = v
    got = hd.ckpt_class_grad(dS.cuda(), hd.ckpt_store(torch.full((N, D), 127.0).cuda())).cpu()
    ref = v.double()[:, None] * 127.0
    assert bool(((got.double() - ref).abs() <= 2 * P.U32 * ref.abs()).all())

"""The cross entropy of class scores that are never kept, and its gradient, against the formulas
in 64 bits. The bounds are those of tests/learn_plain.py."""
import math

import pytest
import torch

import learn_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def make(N, K, D, dtype, seed, mask=None, spread=3.0):
    """Encodings, class vectors, classes (some rows ask for none), mask, upstream gradient and
    scale. Closed classes and rows that ask for none hold infinities and NaN."""
    g = torch.Generator().manual_seed(seed)
    H = torch.randn(N, D, generator=g).to(dtype)
    C = torch.randn(K, D, generator=g).to(dtype)
    y = torch.randint(0, K, (N,), dtype=torch.int32, generator=g)
    drop = torch.rand(N, generator=g) < 0.15
    y[drop] = torch.tensor([-1, K, 2 ** 31 - 1], dtype=torch.int32)[
        torch.randint(0, 3, (int(drop.sum()),), generator=g)]
    m = None
    if mask is not None:
        m = torch.rand(K, generator=g) < mask
        bad = torch.tensor([math.nan, math.inf, -math.inf])
        C[~m, K % D] = bad[torch.randint(0, 3, (int((~m).sum()),), generator=g)].to(dtype)
        H[drop, 0] = math.nan
    up = torch.randn(N, generator=g)
    return H, C, y, m, up, spread / math.sqrt(D)


def same_kind(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.isinf(a), torch.isinf(b))
    assert torch.equal(a[torch.isinf(a)], b[torch.isinf(b)])


def within(a, b, tol):
    a = a.cpu().double()
    same_kind(a, b)
    ok = torch.isfinite(b)
    tol = tol.expand_as(b) if isinstance(tol, torch.Tensor) else torch.full_like(b, tol)
    over = ((a - b).abs() - tol)[ok]
    assert over.numel() == 0 or float(over.max()) <= 0, (float(over.max()),
                                                        float((a - b).abs()[ok].max()))


def check(hd, H, C, y, m, up, scale, wrt="both"):
    dtype = H.dtype
    Hc, Cc, yc, uc = H.cuda(), C.cuda(), y.cuda(), up.cuda()
    mc = None if m is None else m.cuda()
    return check_on(hd, (Hc, Cc, yc, mc, uc), (H, C, y, m, up), scale, wrt, dtype)


def check_on(hd, dev, host, scale, wrt, dtype):
    Hc, Cc, yc, mc, uc = dev
    H, C, y, m, up = host
    N, K = H.shape[0], C.shape[0]
    cl = hd.class_loss(Hc, Cc, yc, scale=scale, mask=mc)
    # (the reference on the GPU in 64 bits, for its speed)
    loss, stats, t, d, top = (v.cpu() for v in P.class_loss(H.cuda(), C.cuda(), y.cuda(), scale,
                                                            None if m is None else m.cuda()))
    within(cl.loss, loss, d[:, 0] + 2 * P.U32 * loss.abs())
    within(cl.stats[:, 0], stats[:, 0], top[:, 0] + 2 * P.U32 * stats[:, 0].abs())
    within(cl.stats[:, 1], stats[:, 1], d[:, 0])
    again = hd.class_loss(Hc, Cc, yc, scale=scale, mask=mc)
    assert torch.equal(torch.nan_to_num(again.stats, nan=9.0),
                       torch.nan_to_num(cl.stats, nan=9.0))
    dH, dC = hd.class_loss_grad(Hc, Cc, yc, cl, uc, scale=scale, mask=mc, wrt=wrt)
    dS, rH, rC, H0, C0 = P.class_grad(H.cuda(), C.cuda(), y.cuda(), t.cuda(), up.cuda(), scale,
                                      None if m is None else m.cuda())
    eH, eC = P.grad_bounds(dS, t.cuda(), d.cuda(), up.cuda(), scale, H0, C0, dtype)
    u = P.out_round(dtype)
    if wrt == "classes":
        assert dH is None
    else:
        assert dH.dtype == dtype and dH.shape == H.shape
        within(dH, rH.cpu(), (eH + u * (rH.abs() + eH)).cpu())
    if wrt == "encodings":
        assert dC is None
    else:
        assert dC.dtype == dtype and dC.shape == C.shape
        within(dC, rC.cpu(), (eC + u * (rC.abs() + eC)).cpu())
    twice = hd.class_loss_grad(Hc, Cc, yc, cl, uc, scale=scale, mask=mc, wrt=wrt)
    for a, b in zip((dH, dC), twice):
        assert (a is None) == (b is None)
        if a is not None:
            assert torch.equal(torch.nan_to_num(a.float(), nan=9.0),
                               torch.nan_to_num(b.float(), nan=9.0))
    return cl, dH, dC


# N, K, D
SMALL = [
    (1, 1, 1), (1, 2, 3), (3, 1, 5), (2, 3, 64), (5, 7, 33), (31, 31, 31), (32, 32, 32),
    (33, 33, 65), (64, 26, 127), (200, 26, 130), (129, 10, 2048), (40, 50, 3000), (20, 300, 64),
    (1, 4099, 33), (1, 1000, 4100), (7, 600, 520), (150, 200, 100), (128, 128, 128),
    (130, 257, 264), (64, 100, 10240), (300, 300, 9), (2, 20000, 72), (513, 65, 200),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mask", [None, 0.6])
@pytest.mark.parametrize("N,K,D", SMALL)
def test_class_loss(N, K, D, mask, dtype):
    hd = hd_gpu()
    announce(f"class loss {N} rows, {K} classes, D {D} {dtype} mask {mask}")
    check(hd, *make(N, K, D, dtype, seed=N * 31 + K + D, mask=mask))


# enough tiles for the large ones; classes in pieces in the backward pass
LARGE = [(3600, 3601, 40, BF16, None), (3601, 3600, 72, F32, 0.7), (70, 50000, 130, BF16, 0.5),
         (8200, 9001, 16, BF16, None), (8200, 4900, 24, F32, 0.8), (9000, 20, 600, F32, None),
         (4000, 130, 1001, BF16, 0.9)]


@pytest.mark.parametrize("N,K,D,dtype,mask", LARGE)
def test_many_tiles(N, K, D, dtype, mask):
    hd = hd_gpu()
    announce(f"class loss {N} rows, {K} classes, D {D} {dtype} mask {mask}")
    check(hd, *make(N, K, D, dtype, seed=N + K + D, mask=mask))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wrt", ["encodings", "classes"])
@pytest.mark.parametrize("N,K,D", [(70, 90, 200), (2000, 26, 300), (9, 2000, 64)])
def test_one_gradient(N, K, D, wrt, dtype):
    hd = hd_gpu()
    announce(f"class loss {N} rows, {K} classes, D {D} {dtype} wrt {wrt}")
    check(hd, *make(N, K, D, dtype, seed=5, mask=0.8), wrt=wrt)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lead,gap", [(1, 0), (0, 3), (3, 6), (8, 8)])
@pytest.mark.parametrize("N,K,D", [(45, 70, 203), (300, 290, 128)])
def test_strides(N, K, D, lead, gap, dtype):
    """Parts of wider matrices, at any alignment, with NaN beside them: nothing of what lies
    beside a row is read into it, and the results are those of contiguous rows."""
    hd = hd_gpu()
    announce(f"class loss strides {N} {K} {D} {dtype} lead {lead} gap {gap}")
    H, C, y, m, up, scale = make(N, K, D, dtype, seed=11, mask=0.7)

    def wide(x):
        w = torch.full((x.shape[0], lead + D + gap), math.nan, dtype=dtype)
        w[:, lead:lead + D] = x
        return w.cuda()[:, lead:lead + D]

    cl, dH, dC = check_on(hd, (wide(H), wide(C), y.cuda(), m.cuda(), up.cuda()),
                          (H, C, y, m, up), scale, "both", dtype)
    cl2, dH2, dC2 = check(hd, H, C, y, m, up, scale)
    for a, b in ((cl.stats, cl2.stats), (dH, dH2), (dC, dC2)):
        assert torch.equal(torch.nan_to_num(a.float(), nan=9.0),
                           torch.nan_to_num(b.float(), nan=9.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,K,D", [(5, 40, 64), (200, 300, 256), (40, 9000, 64)])
def test_nothing_open(N, K, D, dtype):
    """A mask that leaves no class, and one that leaves one."""
    hd = hd_gpu()
    announce(f"class loss, nothing open {N} {K} {D} {dtype}")
    H, C, y, _, up, scale = make(N, K, D, dtype, seed=3)
    m = torch.zeros(K, dtype=torch.bool)
    C[:] = math.nan
    cl, dH, dC = check(hd, H, C, y, m, up, scale)
    asked = (y >= 0) & (y < K)
    assert bool((cl.loss.cpu()[asked] == math.inf).all()) and bool((cl.loss.cpu()[~asked] == 0).all())
    assert bool((cl.stats.cpu() == torch.tensor([-math.inf, 0.0])).all())
    assert not bool(dH.any()) and not bool(dC.any())
    m[K // 2] = True
    C[K // 2] = 0.5
    cl, dH, dC = check(hd, H, C, y, m, up, scale)
    hit = y == K // 2
    assert bool((cl.loss.cpu()[asked & ~hit] == math.inf).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,K,D", [(6, 40, 64), (260, 300, 200)])
def test_not_finite(N, K, D, dtype):
    """NaN and infinities in rows that ask for a class: those rows alone are NaN, and with them
    every class's gradient; the other rows' loss and dH are what they are without them."""
    hd = hd_gpu()
    announce(f"class loss, not finite {N} {K} {D} {dtype}")
    H, C, y, _, up, scale = make(N, K, D, dtype, seed=4)
    y = y.clamp(0, K - 1)
    clean = hd.class_loss(H.cuda(), C.cuda(), y.cuda(), scale=scale)
    cH, _ = hd.class_loss_grad(H.cuda(), C.cuda(), y.cuda(), clean, up.cuda(), scale=scale)
    H[1, 3], H[3, 5] = math.nan, math.inf
    cl = hd.class_loss(H.cuda(), C.cuda(), y.cuda(), scale=scale)
    dH, dC = hd.class_loss_grad(H.cuda(), C.cuda(), y.cuda(), cl, up.cuda(), scale=scale)
    rest = torch.ones(N, dtype=torch.bool)
    rest[[1, 3]] = False
    assert bool(torch.isnan(cl.loss.cpu()[~rest]).all())
    assert bool(torch.isnan(cl.stats.cpu()[~rest]).all())
    assert torch.equal(cl.loss.cpu()[rest], clean.loss.cpu()[rest])
    assert bool(torch.isnan(dH.cpu()[~rest]).all()) and bool(torch.isnan(dC).all())
    assert torch.equal(dH.cpu()[rest], cH.cpu()[rest])


@pytest.mark.parametrize("size", [1e3, 1e18])
def test_far_scores(size):
    """Scores far from 0, and class vectors of the type's largest sizes."""
    hd = hd_gpu()
    announce(f"class loss, scores of size {size}")
    g = torch.Generator().manual_seed(8)
    H, C = torch.randn(50, 96, generator=g), torch.randn(70, 96, generator=g) * size
    C[:, 0] = 0
    H[:, 0] = 1
    C[:, 0] = size * 100                               # a large number in every score
    y = torch.randint(0, 70, (50,), dtype=torch.int32, generator=g)
    check(hd, H, C, y, None, torch.randn(50, generator=g), 1.0 / size)


def test_differences():
    """The gradient against differences of the loss (both in fp32 inputs, losses in 64 bits of the
    formula): a step of h in one value changes the weighted loss by h times its gradient, up to
    h^2 / 2 of a second derivative, at most sum |g| (scale |C|)^2 or (scale |H|)^2."""
    hd = hd_gpu()
    announce("class loss, differences")
    N, K, D = 12, 9, 20
    H, C, y, _, up, scale = make(N, K, D, F32, seed=6)
    cl = hd.class_loss(H.cuda(), C.cuda(), y.cuda(), scale=scale)
    dH, dC = hd.class_loss_grad(H.cuda(), C.cuda(), y.cuda(), cl, up.cuda(), scale=scale)

    def total(H, C):
        return float((P.class_loss(H, C, y, scale, None)[0] * up.double()).sum())

    h = 2.0 ** -12
    size = float(up.abs().sum()) * (scale * 5.0) ** 2 * h  # |values| < 5 here
    base = total(H.double(), C.double())
    for X, d, which in ((H, dH, 0), (C, dC, 1)):
        for at in [(0, 0), (3, 7), (8, 19)]:
            Z = X.double().clone()
            Z[at] += h
            moved = total(Z, C.double()) if which == 0 else total(H.double(), Z)
            assert abs((moved - base) / h - float(d[at])) <= size + 1e-4


def test_gradient_of_no_rows():
    hd = hd_gpu()
    announce("class loss, no rows")
    H, C = torch.zeros(0, 8).cuda(), torch.ones(5, 8).cuda()
    y = torch.zeros(0, dtype=torch.int32).cuda()
    cl = hd.class_loss(H, C, y)
    assert cl.loss.shape == (0,) and cl.stats.shape == (0, 2)
    dH, dC = hd.class_loss_grad(H, C, y, cl, torch.zeros(0).cuda())
    assert dH.shape == (0, 8) and not bool(dC.any()) and dC.shape == (5, 8)


def test_other_stream_and_graph():
    """On a stream of its own, and captured: replays on other inputs give what eager calls give,
    with eager calls between them; two graphs and an eager call do not share a workspace."""
    hd = hd_gpu()
    announce("class loss, stream and graph")
    H, C, y, m, up, scale = (v.cuda() if isinstance(v, torch.Tensor) else v
                             for v in make(40, 500, 1000, F32, seed=9, mask=0.7))
    H2 = H.flip(0).contiguous()

    def step():
        cl = hd.class_loss(H, C, y, scale=scale, mask=m)
        return (cl.loss, cl.stats) + hd.class_loss_grad(H, C, y, cl, up, scale=scale, mask=m)

    keep = H.clone()
    want = []
    for v in (keep, H2):
        H.copy_(v)
        want.append([o.clone() for o in step()])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            outs.append(step())
    for turn in (0, 1, 1, 0):
        H.copy_((keep, H2)[turn])
        for gr, out in zip(graphs, outs):
            gr.replay()
            eager = step()
            torch.cuda.synchronize()
            for a, e, b in zip(out, eager, want[turn]):
                a, e, b = (torch.nan_to_num(v, nan=9.0) for v in (a, e, b))
                assert torch.equal(a, b) and torch.equal(e, b)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = step()
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    for a, b in zip(got, want[0]):
        assert torch.equal(torch.nan_to_num(a, nan=9.0), torch.nan_to_num(b, nan=9.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_far_apart(dtype):
    """Strides at which offsets pass 32 bits: the bits of contiguous rows."""
    hd = hd_gpu()
    announce(f"class loss, rows far apart {dtype}")
    N, K, D, ld = 1100, 60, 200, 1 << 20
    H, C, y, m, up, scale = make(N, K, D, dtype, seed=13, mask=0.8)
    wide = torch.empty(N, ld, dtype=dtype, device="cuda")  # 4.6 GB in fp32
    wide[:, 7:7 + D] = H.cuda()
    far = wide[:, 7:7 + D]
    dev = (C.cuda(), y.cuda())
    got, want = [], []
    for x, out in ((far, got), (H.cuda(), want)):
        cl = hd.class_loss(x, *dev, scale=scale, mask=m.cuda())
        out += [cl.loss, cl.stats, *hd.class_loss_grad(x, *dev, cl, up.cuda(), scale=scale,
                                                       mask=m.cuda())]
    for a, b in zip(got, want):
        assert torch.equal(torch.nan_to_num(a.float(), nan=9.0), torch.nan_to_num(b.float(), nan=9.0))

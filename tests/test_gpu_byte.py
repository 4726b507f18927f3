"""Products with 8-bit weights against the rule of the header, bit for bit: the sums are exact,
the scales are applied in 64 bits and rounded once to fp32 and once to the output type."""
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


def weights(outer, inner, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-128, 128, (outer, inner), dtype=torch.int8, generator=g)
    return codes, torch.randn(outer, generator=g), g


def equal(a, b):
    a, b = a.cpu(), b.cpu()
    assert a.dtype == b.dtype and a.shape == b.shape
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    same = (a == b) | torch.isnan(a)
    assert bool(same.all()), float((a.double() - b.double()).abs()[~same].max())


# N, inner, outer
SHAPES = [(1, 1, 1), (1, 561, 617), (1, 4096, 100), (2, 17, 33), (3, 128, 32), (4, 129, 31),
          (7, 1000, 500), (16, 64, 1024), (17, 513, 65), (32, 2048, 300), (33, 300, 2000),
          (64, 1024, 129), (100, 33, 40), (129, 4096, 257), (300, 260, 900), (512, 128, 256),
          (1000, 100, 1), (4000, 200, 3700)]


@pytest.mark.parametrize("x", ["f32", "bf16", "int8", "int8s"])
@pytest.mark.parametrize("N,inner,outer", SHAPES)
def test_product(N, inner, outer, x):
    hd = hd_gpu()
    announce(f"8-bit product {N} x {inner} x {outer}, X {x}")
    codes, scales, g = weights(outer, inner, N + inner + outer)
    w = hd.byte_pack(codes.cuda(), scales.cuda())
    if x.startswith("int8"):
        q = torch.randint(-128, 128, (N, inner), dtype=torch.int8, generator=g)
        rs = torch.randn(N, generator=g) if x == "int8s" else None
        got = hd.byte_product(q.cuda(), w, row_scales=None if rs is None else rs.cuda())
        dtype = F32
    else:
        dtype = F32 if x == "f32" else BF16
        X = (torch.randn(N, inner, generator=g) * 5).to(dtype)
        q, rs = P.int8_codes(X)
        got = hd.byte_product(X.cuda(), w)
        other = BF16 if dtype == F32 else F32
        equal(hd.byte_product(X.cuda(), w, dtype=other),
              P.int8_product(q, rs, codes, scales, "identity", other))
        equal(hd.byte_product(X.cuda(), w, act="hardsign"),
              P.int8_product(q, rs, codes, scales, "hardsign", dtype))
    equal(got, P.int8_product(q, rs, codes, scales, "identity", dtype))


def test_largest_sums():
    """Codes whose sums come nearest to 2^31."""
    hd = hd_gpu()
    announce("8-bit product, largest sums")
    inner = 131071
    codes = torch.full((40, inner), -128, dtype=torch.int8)
    codes[1::2] = 127
    q = torch.full((3, inner), 127, dtype=torch.int8)
    q[1] = -128
    s = torch.ones(40)
    got = hd.byte_product(q.cuda(), hd.byte_pack(codes.cuda(), s.cuda()))
    equal(got, P.int8_product(q, None, codes, s, "identity", F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_are_not_finite(dtype):
    """A row with NaN or an infinity is NaN, rows of 0 and of the smallest numbers give 0; the rows
    beside them are what they are without."""
    hd = hd_gpu()
    announce(f"8-bit rows that are not finite {dtype}")
    codes, scales, g = weights(50, 70, 3)
    X = torch.randn(9, 70, generator=g).to(dtype)
    X[1, 3], X[2, 69], X[4, 0] = math.nan, math.inf, -math.inf
    X[5], X[6] = 0.0, 2.0 ** -130
    X[7] = 3e38
    q, rs = P.int8_codes(X)
    w = hd.byte_pack(codes.cuda(), scales.cuda())
    equal(hd.byte_product(X.cuda(), w), P.int8_product(q, rs, codes, scales, "identity", dtype))
    c, s = hd.byte_rows(X.cuda())
    assert torch.equal(c.cpu(), q)
    equal(s, rs)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("outer,inner", [(1, 1), (33, 31), (100, 617), (513, 128), (64, 1000)])
def test_quantize(outer, inner, rows, dtype):
    hd = hd_gpu()
    announce(f"8-bit weights {outer} x {inner} rows {rows} {dtype}")
    g = torch.Generator().manual_seed(outer * 7 + inner)
    W = torch.randn(outer, inner, generator=g).to(dtype)
    if outer > 20:
        W[2], W[3, inner // 2], W[4, 0] = 0.0, math.nan, math.inf
    q, s = P.int8_codes(W)
    src = W.t().contiguous() if rows else W
    wide = torch.full((src.shape[0], src.shape[1] + 3), math.nan, dtype=dtype)
    wide[:, 1:1 + src.shape[1]] = src
    w = hd.byte_quantize(wide.cuda()[:, 1:1 + src.shape[1]], inner_rows=rows)
    assert (w.outer, w.inner) == (outer, inner)
    equal(hd.byte_unpack(w), (q.float() * s[:, None]))
    X = torch.randn(5, inner, generator=g)
    xq, rs = P.int8_codes(X)
    equal(hd.byte_product(X.cuda(), w), P.int8_product(xq, rs, q, s, "identity", F32))


@pytest.mark.parametrize("x", ["f32", "bf16", "int8"])
def test_strides(x):
    """X and Y as parts of wider matrices at odd offsets; what lies beside Y stays."""
    hd = hd_gpu()
    announce(f"8-bit product, strides, X {x}")
    N, inner, outer = 37, 203, 90
    codes, scales, g = weights(outer, inner, 1)
    w = hd.byte_pack(codes.cuda(), scales.cuda())
    wide = torch.randint(-128, 128, (N, inner + 9), dtype=torch.int8, generator=g)
    if x != "int8":
        wide = wide.to(F32 if x == "f32" else BF16) * 0.37
        wide[:, :3], wide[:, 3 + inner:] = math.nan, math.inf
    X = wide[:, 3:3 + inner]
    q, rs = (X, None) if x == "int8" else P.int8_codes(X)
    for dtype in (F32, BF16):
        Y = torch.full((N, outer + 5), 7.0, dtype=dtype).cuda()
        hd.byte_product(wide.cuda()[:, 3:3 + inner], w, out=Y[:, 1:1 + outer])
        equal(Y[:, 1:1 + outer], P.int8_product(q, rs, codes, scales, "identity", dtype))
        assert bool((Y[:, 0] == 7).all()) and bool((Y[:, 1 + outer:] == 7).all())


def test_graph():
    hd = hd_gpu()
    announce("8-bit product, graph")
    codes, scales, g = weights(300, 1500, 2)
    w = hd.byte_pack(codes.cuda(), scales.cuda())
    Xs = [torch.randn(20, 1500, generator=g).cuda() for _ in range(3)]
    X = Xs[0].clone()
    want = [hd.byte_product(v, w) for v in Xs]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=stream):
        out = hd.byte_product(X, w)
    for k in (0, 1, 2, 1):
        X.copy_(Xs[k])
        gr.replay()
        eager = hd.byte_product(X, w)
        torch.cuda.synchronize()
        assert torch.equal(out, want[k]) and torch.equal(eager, want[k])

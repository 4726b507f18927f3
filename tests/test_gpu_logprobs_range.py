"""Log probabilities of scores of any size: only differences of a row's scores count, however
far from 0 they lie.

Tolerances, with u = 2^-24: a log probability t = scale (s - m) - L carries 4 u |t| from the
difference and the two products, and L a relative error of the sum: its terms' own, 4 u |z| e^z
each, at most 2 u in all the terms whose z is not 0 (|z| e^z <= 0.37, for each term of size e^z
>= e^-40 that counts), and of adding them, K / 64 + 64 roundings. Terms below e^-40 of the
largest do not show. Entropy weighs |t| <= 40 + log K by p.
"""
import math

import pytest
import torch

import ops_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
LOG2E = 1.4426950408889634


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def same(a, b):
    return bool(((a == b) | ((a != a) & (b != b))).all())


def spacing(x, dtype):
    """Distance of neighbouring values of the type at x."""
    return 2.0 ** (math.frexp(x)[1] - (8 if dtype == BF16 else 24))


def rows_of(K, dtype, scale, g):
    """Rows far from 0, of equal scores, with a few neighbours below, and of scores around the
    size from which the kernels take differences before they scale (2^24 powers of two)."""
    low = float(torch.finfo(dtype).min)
    rows = []
    for m in (1e10, -1e10, 1e12, -1e12, 1e30, -1e30, 3e9 / scale, -3e9 / scale, low, low / 2,
              -low):
        x = torch.full((K,), m).to(dtype).double()
        rows.append(x)
        x = x.clone()
        x[::3] -= spacing(m, dtype)       # (past the lowest value: -inf)
        rows.append(x)
    edge = 2.0 ** 24 / (scale * LOG2E)
    for sign in (1, -1):
        step = spacing(edge, dtype)
        if dtype == F32:
            near = torch.randint(-4, 5, (K,), generator=g).double()
        else:                             # a neighbour is thousands of powers of two away
            near = torch.randint(0, 2, (K,), generator=g).double()
        base = sign * round(edge / step) * step
        rows.append(base + near * step)
        rows.append(torch.sort(rows[-1]).values)
        rows.append(rows[-1].flip(0))
        x = torch.randn(K, generator=g).double()
        x[K // 2] = base                  # one large score among small ones
        rows.append(x)
    s = torch.stack(rows)
    s[s.abs() > -low] = -math.inf
    return s.to(dtype)


def close(a, b, tol):
    a, tol = a.cpu().double(), torch.as_tensor(tol).expand(b.shape)
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(a[torch.isinf(b)], b[torch.isinf(b)])
    ok = torch.isfinite(b)
    assert bool(((a - b).abs()[ok] <= tol[ok]).all()), float(((a - b).abs() / tol)[ok].max())


# (rows, classes): lanes to a row; a wave a row; a workgroup a row; a row in parts
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.1, 0.5, 0.69, 1.0])
@pytest.mark.parametrize("N,K", [(30, 5), (30, 100), (30, 300), (30, 1000), (2100, 1100),
                                 (600, 1100), (600, 4100), (30, 5000), (30, 20001)])
def test_scores_far_from_zero(N, K, dtype, scale):
    hd = hd_gpu()
    announce(f"far scores {N}x{K} scale {scale} {dtype}")
    g = torch.Generator().manual_seed(K)
    few = rows_of(K, dtype, scale, g)
    n = few.shape[0]
    s = few.repeat(-(-N // n), 1)
    N = s.shape[0]
    y = torch.arange(N, dtype=torch.int32) * 7 % K
    top = 9
    got = hd.logprobs(s.cuda(), y.cuda(), top=top, scale=scale)
    for a in got[1:]:                     # the copies of a row agree (but for the class asked for)
        a = a.view(N // n, n, -1)
        assert same(a, a[:1].expand_as(a))
    c32 = float(torch.tensor(scale, dtype=F32))
    ref = P.logprobs(few, y[:n], top, c32, None)
    t = ref[5]
    add = (K / 64 + 64 + 8) * P.U32
    T = 40 + math.log(K)
    close(got.logp[:n], ref[0], 4 * P.U32 * ref[0].abs().nan_to_num(0, 0, 0) + add)
    close(got.entropy[:n], ref[1], T * 2 * add)
    assert same(got.stats[:n, 0].cpu().double(), ref[2][:, 0])
    close(got.stats[:n, 1], ref[2][:, 1], add + 4 * P.U32 * ref[2][:, 1].abs())
    assert torch.equal(got.ids[:n].cpu(), ref[3])
    close(got.top_logp[:n], ref[4], 4 * P.U32 * ref[4].abs().nan_to_num(0, 0, 0) + add)

    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g)
    grad = hd.logprobs_grad(s.cuda(), y.cuda(), got, gl.cuda(), ge.cuda(), scale=scale)
    want = P.logprobs_grad(t, ref[1], y[:n], gl, ge, c32)
    # p is within its log's error, and p |t| <= 0.37; a factor T for the entropy's part
    p = torch.exp(t.nan_to_num(0, 0, -1e4))
    size = gl[:n].abs()[:, None] + ge[:n].abs()[:, None] * 2 * T
    e = c32 * size.double() * ((p * T * 4 + 1) * add)
    close(grad[:n], want, e + P.out_round(dtype) * (want.abs() + e) + 2.0 ** -133)

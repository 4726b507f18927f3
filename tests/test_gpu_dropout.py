"""Dropout against the generator written out in numpy, bit for bit."""
import math

import pytest
import torch

import learn_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SEED, STEP = 0xFEDCBA9876543210, 0x1234567890ABCDEF


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def same(a, b):
    a, b = a.cpu(), b.cpu()
    assert a.dtype == b.dtype
    assert bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
@pytest.mark.parametrize("N,D", [(1, 1), (1, 3), (3, 4), (2, 5), (300, 7), (5, 8), (1, 4097), (33, 100),
                                 (70, 1023), (9, 2049), (4, 20000)])
def test_dropout(N, D, p, dtype):
    hd = hd_gpu()
    announce(f"dropout {N} x {D} p {p} {dtype}")
    X = torch.randn(N, D, generator=torch.Generator().manual_seed(N + D)).to(dtype)
    want = P.dropout(X, p, SEED, STEP)
    same(hd.dropout(X.cuda(), p, SEED, step=STEP), want)
    at = torch.tensor([STEP], dtype=torch.int64).cuda()
    same(hd.dropout(X.cuda(), p, SEED, step=at), want)
    Y = X.cuda()
    assert hd.dropout(Y, p, SEED, step=STEP, out=Y) is Y
    same(Y, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_what_is_dropped(dtype):
    """Parts of wider matrices at odd offsets draw the same mask; what is dropped is 0 also where it
    is NaN or infinite, what is kept stays NaN; what lies beside Y stays."""
    hd = hd_gpu()
    announce(f"dropout strides {dtype}")
    N, D = 41, 203
    wide = torch.randn(N, D + 8, generator=torch.Generator().manual_seed(2)).to(dtype)
    wide[:, 5::7] = math.nan
    wide[:, 6::9] = math.inf
    X = wide[:, 3:3 + D]
    want = P.dropout(X, 0.4, 7, 0)
    same(hd.dropout(wide.cuda()[:, 3:3 + D], 0.4, 7), want)
    Y = torch.full((N, D + 6), 9.0, dtype=dtype).cuda()
    hd.dropout(wide.cuda()[:, 3:3 + D], 0.4, 7, out=Y[:, 1:1 + D])
    same(Y[:, 1:1 + D], want)
    assert bool((Y[:, 0] == 9).all()) and bool((Y[:, 1 + D:] == 9).all())


def test_gradient():
    """The call on the gradient is the backward pass: dropout is linear in X, so its gradient is
    itself, value by value; and against differences of sum(g Y), exact where p is 0.5."""
    hd = hd_gpu()
    announce("dropout, gradient")
    g = torch.Generator().manual_seed(3)
    X, G = (torch.randint(-64, 64, (6, 50), generator=g).float() for _ in range(2))
    dX = hd.dropout(G.cuda(), 0.5, 1, step=2).cpu()
    base = (hd.dropout(X.cuda(), 0.5, 1, step=2).cpu() * G).sum(dtype=torch.float64)
    for at in [(0, 0), (2, 17), (5, 49)]:
        Z = X.clone()
        Z[at] += 1.0
        moved = (hd.dropout(Z.cuda(), 0.5, 1, step=2).cpu() * G).sum(dtype=torch.float64)
        assert float(moved - base) == float(dX[at])


def test_steps_differ_and_replays_read_theirs():
    hd = hd_gpu()
    announce("dropout, graph")
    X = torch.ones(64, 1000).cuda()
    at = torch.zeros(1, dtype=torch.int64).cuda()
    stream = torch.cuda.Stream()
    hd.dropout(X, 0.3, 5, step=at)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=stream):
        Y = hd.dropout(X, 0.3, 5, step=at)
    seen = []
    for k in (3, 4, 2 ** 40, 3):
        at.fill_(k)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, hd.dropout(X, 0.3, 5, step=k))
        seen.append(Y.clone())
    assert torch.equal(seen[0], seen[3]) and not torch.equal(seen[0], seen[1])
    kept = float((seen[2] != 0).double().mean())  # 64000 draws: within six deviations
    assert abs(kept - 0.7) < 6 * math.sqrt(0.21 / 64000)


def test_rows_past_a_launch():
    """More rows than a launch has blocks: a block walks over them."""
    hd = hd_gpu()
    announce("dropout, many rows")
    N = 65535 * 256 + 1000  # of one piece each, 256 to a block
    X = torch.ones(N, 2, dtype=BF16).cuda()
    Y = hd.dropout(X, 0.5, 11, step=1)
    torch.cuda.synchronize()
    for n in (0, 255, 65535 * 256 - 1, 65535 * 256, N - 1):
        w = P.philox((0, n, 1, 0), (11, 0))
        want = [2.0 if int(w[e]) >= 2 ** 31 else 0.0 for e in range(2)]
        assert Y[n].cpu().tolist() == want

"""The operators behind learning together, as a user's training step runs them: readings encoded
through 8-bit base vectors, dropout, the cross entropy, its gradient, dropout's backward pass."""
import pytest
import torch

import learn_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step(dtype):
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"a training step {dtype}")
    N, F, D, K, p, scale = 150, 70, 1000, 12, 0.25, 0.05
    g = torch.Generator().manual_seed(1)
    X, B = torch.randn(N, F, generator=g), torch.randn(F, D, generator=g)
    C = torch.randn(K, D, generator=g).to(dtype)
    y = torch.randint(0, K, (N,), dtype=torch.int32, generator=g)
    y[::9] = -1                                       # rows that fill up the batch
    up = torch.full((N,), 1.0 / N)
    w = hd.byte_quantize(B.cuda(), inner_rows=True)
    H = hd.byte_product(X.cuda(), w, act="hardsign", dtype=dtype)
    q, rs = P.int8_codes(X)
    wq, ws = P.int8_codes(B.t().contiguous())
    assert torch.equal(H.cpu(), P.int8_product(q, rs, wq, ws, "hardsign", dtype))
    step = torch.tensor([41], dtype=torch.int64).cuda()
    Hd = hd.dropout(H, p, 99, step=step)
    want = P.dropout(H.cpu(), p, 99, 41)
    assert torch.equal(Hd.cpu(), want)
    cl = hd.class_loss(Hd, C.cuda(), y.cuda(), scale=scale)
    loss, _, t, d, _ = P.class_loss(want, C, y, scale, None)
    assert bool(((cl.loss.cpu().double() - loss).abs() <= d[:, 0] + 2 * P.U32 * loss.abs()).all())
    dH, dC = hd.class_loss_grad(Hd, C.cuda(), y.cuda(), cl, up.cuda(), scale=scale)
    dS, rH, rC, H0, C0 = P.class_grad(want, C, y, t, up, scale, None)
    eH, eC = P.grad_bounds(dS, t, d, up, scale, H0, C0, dtype)
    u = P.out_round(dtype)
    assert bool(((dC.cpu().double() - rC).abs() <= eC + u * (rC.abs() + eC)).all())
    back = hd.dropout(dH, p, 99, step=step)
    assert torch.equal(back.cpu(), P.dropout(dH.cpu(), p, 99, 41))
    assert not bool(back[y.cuda() < 0].any())
    # the same loss as the stored scores give, through the operators that were there
    if dtype == F32:
        _, S = hd.similarity(Hd, C.cuda(), return_scores=True)
        lp = hd.logprobs(S, y.cuda(), scale=scale)
        e = d[:, 0] + 2 * P.U32 * loss.abs()
        assert bool(((lp.logp.cpu().double() + cl.loss.cpu().double()).abs() <= 2 * e).all())


@pytest.mark.parametrize("n", [1, 30, 128, 129])
def test_few_rows_keep_more_of_the_gradient(n):
    """bf16 gradients of up to 128 rows: dS is two bf16 values, whose rounding is 2^-16 of it (and
    more rows' one value 2^-8), so dC of rows alone in their class is the product rounded once."""
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class gradient, {n} rows in bf16")
    D, K, scale = 256, n, 0.05
    g = torch.Generator().manual_seed(n)
    H, C = (torch.randn(n, D, generator=g).to(BF16) for _ in range(2))
    y = torch.arange(n, dtype=torch.int32)
    up = torch.rand(n, generator=g) + 0.5
    cl = hd.class_loss(H.cuda(), C.cuda(), y.cuda(), scale=scale)
    dH, dC = hd.class_loss_grad(H.cuda(), C.cuda(), y.cuda(), cl, up.cuda(), scale=scale)
    _, _, t, d, _ = P.class_loss(H, C, y, scale, None)
    dS, rH, rC, H0, C0 = P.class_grad(H, C, y, t, up, scale, None)
    eH, eC = P.grad_bounds(dS, t, d, up, scale, H0, C0, F32)
    part = 2.0 ** -16 if n <= 128 else 2.0 ** -8
    for got, ref, e, size in ((dH, rH, eH, dS.abs() @ C0.abs()),
                              (dC, rC, eC, dS.t().abs() @ H0.abs())):
        e = e + part * size
        assert bool(((got.cpu().double() - ref).abs() <= e + 2.0 ** -8 * (ref.abs() + e)).all())

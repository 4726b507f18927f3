"""The operators behind answers and learning together, as examples/answers.py runs them."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from gpu_util import check_against_oracle, torch_or_skip

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def test_learning_and_answering():
    torch_or_skip()
    import answers as ex
    import paper_2506_09282_amd as hd
    F, D, K, N = 70, 1536, 5, 1200
    B = torch.randn(F, D, generator=torch.Generator().manual_seed(1)).cuda()
    X, y = ex.readings(N, F, K, seed=2)
    C = ex.bundled(X, B, y, K)
    H = hd.encode(X, B)
    # encodings are kept exactly, so a step is the plain gradient step
    C2, losses = ex.refine(C, H, y, 1, rate=50.0, scale=0.02)
    S = H.double() @ C.double().t()
    p = torch.softmax(0.02 * S, 1)
    p[torch.arange(N, device="cuda"), y.long()] -= 1.0
    plain = C.double() - 50.0 * (0.02 / N) * p.t() @ H.double()
    # the step's fp32 sums over N rows of terms up to 1 / N
    assert float((C2.double() - plain).abs().max()) <= 50.0 * 0.02 * N * 2.0 ** -24
    _, losses = ex.refine(C, H, y, 12, rate=50.0, scale=0.02)
    assert all(b < a for a, b in zip(losses, losses[1:]))
    # four bits: the same answers as the oracle's on the weights that the codes stand for
    model = ex.FourBitModel(B, C2, group=32)
    Xt, _ = ex.readings(33, F, K, seed=5)
    S4 = model.scores(Xt)
    lp = model.answer(Xt, 0.02, top=K)
    Bq = hd.nibble_unpack(model.B).t().contiguous().cpu().numpy()
    Cq = hd.nibble_unpack(model.C).cpu().numpy()
    rep, _ = check_against_oracle(Xt.cpu().numpy(), Bq, Cq, lp.ids[:, 0].cpu().numpy(),
                                  S4.cpu().numpy())
    assert rep["ok"], rep
    ref = torch.log_softmax(0.02 * S4.double(), 1)
    assert torch.equal(lp.ids.long(), torch.argsort(S4, dim=1, descending=True, stable=True))
    assert float((lp.top_logp.double() - ref.gather(1, lp.ids.long())).abs().max()) < 1e-5
    one = model.answer(Xt[:1], 0.02, top=K)
    assert torch.equal(one.ids, lp.ids[:1])
    assert np.isfinite(oracle.infer(Xt[:1].cpu().numpy(), Bq, Cq)["S"]).all()

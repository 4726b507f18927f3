"""8-bit products of parts of wider matrices in every kernel: rows that code themselves, few rows,
tiles whose reduction is in parts and tiles that write Y themselves."""
import math

import pytest
import torch

import learn_plain as P
from gpu_util import announce, torch_or_skip
from test_gpu_byte import equal, weights

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("x", ["f32", "bf16", "int8", "int8s"])
@pytest.mark.parametrize("N,inner,outer", [(1, 203, 90), (2, 203, 90), (37, 203, 90),
                                           (100, 1003, 90), (100, 333, 31), (300, 77, 1001),
                                           (4000, 203, 3701)])
def test_strides(N, inner, outer, x):
    """What lies beside X is not read into its rows, and what lies beside Y stays."""
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"8-bit product, strides, {N} x {inner} x {outer}, X {x}")
    codes, scales, g = weights(outer, inner, N)
    w = hd.byte_pack(codes.cuda(), scales.cuda())
    wide = torch.randint(-128, 128, (N, inner + 9), dtype=torch.int8, generator=g)
    rs = torch.randn(N, generator=g) if x == "int8s" else None
    if x in ("f32", "bf16"):
        wide = wide.to(F32 if x == "f32" else BF16) * 0.37
        wide[:, :3], wide[:, 3 + inner:] = math.nan, math.inf
    X = wide[:, 3:3 + inner]
    q, s = (X, rs) if x.startswith("int8") else P.int8_codes(X)
    for dtype in (F32, BF16):
        Y = torch.full((N, outer + 5), 7.0, dtype=dtype).cuda()
        hd.byte_product(wide.cuda()[:, 3:3 + inner], w, out=Y[:, 1:1 + outer],
                        row_scales=None if rs is None else rs.cuda())
        equal(Y[:, 1:1 + outer], P.int8_product(q, s, codes, scales, "identity", dtype))
        assert bool((Y[:, 0] == 7).all()) and bool((Y[:, 1 + outer:] == 7).all())

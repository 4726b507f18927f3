"""One of the two gradients alone, in a workspace of its own size: the bits that the call for both
gives, with classes in pieces, products in parts and large tiles."""
import ctypes

import pytest
import torch

from gpu_util import announce, torch_or_skip
from test_gpu_class import make

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

SIZES = [(64, 100, 1030), (9000, 20, 600), (3601, 3600, 72), (8200, 4900, 24)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,K,D", SIZES)
def test_bits_of_one_gradient(N, K, D, dtype):
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class gradient alone {N} rows, {K} classes, D {D} {dtype}")
    H, C, y, m, up, scale = (v.cuda() if isinstance(v, torch.Tensor) else v
                             for v in make(N, K, D, dtype, seed=N + D, mask=0.8))
    cl = hd.class_loss(H, C, y, scale=scale, mask=m)
    dH, dC = hd.class_loss_grad(H, C, y, cl, up, scale=scale, mask=m)
    L, dt = hd.lib(), hd.HD_F32 if dtype == F32 else hd.HD_BF16
    for h, c in ((1, 0), (0, 1)):
        need = L.hd_class_loss_grad_workspace_bytes_of(N, D, K, dt, h, c)
        guard = 4096
        ws = torch.full((need + guard,), 0x5A, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(H if h else C)
        st = L.hd_class_loss_grad(
            H.data_ptr(), D, C.data_ptr(), D, m.data_ptr(), y.data_ptr(), ctypes.c_float(scale),
            cl.stats.data_ptr(), up.data_ptr(), out.data_ptr() if h else None,
            out.data_ptr() if c else None, N, D, K, dt, ws.data_ptr(), need,
            torch.cuda.current_stream().cuda_stream)
        assert st == hd.HD_OK
        assert bool((ws[need:] == 0x5A).all())  # nothing past its end
        want = dH if h else dC
        assert torch.equal(torch.nan_to_num(out.float(), nan=9.0),
                           torch.nan_to_num(want.float(), nan=9.0))
        alone = hd.class_loss_grad(H, C, y, cl, up, scale=scale, mask=m,
                                   wrt="encodings" if h else "classes")
        assert alone[1 if h else 0] is None
        assert torch.equal(torch.nan_to_num(alone[0 if h else 1].float(), nan=9.0),
                           torch.nan_to_num(want.float(), nan=9.0))

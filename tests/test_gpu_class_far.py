"""The cross entropy of class scores at the largest row stride, where offsets within a tile of 256
rows come just under 2^32 bytes, and of parts of wider matrices in the large tile: the bits of
contiguous rows."""
import math

import pytest
import torch

from gpu_util import announce, torch_or_skip
from test_gpu_class import make

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def results(hd, H, C, y, m, up, scale):
    cl = hd.class_loss(H, C, y, scale=scale, mask=m)
    return [cl.loss, cl.stats, *hd.class_loss_grad(H, C, y, cl, up, scale=scale, mask=m)]


def same_bits(got, want):
    for a, b in zip(got, want):
        assert torch.equal(torch.nan_to_num(a.float(), nan=9.0),
                           torch.nan_to_num(b.float(), nan=9.0))


# narrow tiles of 256 rows of H, and of 256 classes
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,K,which", [(256, 26, "H"), (20, 300, "C")])
def test_largest_stride(N, K, which, dtype):
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class loss, largest stride of {which} {dtype}")
    D, ld = 200, 1 << 22
    H, C, y, m, up, scale = (v.cuda() if isinstance(v, torch.Tensor) else v
                             for v in make(N, K, D, dtype, seed=17, mask=0.8))
    want = results(hd, H, C, y, m, up, scale)
    x = H if which == "H" else C
    wide = torch.empty(x.shape[0], ld, dtype=dtype, device="cuda")  # 4 to 5 GB in fp32
    wide[:, ld - D:] = x
    far = wide[:, ld - D:]
    got = results(hd, far if which == "H" else H, far if which == "C" else C, y, m, up, scale)
    same_bits(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lead,gap", [(1, 0), (3, 6), (8, 8)])
def test_strides_of_the_large_tile(lead, gap, dtype):
    torch_or_skip()
    import paper_2506_09282_amd as hd
    announce(f"class loss, strides of the large tile, {dtype} lead {lead} gap {gap}")
    N, K, D = 3601, 3600, 203
    H, C, y, m, up, scale = (v.cuda() if isinstance(v, torch.Tensor) else v
                             for v in make(N, K, D, dtype, seed=19, mask=0.7))

    def wide(x):
        w = torch.full((x.shape[0], lead + D + gap), math.nan, dtype=dtype, device="cuda")
        w[:, lead:lead + D] = x
        return w[:, lead:lead + D]

    same_bits(results(hd, wide(H), wide(C), y, m, up, scale), results(hd, H, C, y, m, up, scale))

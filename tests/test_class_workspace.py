"""Workspaces of the class gradient, without a GPU: a call for one of the two gradients asks for
nothing of the other's, and is refused with less than its own."""
import pytest

import paper_2506_09282_amd as hd

FAKE = 0x10000  # never dereferenced: validation fails first
F32, BF16 = hd.HD_F32, hd.HD_BF16
MIB = 1 << 20

# N, D, K: classes in pieces (dH's sums), products in parts, one piece whole, a piece of 256 classes
SIZES = [(65536, 2560, 16384), (64, 10240, 100), (16384, 10240, 26), (4096, 4096, 4096),
         (300000, 64, 1000)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,K", SIZES)
def test_one_gradient_needs_no_more_than_its_own(N, D, K, dt):
    L = hd.lib()
    both, dH, dC = (L.hd_class_loss_grad_workspace_bytes_of(N, D, K, dt, h, c)
                    for h, c in ((1, 1), (1, 0), (0, 1)))
    assert both == L.hd_class_loss_grad_workspace_bytes(N, D, K, dt)
    assert 0 < dH <= both and 0 < dC <= both
    if N * K * 4 > 128 * MIB and K > 256:  # in pieces: the sums of dH
        assert both - dC >= 4 * N * D
        # dS, parts of at most 512 tiles of 128 x 128 fp32 sums, and bits
        assert dC <= max(128 * MIB, 1024 * N) + 32 * MIB + MIB

    def f(need, h, c):
        return L.hd_class_loss_grad(FAKE, D, FAKE, D, None, FAKE, 1.0, FAKE, FAKE,
                                    FAKE if h else None, FAKE if c else None, N, D, K, dt, FAKE,
                                    need - 1, None)

    assert f(both, 1, 1) == f(dH, 1, 0) == f(dC, 0, 1) == hd.HD_ERR_WORKSPACE


def test_refusals():
    L = hd.lib()
    for bad in ((0, 8, 10, F32, 1, 1), (4, 8, 10, hd.HD_I8, 1, 1), (4, 8, 10, F32, 0, 0)):
        assert L.hd_class_loss_grad_workspace_bytes_of(*bad) == 0

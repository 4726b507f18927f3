"""The workspace that the binding keeps for rows split over workgroups."""
import pytest
import torch

import ops_plain as P
from gpu_util import torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def test_one_workspace_for_all_shapes():
    """Shapes of all sizes after one another keep one buffer, and give what each gives in a
    zeroed one of its own."""
    hd = hd_gpu()
    stream = torch.cuda.Stream()
    g = torch.Generator().manual_seed(0)
    with torch.cuda.stream(stream):
        before = len(hd._ws_cache)
        shapes = [(1, 40000, F32), (2, 100003, BF16), (300, 3000, F32), (7, 5000, BF16),
                  (1, 131072, F32), (511, 2049, BF16), (3, 30000, F32), (100, 20001, BF16),
                  (1, 1025, F32), (64, 9001, F32)]
        for N, K, dtype in shapes + shapes[::-1]:
            s = torch.randn(N, K, generator=g).to(dtype).cuda()
            y = torch.randint(0, K, (N,), generator=g, dtype=torch.int32).cuda()
            need = hd.logprobs_workspace_bytes(N, K, dtype)
            own = torch.zeros(need, dtype=torch.uint8, device="cuda") if need else None
            got = hd.logprobs(s, y, top=11)
            want = hd.logprobs(s, y, top=11, workspace=own)
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        assert len(hd._ws_cache) == before + 1
    stream.synchronize()


def test_results_of_split_rows():
    hd = hd_gpu()
    g = torch.Generator().manual_seed(4)
    for N, K in ((2, 60001), (5, 4100)):
        s = torch.randn(N, K, generator=g)
        got = hd.logprobs(s.cuda(), top=3)
        ref = P.logprobs(s, None, 3, 1.0, None)
        assert torch.equal(got.ids.cpu(), ref[3])
        # |z| < 16, and the sum of K terms
        assert bool(((got.entropy.cpu().double() - ref[1]).abs()
                     <= 16 * (K / 64 + 72) * P.U32 * 2).all())


def test_refused_workspaces():
    """The kernels write to it: memory of the host, or of other tensors between, is refused."""
    hd = hd_gpu()
    s = torch.randn(2, 30000, generator=torch.Generator().manual_seed(1)).cuda()
    need = hd.logprobs_workspace_bytes(2, 30000, F32)
    assert need > 0
    for bad in (torch.zeros(need, dtype=torch.uint8),
                torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2],
                torch.zeros(need, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError, match="workspace"):
            hd.logprobs(s, workspace=bad)

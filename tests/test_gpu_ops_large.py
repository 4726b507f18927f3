"""Operators on data past the caches, whose loads and stores are others, and on offsets that
do not fit 32 bits."""
import pytest
import torch

import ops_plain as P
from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def same(a, b):
    return bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("top", [0, 7])
@pytest.mark.parametrize("N,K,dtype", [(1100, 50003, F32), (2100, 50003, BF16)])
def test_logprobs_past_the_caches(N, K, dtype, top, masked):
    """A row's results do not depend on how much there is besides it."""
    hd = hd_gpu()
    announce(f"logprobs {N}x{K} top {top} {dtype} mask {masked}")
    g = torch.Generator(device="cuda").manual_seed(K + N)
    s = (3 * torch.randn(N, K, generator=g, device="cuda")).to(dtype)
    y = torch.randint(0, K, (N,), dtype=torch.int32, generator=g, device="cuda")
    m = torch.rand(N, K, generator=g, device="cuda") < 0.5 if masked else None
    if masked:
        m[N - 1] = False
    whole = hd.logprobs(s, y, top=top, mask=m)
    few = slice(N - 600, N)  # (as many as are not split)
    part = hd.logprobs(s[few], y[few], top=top, mask=m[few] if masked else None)
    for a, b in zip(whole, part):
        assert a is None or same(a[few], b)
    pick = torch.tensor([0, N // 2])
    at = pick.cuda()
    ref = P.logprobs(s[at].cpu(), y[at].cpu(), top, 1.0, m[at].cpu() if masked else None)
    # |z| < 64 here; bounds as for the small calls
    tol = (4 * 64 + 2 * (K / 64 + 64)) * P.U32
    logp, there = whole.logp[at].cpu().double(), torch.isfinite(ref[0])
    assert torch.equal(logp[~there], ref[0][~there])  # -inf: the class is masked
    assert bool(((logp - ref[0]).abs()[there] <= tol).all())
    assert bool(((whole.entropy[at].cpu().double() - ref[1]).abs()
                 <= tol + 64 * (K / 64 + 72) * P.U32).all())
    if top:
        assert torch.equal(whole.ids[at].cpu(), ref[3])

    gl = torch.randn(N, generator=g, device="cuda")
    grad = hd.logprobs_grad(s, y, whole, g_logp=gl, g_entropy=gl, mask=m)
    few = slice(N - 100, N)
    sub = hd.LogProbs(*(None if v is None else v[few].contiguous() for v in whole))
    again = hd.logprobs_grad(s[few], y[few], sub, g_logp=gl[few], g_entropy=gl[few],
                             mask=m[few] if masked else None)
    assert same(grad[few], again)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [10240, 10241, 10244])
def test_checkpoints_past_the_caches(D, dtype):
    hd = hd_gpu()
    N = 64 * 80
    announce(f"ckpt {N}x{D} {dtype}")
    H = torch.randn(N, D, generator=torch.Generator(device="cuda").manual_seed(4),
                    device="cuda").to(dtype)
    kept = hd.ckpt_store(H)
    back = hd.ckpt_load(kept, dtype=dtype)
    for n0 in (0, 64 * 37, N - 64):  # whole groups: the same scales
        small = hd.ckpt_store(H[n0:n0 + 64])
        assert same(hd.ckpt_load(small, dtype=dtype), back[n0:n0 + 64])
    ref = P.ckpt_values(*P.ckpt(H[:64].cpu()))
    assert torch.equal(back[:64].cpu(), ref.float().to(dtype))


# Rows 2^31 elements apart: the last one's offset passes 2^32.
FAR = 1 << 31


def far_rows(rows):
    n, k = rows.shape
    room = torch.empty((n - 1) * FAR + k, dtype=rows.dtype, device="cuda")
    out = room.as_strided((n, k), (FAR, 1))
    out.copy_(rows)
    return out


@pytest.mark.parametrize("K", [26, 4099])
def test_logprobs_of_far_rows(K):
    hd = hd_gpu()
    announce(f"far rows {K}")
    s = torch.randn(4, K, generator=torch.Generator().manual_seed(K)).to(BF16).cuda()
    y = torch.tensor([0, 1, K - 1, 5], dtype=torch.int32, device="cuda")
    near, far = s, far_rows(s)
    a, b = hd.logprobs(near, y, top=4), hd.logprobs(far, y, top=4)
    assert all(same(u, v) for u, v in zip(a, b))
    g = torch.ones(4, device="cuda")
    want = hd.logprobs_grad(near, y, a, g_logp=g, g_entropy=g)
    assert same(hd.logprobs_grad(far, y, a, g_logp=g, g_entropy=g, out=far), want)
    assert same(far.contiguous(), want)


def test_checkpoint_and_products_of_far_rows():
    hd = hd_gpu()
    announce("far rows of activations")
    H = torch.randn(4, 300, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    far = far_rows(H)
    near_kept, far_kept = hd.ckpt_store(H), hd.ckpt_store(far)
    assert torch.equal(near_kept.image, far_kept.image)
    w = hd.nibble_quantize(torch.randn(40, 300, device="cuda"), group=32)
    assert same(hd.nibble_product(far, w), hd.nibble_product(H, w))
    for K in (20, 40):
        dS = torch.randn(4, K, generator=torch.Generator().manual_seed(K)).to(BF16).cuda()
        del far
        far = far_rows(dS)
        assert same(hd.ckpt_class_grad(far, near_kept), hd.ckpt_class_grad(dS, near_kept))
    want = hd.ckpt_load(near_kept, dtype=BF16)
    del far
    far = far_rows(torch.zeros_like(H))
    assert same(hd.ckpt_load(near_kept, out=far), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_of_more_outputs_than_a_launch_holds(dtype):
    """4096 rows and 4.2 million outputs: 2^32 threads and more, 34 GB of results. Whole numbers:
    exact in every order of the sums, one rounding is left."""
    hd = hd_gpu()
    N, inner, group = 4096, 400, 32
    outer = 16 * 4 * 65536 + 16 * 700 + 5      # 65536 workgroups of four tiles, and more
    announce(f"nibble {N}x{outer}x{inner} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 256, (outer, inner // 2), dtype=torch.uint8, generator=g,
                          device="cuda")
    ngroups = -(-inner // group)
    ones = torch.ones(outer, ngroups, dtype=BF16, device="cuda")
    z = torch.randint(0, 16, (outer, ngroups), dtype=torch.uint8, generator=g, device="cuda")
    X = torch.randint(-3, 4, (N, inner), generator=g, device="cuda").to(dtype)
    for zeros in (z, None):
        w = hd.nibble_pack(codes, ones, zeros, inner=inner, group=group)
        Y = hd.nibble_product(X, w, dtype=BF16)
        for o in list(range(0, outer, 524288)) + [outer - 20000]:
            part = slice(o, min(outer, o + 20000))
            W = hd.nibble_unpack(hd.nibble_pack(codes[part], ones[part],
                                                None if zeros is None else zeros[part],
                                                inner=inner, group=group))
            assert torch.equal(Y[:, part], (X.float() @ W.t()).to(BF16))
        del Y, w

"""Log probabilities with entropy and alternatives, and their gradient, against the
formulas in 64 bits.

Tolerances: z = scale (s - m) carries two roundings of its size, log2(e) scale one
more, exp and log are within two units, and a sum of K terms within log2(K) + 32
roundings (threads add chunks in order, then in a tree), all of positive terms. With
u = 2^-24 and |z| <= Z a log probability is within (4 Z + K_terms) u of its value.
"""
import math

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


def cuda(t):
    return None if t is None else t.cuda()


def sum_terms(K):
    """Additions one after another on the way of one term: a thread's own (a row is
    walked by at least 64 lanes, or held by one to 16 a lane), then the tree."""
    return K / 64 + 64


def check(got, ref, scores, scale, K, top):
    logp, entropy, stats, ids, best, t = ref
    fin = t[torch.isfinite(t)]
    Z = float(-fin.min()) + 1 if fin.numel() else 1.0
    tol = (4 * Z + 2 * sum_terms(K)) * P.U32

    def close(a, b, tol):
        a, b = a.cpu().double(), b
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        assert torch.equal(torch.isinf(a), torch.isinf(b))
        ok = torch.isfinite(b)
        assert torch.equal(a[torch.isinf(a)], b[torch.isinf(b)])
        assert bool(((a - b).abs()[ok] <= tol + 2 * P.U32 * b[ok].abs()).all()), \
            float((a - b).abs()[ok].max())

    if got.logp is not None:
        close(got.logp, logp, tol)
    # entropy adds |t| p: its error is that of t, and of the sum of p |t| <= Z
    close(got.entropy, entropy, tol + Z * (sum_terms(K) + 8) * P.U32)
    close(got.stats[:, 1], stats[:, 1], tol)
    m = got.stats[:, 0].cpu().double()
    assert torch.equal(torch.nan_to_num(m, nan=9.0), torch.nan_to_num(stats[:, 0], nan=9.0))
    if top:
        assert torch.equal(got.ids.cpu(), ids)
        close(got.top_logp, best, tol)


def random_scores(N, K, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    s = (torch.randn(N, K, generator=g) * spread).to(dtype)
    y = torch.randint(-1, K + 1, (N,), dtype=torch.int32, generator=g)  # -1 and K ask for none
    return s, y, g


# N, K, top, dtype, scale
SHAPES = [
    (1, 1, 1, F32, 1.0), (3, 1, 4, BF16, 1.0), (5, 2, 2, F32, 0.3), (70, 6, 3, F32, 1.0),
    (33, 26, 5, BF16, 1.0), (40, 32, 32, F32, 2.0), (9, 33, 8, F32, 1.0), (20, 100, 10, BF16, 0.7),
    (7, 128, 32, F32, 1.0), (7, 129, 3, F32, 1.0), (5, 256, 20, F32, 1.0), (5, 257, 20, BF16, 1.0),
    (6, 1000, 32, F32, 1.0), (4, 1024, 1, BF16, 1.0), (4, 1025, 32, F32, 1.0),
    (3, 1031, 8, BF16, 1.0), (3, 4096, 20, F32, 1.0), (2, 4099, 20, BF16, 1.0),
    (1, 10007, 32, F32, 1.0), (1, 40000, 5, BF16, 1.0), (1, 131072, 20, F32, 1.0),
    (600, 2000, 4, F32, 1.0), (300, 5003, 0, BF16, 1.0), (2, 100003, 32, BF16, 0.5),
]


@pytest.mark.parametrize("mask", ["none", "shared", "rows"])
@pytest.mark.parametrize("N,K,top,dtype,scale", SHAPES)
def test_logprobs(N, K, top, dtype, scale, mask):
    hd = hd_gpu()
    announce(f"logprobs {N}x{K} top {top} {dtype} mask {mask}")
    s, y, g = random_scores(N, K, dtype, seed=N * 7 + K)
    m = None
    if mask == "shared":
        m = torch.rand(K, generator=g) < 0.6
    elif mask == "rows":
        m = torch.rand(N, K, generator=g) < 0.6
        m[0] = False                      # nothing is left
        m[-1] = False
        m[-1, K // 2] = True              # one class is left
    if m is not None:                     # what is masked holds anything
        off = ~m if m.dim() == 2 else (~m)[None].expand(N, K)
        s[off] = torch.tensor([math.nan, math.inf, 3e38])[
            torch.randint(0, 3, (int(off.sum()),), generator=g)].to(dtype)
    got = hd.logprobs(s.cuda(), y.cuda(), top=top, scale=scale, mask=cuda(m))
    check(got, P.logprobs(s, y, top, scale, m), s, scale, K, top)
    twice = hd.logprobs(s.cuda(), y.cuda(), top=top, scale=scale, mask=cuda(m))
    for a, b in zip(got, twice):  # the same bits, and a workspace left clean
        assert a is None or bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("top", [0, 3, 32])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,K", [(2100, 1025), (2050, 3001), (2049, 8192), (40, 100), (2100, 100)])
def test_many_rows(N, K, dtype, top, masked):
    """Rows of a wave each; and short rows whose form depends on their number."""
    hd = hd_gpu()
    announce(f"logprobs {N}x{K} top {top} {dtype} mask {masked}")
    s, y, g = random_scores(N, K, dtype, seed=N + K)
    s[3] = 1.0                                     # ties
    s[4, ::2], s[4, 1::2] = 0.0, -0.0
    s[5, K // 2], s[6, K - 1], s[7] = math.nan, math.inf, -math.inf
    s[8] = torch.arange(K).to(dtype)               # each beats all before it
    s[9] = torch.finfo(dtype).min
    m = torch.rand(N, K, generator=g) < 0.6 if masked else None
    if masked:
        m[N - 1] = False
        s[5, K // 2] = s[6, K - 1] = math.nan
        m[5, K // 2] = m[6, K - 1] = False
    got = hd.logprobs(s.cuda(), y.cuda(), top=top, scale=0.7, mask=cuda(m))
    for rows in (slice(0, 12), slice(N - 8, N)):
        sub = hd.LogProbs(*(None if v is None else v[rows] for v in got))
        mm = m[rows] if masked else None
        check(sub, P.logprobs(s[rows], y[rows], top, 0.7, mm), s[rows], 0.7, K, top)
    # rows between: the same alternatives as in calls of a few rows
    for n0 in range(12, N, 500):
        few = hd.logprobs(s[n0:n0 + 7].cuda(), y[n0:n0 + 7].cuda(), top=top, scale=0.7,
                          mask=cuda(m[n0:n0 + 7]) if masked else None)
        if top:
            assert torch.equal(few.ids, got.ids[n0:n0 + 7])
    off = torch.empty(N, K + 5, dtype=dtype, device="cuda")[:, 3:3 + K]
    off.copy_(s)
    wide = hd.logprobs(off, y.cuda(), top=top, scale=0.7, mask=cuda(m))
    for a, b in zip(wide, got):  # strides and alignment change no bit
        assert a is None or bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("K", [5, 32, 100, 1000, 3000, 20001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ties_and_extremes(K, dtype):
    """Equal scores, both zeros, the lowest finite value, infinities and NaN."""
    hd = hd_gpu()
    low = torch.finfo(dtype).min
    rows = [
        torch.zeros(K), torch.full((K,), low), torch.full((K,), -math.inf),
        torch.arange(K).remainder(3).float(), -torch.arange(K).remainder(7).float(),
        torch.full((K,), low), torch.full((K,), 5.0), torch.zeros(K), torch.zeros(K),
        torch.linspace(-50, 50, K), torch.linspace(50, -50, K), torch.zeros(K),
    ]
    rows[0][1::2] = -0.0
    rows[5][K // 2] = 2.0
    rows[6][K - 1] = -math.inf
    rows[7][K // 3] = math.nan
    rows[8][K - 2] = math.inf
    rows[11][:] = -math.inf
    rows[11][K - 1] = low
    s = torch.stack(rows).to(dtype)
    n = s.shape[0]
    y = torch.tensor([K - 1, 0, 1, K // 2, -1, K // 2, K - 1, 0, -1, K - 1, 0, K - 1],
                     dtype=torch.int32)
    announce(f"ties K={K} {dtype}")
    top = min(32, 6)
    got = hd.logprobs(s.cuda(), y.cuda(), top=top)
    check(got, P.logprobs(s, y, top, 1.0, None), s, 1.0, K, top)
    assert got.ids[0].tolist() == [k if k < K else -1 for k in range(top)]
    assert got.entropy.shape == (n,)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ascending_scores(dtype):
    """Every score beats all before it: each enters the list of alternatives."""
    hd = hd_gpu()
    K = 5000
    s = torch.arange(K).float()[None].repeat(2, 1) / 64
    s[1] = s[1].flip(0)
    s = s.to(dtype)
    y = torch.tensor([0, 0], dtype=torch.int32)
    check(hd.logprobs(s.cuda(), y.cuda(), top=32), P.logprobs(s, y, 32, 1.0, None), s, 1.0, K, 32)


def test_large_scores_and_no_class():
    """Similarities of bipolar vectors are large numbers; y may be left out."""
    hd = hd_gpu()
    g = torch.Generator().manual_seed(0)
    s = torch.randint(-10240, 10241, (50, 26), generator=g).float()
    got = hd.logprobs(s.cuda(), top=3, scale=0.01)
    assert got.logp is None
    check(got, P.logprobs(s, None, 3, 0.01, None), s, 0.01, 26, 3)


@pytest.mark.parametrize("K", [26, 700, 3000, 9001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(K, dtype):
    hd = hd_gpu()
    N = 5
    s, y, g = random_scores(N, K, dtype, seed=K)
    wide = torch.zeros(N, K + 7, dtype=dtype).cuda()
    mwide = torch.zeros(N, K + 5, dtype=torch.bool)
    m = torch.rand(N, K, generator=g) < 0.5
    mwide[:, 3:3 + K] = m
    for off in (0, 1, 2, 5):
        wide[:, off:off + K] = s.cuda()
        x = wide[:, off:off + K]
        mm = mwide.cuda()[:, 3:3 + K]
        a = hd.logprobs(x, y.cuda(), top=4, mask=mm)
        b = hd.logprobs(s.cuda(), y.cuda(), top=4, mask=m.cuda())
        for u, v in zip(a, b):
            assert torch.equal(u, v)
        gl = torch.randn(N, generator=torch.Generator().manual_seed(1)).cuda()
        ref = hd.logprobs_grad(s.cuda(), y.cuda(), b, gl, gl, mask=m.cuda())
        out = torch.full((N, K + 4), 9.0, dtype=dtype, device="cuda")
        hd.logprobs_grad(x, y.cuda(), a, gl, gl, mask=mm, out=out[:, 3:3 + K])
        assert torch.equal(out[:, 3:3 + K], ref)
        assert bool((out[:, :3] == 9).all()) and bool((out[:, 3 + K:] == 9).all())


def grad_close(got, ref, t, entropy, gl, ge, scale, dtype):
    """p is within (4 |t| + 8) u of itself (t below -100 adds nothing a fp32 result shows), and
    every factor beside it carries a few roundings of its size."""
    p = torch.exp(torch.nan_to_num(t, nan=0.0, neginf=-1e4))
    tt = torch.nan_to_num(t, nan=0.0, neginf=0.0).abs().clamp(max=100)
    H = torch.nan_to_num(entropy, nan=0.0)[:, None]
    K = t.shape[1]
    dt = (4 * tt + 2 * sum_terms(K) + 4 * float(tt.max()) + 8) * P.U32   # error of t, and of p over p
    dH = dt.amax(1, keepdim=True) + float(tt.max()) * (sum_terms(K) + 8) * P.U32
    size = gl.abs()[:, None] + ge.abs()[:, None] * (tt + H)
    e = scale * (p * (size * dt + ge.abs()[:, None] * (dt + dH)) + 4 * P.U32 * (p * size)
                 + 4 * P.U32 * gl.abs()[:, None] * 1.0)
    g = got.cpu().double()
    assert torch.equal(torch.isnan(g), torch.isnan(ref))
    ok = ~torch.isnan(ref)
    e = e + P.out_round(dtype) * (ref.abs() + e) + 2.0 ** -133  # bf16's subnormals
    assert bool(((g - ref).abs()[ok] <= e[ok]).all())


@pytest.mark.parametrize("mask", ["none", "shared", "rows"])
@pytest.mark.parametrize("N,K,dtype,scale", [
    (1, 1, F32, 1.0), (4, 2, BF16, 1.0), (50, 6, F32, 0.5), (33, 26, F32, 1.0),
    (20, 100, BF16, 2.0), (7, 1000, F32, 1.0), (3, 2047, BF16, 0.7), (5, 2049, BF16, 1.0),
    (3, 4100, F32, 1.0), (2, 30001, F32, 1.0), (2, 65536, BF16, 1.0),
])
def test_gradient(N, K, dtype, scale, mask):
    hd = hd_gpu()
    announce(f"logprobs_grad {N}x{K} {dtype} mask {mask}")
    s, y, g = random_scores(N, K, dtype, seed=K + N)
    m = None
    if mask == "shared":
        m = torch.rand(K, generator=g) < 0.6
    elif mask == "rows":
        m = torch.rand(N, K, generator=g) < 0.6
        m[0] = False
    if m is not None:
        off = ~m if m.dim() == 2 else (~m)[None].expand(N, K)
        s[off] = math.nan
    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g)
    lp = hd.logprobs(s.cuda(), y.cuda(), scale=scale, mask=cuda(m))
    _, H, _, _, _, t = P.logprobs(s, y, 0, scale, m)
    for a, b in ((gl, ge), (gl, None), (None, ge), (None, None)):
        got = hd.logprobs_grad(s.cuda(), y.cuda(), lp, cuda(a), cuda(b), scale=scale, mask=cuda(m))
        ref = P.logprobs_grad(t, H, y, a, b, scale)
        zero = torch.zeros(N)
        grad_close(got, ref, t, H, (zero if a is None else a).double(),
                   (zero if b is None else b).double(), scale, dtype)
    # in place
    x = s.cuda()
    got = hd.logprobs_grad(s.cuda(), y.cuda(), lp, gl.cuda(), ge.cuda(), scale=scale, mask=cuda(m))
    here = hd.logprobs_grad(x, y.cuda(), lp, gl.cuda(), ge.cuda(), scale=scale, mask=cuda(m), out=x)
    assert here.data_ptr() == x.data_ptr() and torch.equal(here, got)


def test_gradient_rows_without_numbers():
    hd = hd_gpu()
    s = torch.zeros(4, 10)
    s[0, 3], s[1, 2], s[2] = math.nan, math.inf, -math.inf
    y = torch.zeros(4, dtype=torch.int32)
    lp = hd.logprobs(s.cuda(), y.cuda())
    g = hd.logprobs_grad(s.cuda(), y.cuda(), lp, torch.ones(4).cuda(), torch.ones(4).cuda()).cpu()
    assert bool(torch.isnan(g[:2]).all()) and bool((g[2] == 0).all())
    assert bool(torch.isfinite(g[3]).all())


def test_gradient_against_differences():
    """Central differences of the kernel's own forward pass: step h = 2^-5 leaves
    h^2 / 6 times a third derivative of at most 2 (of p(1-p)-like terms, scale 1), and
    4e-6 of rounding over 2 h."""
    hd = hd_gpu()
    N, K, h = 6, 9, 2.0 ** -5
    s, _, g = random_scores(N, K, F32, seed=5, spread=1.0)
    y = torch.randint(0, K, (N,), dtype=torch.int32, generator=g).cuda()
    m = torch.ones(N, K, dtype=torch.bool)
    m[1, 4] = False
    gl, ge = torch.rand(N, generator=g).cuda(), torch.rand(N, generator=g).cuda()

    def value(x):
        lp = hd.logprobs(x.cuda(), y, mask=m.cuda())
        return torch.where(torch.isfinite(lp.logp), gl * lp.logp, 0.0) + ge * lp.entropy

    lp = hd.logprobs(s.cuda(), y, mask=m.cuda())
    grad = hd.logprobs_grad(s.cuda(), y, lp, gl, ge, mask=m.cuda()).cpu()
    for k in range(K):
        e = torch.zeros(N, K)
        e[:, k] = h
        num = ((value(s + e) - value(s - e)) / (2 * h)).cpu()
        ok = torch.isfinite(lp.logp).cpu()
        assert bool(((num - grad[:, k]).abs()[ok] <= 2 * 2 * h * h / 6 + 4e-6 / (2 * h)).all())


def test_other_stream_workspace_and_empty():
    hd = hd_gpu()
    s, y, _ = random_scores(2, 50000, F32, seed=9)
    s, y = s.cuda(), y.cuda()
    ref = hd.logprobs(s, y, top=7)
    need = hd.logprobs_workspace_bytes(2, 50000, F32)
    assert need > 0
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = hd.logprobs(s, y, top=7, workspace=ws)
        for a, b in zip(got, ref):
            assert torch.equal(a, b)
        assert bool((ws == 0).all())  # left zeroed
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = hd.logprobs(s, y, top=7)
    st.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    with pytest.raises(hd.HDError, match="HD_ERR_WORKSPACE"):
        hd.logprobs(s, y, top=7, workspace=ws[:256])
    e = hd.logprobs(s[:0], y[:0], top=3)
    assert e.logp.shape == (0,) and e.ids.shape == (0, 3)
    assert hd.logprobs_grad(s[:0], y[:0], e).shape == (0, 50000)


def test_graph_replays():
    """A captured call gives the eager result on every replay."""
    hd = hd_gpu()
    s, y, _ = random_scores(3, 30000, F32, seed=2)
    s, y = s.cuda(), y.cuda()
    gl = torch.ones(3, device="cuda")
    ws = torch.zeros(hd.logprobs_workspace_bytes(3, 30000, F32), dtype=torch.uint8, device="cuda")

    def step():
        lp = hd.logprobs(s, y, top=5, workspace=ws)
        return lp, hd.logprobs_grad(s, y, lp, gl)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp, d = step()
    for seed in range(4):
        s.copy_(torch.randn(3, 30000, generator=torch.Generator().manual_seed(seed)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        elp, ed = step()
        torch.cuda.synchronize()
        for a, b in zip(lp, elp):
            assert torch.equal(a, b)
        assert torch.equal(d, ed)


def test_refusals():
    hd = hd_gpu()
    s = torch.zeros(4, 10, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    lp = hd.logprobs(s, y)
    for bad in (lambda: hd.logprobs(s, y[:3]), lambda: hd.logprobs(s.cpu(), y),
                lambda: hd.logprobs(s, y, mask=torch.ones(9, dtype=torch.bool, device="cuda")),
                lambda: hd.logprobs(s.t(), None), lambda: hd.logprobs(s[0], None),
                lambda: hd.logprobs_grad(s, y, lp, torch.zeros(3, device="cuda")),
                lambda: hd.logprobs_grad(s, y, lp, out=torch.zeros(4, 9, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: hd.logprobs(s.half(), y), lambda: hd.logprobs(s, y.long()),
                lambda: hd.logprobs(s, y, mask=torch.ones(10, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for kw, err in ((dict(top=33), "HD_ERR_UNSUPPORTED"), (dict(scale=0.0), "HD_ERR_ARG"),
                    (dict(scale=math.inf), "HD_ERR_ARG"), (dict(scale=math.nan), "HD_ERR_ARG")):
        with pytest.raises(hd.HDError, match=err):
            hd.logprobs(s, y, **kw)

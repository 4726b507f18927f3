"""The cross entropy of class scores, products with 8-bit weights and dropout, written out in
64 bits from their formulas, and the bounds their results are held to."""
from __future__ import annotations

import math

import numpy as np
import torch

U32 = 2.0 ** -24  # unit roundoff of fp32
PHILOX = (0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85)


def out_round(dtype) -> float:
    """Relative size of the one rounding to an output type."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else U32


# ---- cross entropy ---------------------------------------------------------------------------


def class_scores(H, C, mask):
    """Scores [N, K] in 64 bits and how far fp32 sums of D products may be from them: D + 8
    roundings of the sum of the products' sizes. Classes that take no part are -inf."""
    H, C = H.double(), C.double()
    if mask is not None:
        C = C.masked_fill(~mask.bool()[:, None], 0.0)
    s = H @ C.t()
    e = (H.shape[1] + 8) * U32 * (H.abs() @ C.abs().t())
    if mask is not None:
        s = s.masked_fill(~mask.bool(), -math.inf)
        e = e.masked_fill(~mask.bool(), 0.0)
    return s, e


def class_loss(H, C, y, scale, mask):
    """loss, stats, log probabilities t [N, K], and the bound of an error of t."""
    s, e = class_scores(H, C, mask)
    K = C.shape[0]
    m = s.max(1, keepdim=True).values                     # NaN where there is one
    m = torch.where(m == math.inf, torch.full_like(m, math.nan), m)
    empty = m == -math.inf
    z = scale * (s - torch.where(empty, torch.zeros_like(m), m))
    L = torch.log(torch.exp(z).sum(1, keepdim=True))
    L = torch.where(empty, torch.zeros_like(L), L)
    t = z - L
    asked = (y >= 0) & (y < K)
    at = torch.where(asked, y, torch.zeros_like(y)).long()[:, None]
    loss = torch.where(asked, -t.gather(1, at)[:, 0], torch.zeros_like(L[:, 0]))
    # z and L: each of two scores off by e, then s - m, its product and log2(e), each a rounding
    # of z; exp2 and log within two units, a sum of K terms in runs of 16 and a tree of runs
    live = torch.isfinite(t)
    Z = torch.where(live, z.abs(), torch.zeros_like(z))
    top = torch.where(torch.isfinite(e), e, torch.zeros_like(e)).max(1, keepdim=True).values
    d = 2 * scale * top + (6 * Z.max(1, keepdim=True).values + 2 * (K / 64 + 64)) * U32
    return loss, torch.cat((m, L), 1), t, d, top


def class_grad(H, C, y, t, g, scale, mask):
    """dS, dH and dC in 64 bits."""
    N, K = t.shape
    asked = (y >= 0) & (y < K)
    at = torch.where(asked, y, torch.zeros_like(y)).long()[:, None]
    hit = (t.gather(1, at) != -math.inf).double()
    p = torch.exp(t)
    p.scatter_add_(1, at, -hit)
    dS = p * (scale * g.double())[:, None]
    dS = torch.where(asked[:, None], dS, torch.zeros_like(dS))
    H, C = H.double(), C.double()
    H = torch.where(asked[:, None], H, torch.zeros_like(H))
    if mask is not None:
        dS = torch.where(mask.bool(), dS, torch.zeros_like(dS))
        C = torch.where(mask.bool()[:, None], C, torch.zeros_like(C))
    return dS, dS @ C, dS.t() @ H, H, C


def grad_bounds(dS, t, d, g, scale, H, C, dtype):
    """Bounds of errors of dH and dC. p is off by p (exp(d) - 1) and two units; dS by the product
    and, for bf16, its rounding; a sum of n terms by n + 8 roundings of their sizes."""
    p = torch.exp(torch.where(torch.isnan(t), torch.full_like(t, -math.inf), t))
    size = (scale * g.double().abs())[:, None]
    e = size * p * (torch.expm1(d) + 4 * U32) + 3 * U32 * (dS.abs() + size * p)
    if dtype == torch.bfloat16:
        e = e + 2.0 ** -8 * (dS.abs() + e)
    a, N, K = dS.abs() + e, dS.shape[0], dS.shape[1]
    eH = e @ C.abs() + (K + 8) * U32 * (a @ C.abs())
    eC = e.t() @ H.abs() + (N + 8) * U32 * (a.t() @ H.abs())
    return eH, eC


# ---- 8 bits ------------------------------------------------------------------------------------


def int8_codes(X):
    """(codes [N, I], scales [N]) by the header's rule, each step rounded to fp32 (numpy)."""
    x = X.float().cpu().numpy()
    top = np.abs(x).max(1) if x.shape[1] else np.zeros(x.shape[0], np.float32)
    bad = ~np.isfinite(x).all(1)
    with np.errstate(all="ignore"):
        s = (np.where(bad, np.float32(0), top) * (np.float32(1) / np.float32(127))).astype(np.float32)
        r = (np.float32(1) / s).astype(np.float32)
        r[~np.isfinite(r)] = 0
        q = np.rint(np.where(bad[:, None], np.float32(0), x) * r[:, None])
    q = np.clip(q, -127, 127).astype(np.int8)
    s[bad] = np.nan
    return torch.from_numpy(q), torch.from_numpy(s)


def int8_product(codes, row_scales, w_codes, scales, act, dtype):
    """The product as the header states it: exact sums, scales in 64 bits, one rounding to fp32
    and one to the output type."""
    v = codes.double() @ w_codes.double().t() * scales.double()
    if row_scales is not None:
        v = v * row_scales.double()[:, None]
    if act == "hardsign":
        v = torch.where(v >= 0, torch.ones_like(v), -torch.ones_like(v))
    return v.float().to(dtype)


# ---- dropout -----------------------------------------------------------------------------------


def philox(counter, key):
    """Philox 4x32, 10 rounds, on arrays of uint32 values (as uint64)."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [np.uint64(v) for v in key]
    m0, m1, w0, w1 = (np.uint64(v) for v in PHILOX)
    for _ in range(10):
        a, b = m0 * c[0], m1 * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1],
             a & low]
        k = [(k[0] + w0) & low, (k[1] + w1) & low]
    return c


def dropout_words(N, D, seed, step):
    groups = -(-D // 4)
    j, n = np.meshgrid(np.arange(groups), np.arange(N))
    w = philox((j, n, np.full_like(j, step & 0xFFFFFFFF), np.full_like(j, step >> 32)),
               (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack(w, 2).reshape(N, 4 * groups)[:, :D]


def dropout(X, p, seed, step):
    """What the call gives, bit for bit."""
    N, D = X.shape
    kept = torch.from_numpy(dropout_words(N, D, seed, step) >= np.uint64(round(p * 2 ** 32)))
    x = X.float().cpu()
    scale = torch.tensor(1.0 / (1.0 - p) if p < 1 else 0.0, dtype=torch.float64).float()
    return torch.where(kept, x * scale, torch.zeros_like(x)).to(X.dtype)

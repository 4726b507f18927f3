"""The operators behind answers and learning, written out in 64 bits from their
formulas (numpy and torch on the CPU), and the bounds their results are held to."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -24           # unit roundoff of fp32
ROWS = 64                  # rows of one group of an 8-bit checkpoint


def out_round(dtype) -> float:
    """Relative size of the one rounding to an output type."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else U32


# ---- products with 4-bit weights -----------------------------------------------------------


def random_nibble(outer, inner, group, zeros, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (outer, -(-inner // 2)), dtype=torch.uint8, generator=g)
    groups = -(-inner // group)
    scales = (torch.rand(outer, groups, generator=g) + 0.25).to(torch.bfloat16)
    z = torch.randint(0, 16, (outer, groups), dtype=torch.uint8, generator=g) if zeros else None
    return codes, scales, z


def nibble_codes(codes, inner):
    """[outer, inner] codes from packed bytes."""
    return torch.stack((codes & 15, codes >> 4), 2).flatten(1)[:, :inner].long()


def nibble_weights(codes, scales, zeros, inner, group):
    """(weights, and the sizes code + zero times scale) in 64 bits."""
    q = nibble_codes(codes, inner).double()
    of = torch.arange(inner) // group
    z = torch.full_like(q, 8.0) if zeros is None else zeros.double()[:, of]
    s = scales.double()[:, of]
    return (q - z) * s, (q + z) * s


def nibble_bound(X, size, ref, dtype):
    """A sum of I fp32 terms, and its parts q and z apart, is within (I + 8) roundings
    of the sum of their sizes; then one rounding to the output type."""
    inner = X.shape[1]
    e = (inner + 8) * U32 * (X.double().abs() @ size.t())
    return e + out_round(dtype) * (ref.abs() + e)


# ---- log probabilities ----------------------------------------------------------------------


def logprobs(s, y, top, scale, mask):
    """logp, entropy, stats, ids, top_logp in 64 bits; row by row, as the header
    states them."""
    n, k = s.shape
    logp = torch.zeros(n, dtype=torch.float64)
    entropy = torch.zeros(n, dtype=torch.float64)
    stats = torch.zeros(n, 2, dtype=torch.float64)
    ids = torch.full((n, top), -1, dtype=torch.int32)
    best = torch.full((n, top), -math.inf, dtype=torch.float64)
    t_all = torch.full((n, k), -math.inf, dtype=torch.float64)
    for r in range(n):
        x = s[r].double().clone()
        if mask is not None:
            x[~(mask if mask.dim() == 1 else mask[r]).bool()] = -math.inf
        asked = y is not None and 0 <= int(y[r]) < k
        m = float(x.max())  # NaN if there is one
        if math.isnan(m) or m == math.inf:
            logp[r] = math.nan if asked else 0.0
            entropy[r], stats[r], best[r], t_all[r] = math.nan, math.nan, math.nan, math.nan
            continue
        if m == -math.inf:
            logp[r] = -math.inf if asked else 0.0
            stats[r, 0] = -math.inf
            continue
        z = (x - m) * scale
        e = torch.exp(z)
        L = math.log(float(e.sum()))
        t = z - L
        p = torch.exp(t)
        t_all[r] = t
        stats[r, 0], stats[r, 1] = m, L
        entropy[r] = -float((p * t)[p > 0].sum())
        if asked:
            logp[r] = t[int(y[r])]
        order = torch.sort(x, descending=True, stable=True).indices[:top]
        order = order[x[order] > -math.inf]
        ids[r, :len(order)] = order.int()
        best[r, :len(order)] = t[order]
    return logp, entropy, stats, ids, best, t_all


def logprobs_grad(t, entropy, y, g_logp, g_entropy, scale):
    """dscores in 64 bits from the log probabilities t [N, K] of ``logprobs``."""
    n, k = t.shape
    p = torch.exp(t)
    d = torch.zeros_like(t)
    for r in range(n):
        asked = y is not None and 0 <= int(y[r]) < k
        g = float(g_logp[r]) if asked and g_logp is not None else 0.0
        h = float(g_entropy[r]) if g_entropy is not None else 0.0
        if bool(torch.isnan(t[r]).any()):
            d[r] = math.nan
            continue
        live = p[r] > 0
        d[r][live] = -g * p[r][live] - h * p[r][live] * (t[r][live] + entropy[r])
        if asked and t[r, int(y[r])] > -math.inf:
            d[r, int(y[r])] += g
    return d * scale


# ---- checkpoints in 8 bits ---------------------------------------------------------------------


def ckpt(H):
    """(kept values q [N, D] int, scales [groups, D]) by the header's rule, each
    step rounded to fp32."""
    n, d = H.shape
    q = torch.zeros((n, d), dtype=torch.int64)
    scales = torch.zeros((-(-n // ROWS), d), dtype=torch.float32)
    inv127 = torch.tensor(1.0, dtype=torch.float32) / torch.tensor(127.0, dtype=torch.float32)
    for b in range(scales.shape[0]):
        x = H[b * ROWS:(b + 1) * ROWS].float()
        bad = ~torch.isfinite(x).all(0)
        s = x.abs().amax(0) * inv127
        inv = torch.ones_like(s) / s
        inv[~torch.isfinite(inv)] = 0.0
        v = torch.round(torch.where(bad, torch.zeros_like(x), x) * torch.where(bad, 0.0, inv))
        q[b * ROWS:(b + 1) * ROWS] = v.clamp(-127, 127).long()
        scales[b] = torch.where(bad, torch.full_like(s, math.nan), s)
    return q, scales


def ckpt_values(q, scales):
    return q.double() * scales.double().repeat_interleave(ROWS, 0)[:q.shape[0]]

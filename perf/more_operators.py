"""The operators behind learning from encodings and answering in 8 bits, as measured cases.

* ``class_loss``: the softmax cross entropy of given classes straight from encodings (or any
  layer's outputs) and class vectors, without the scores ever being kept;
* ``class_loss_grad``: its gradient with respect to both, or to the class vectors alone;
* ``int8``: products in 8-bit integers, with a scale for each row and each output;
* ``dropout``: dropout from a counter-based generator (Philox 4x32, 10 rounds), whose mask is
  never stored: the backward pass is the same call on the gradient.

``run`` computes an operator in its plain form, from elementary operations in 32 bits, or,
where ``own`` is true, by this package's entry points. ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2}

# The largest listed case of each operator, which drawn ones stay within.
MOST_LOSS = 4096 * 4096 * 131072    # class_loss: products
MOST_GRAD = 4096 * 4096 * 65536     # class_loss_grad: products
MOST_INT8 = 8192 * 4096 * 16384     # int8: products
MOST_ROWS = 16384 * 10240           # values of an encoding matrix, or of a dropout


def listed():
    return [
        # a bulk of spoken letters' encodings (signs) under 26 class vectors
        dict(name="loss_letters", op="class_loss", n=16384, d=10240, k=26, dtype="f32",
             signs=True, mask=False),
        # a training chunk of a large vocabulary
        dict(name="loss_tokens", op="class_loss", n=4096, d=4096, k=131072, dtype="bf16",
             signs=False, mask=False),
        # a padded batch, some classes closed; no size is even
        dict(name="loss_ragged", op="class_loss", n=777, d=2047, k=32003, dtype="f32",
             signs=False, mask=True),
        # a request batch learned from at once (latency), both gradients
        dict(name="grad_batch", op="class_loss_grad", n=64, d=10240, k=100, dtype="f32",
             signs=True, mask=False, wrt="both"),
        # one refining pass of the class vectors over a bulk of spoken letters
        dict(name="grad_letters", op="class_loss_grad", n=16384, d=10240, k=26, dtype="f32",
             signs=True, mask=False, wrt="classes"),
        # a training chunk of a large vocabulary
        dict(name="grad_tokens", op="class_loss_grad", n=4096, d=4096, k=65536, dtype="bf16",
             signs=False, mask=False, wrt="both"),
        # a padded batch, some classes closed
        dict(name="grad_ragged", op="class_loss_grad", n=1999, d=1030, k=10007, dtype="bf16",
             signs=False, mask=True, wrt="both"),
        # one wearable-sensor reading encoded through 8-bit base vectors (latency)
        dict(name="sensor_int8_n1", op="int8", n=1, inner=561, outer=10240, dtype="f32"),
        # a request batch through one layer
        dict(name="requests_int8", op="int8", n=32, inner=4096, outer=14336, dtype="bf16"),
        # prompts, or a bulk of readings, through one layer
        dict(name="prompts_int8", op="int8", n=8192, inner=4096, outer=16384, dtype="bf16"),
        # a small batch's activations of an odd width (latency)
        dict(name="dropout_small", op="dropout", n=33, d=4097, dtype="bf16", p=0.1),
        # a bulk of encodings
        dict(name="dropout_bulk", op="dropout", n=16384, d=10240, dtype="f32", p=0.25),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(["class_loss", "class_loss", "class_loss_grad", "class_loss_grad", "int8",
                     "int8", "dropout"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("class_loss", "class_loss_grad"):
        # fp32 products cost several times as much
        most = (MOST_LOSS if op == "class_loss" else MOST_GRAD) // (8 if dtype == "f32" else 1)
        d = _log(rng, 64, 16384)
        k = _log(rng, 2, min(131072, MOST_GRAD // (4096 * d)))
        n = _log(rng, 1, min(65536, MOST_ROWS // d, most // (d * k), 2 ** 30 // k))
        c = dict(op=op, n=n, d=d, k=k, dtype=dtype, signs=rng.random() < 0.3,
                 mask=rng.random() < 0.4)
        if op == "class_loss_grad":
            c["wrt"] = rng.choice(["both", "both", "classes"])
        return c
    if op == "int8":
        inner = _log(rng, 32, 16384)
        outer = _log(rng, 6, min(57344, 2 ** 28 // inner))
        return dict(op=op, n=_log(rng, 1, min(8192, MOST_INT8 // (inner * outer))), inner=inner,
                    outer=outer, dtype=dtype)
    d = _log(rng, 8, 16384)
    return dict(op=op, n=_log(rng, 1, min(65536, MOST_ROWS // d)), d=d, dtype=dtype,
                p=rng.choice([0.05, 0.1, 0.25, 0.5]))


def work(case):
    op, n, es = case["op"], case["n"], ESIZE[case["dtype"]]
    if op == "int8":
        i, o = case["inner"], case["outer"]
        return {"bytes": o * i + 4 * o + es * n * (i + o), "flops": 2 * n * i * o}
    d = case["d"]
    if op == "dropout":
        return {"bytes": 2 * es * n * d, "flops": n * d}
    k = case["k"]
    read = es * (n * d + k * d) + (k if case["mask"] else 0) + 4 * n
    if op == "class_loss":
        return {"bytes": read + 12 * n, "flops": 2 * n * d * k}
    both = case["wrt"] == "both"  # the scores again, and one product for each gradient
    return {"bytes": read + 12 * n + es * (k * d + (n * d if both else 0)),
            "flops": (6 if both else 4) * n * d * k}


# ---- inputs -------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _loss_inputs(case, seed):
    """Encodings near their class's vector, class vectors, the classes asked for (some rows
    ask for none), the mask and the rows' upstream gradient. Closed classes and, in a padded
    batch, rows that ask for none hold anything."""
    g, n, d, k = _gen(seed), case["n"], case["d"], case["k"]
    dtype = DTYPES[case["dtype"]]
    C = torch.empty((k, d), dtype=dtype, device="cuda")
    for r in range(0, k, 16384):
        rows = min(16384, k - r)
        C[r:r + rows] = torch.randn(rows, d, device="cuda", generator=g).to(dtype)
    y = torch.randint(0, k, (n,), dtype=torch.int32, device="cuda", generator=g)
    H = torch.randn(n, d, device="cuda", generator=g)
    H += (2.0 / math.sqrt(d)) * C[y.long()].float()
    if case["signs"]:
        H = torch.where(H >= 0, torch.ones_like(H), -torch.ones_like(H))
    H = H.to(dtype)
    y[torch.rand(n, device="cuda", generator=g) < 0.05] = -1
    mask = None
    if case["mask"]:
        mask = torch.rand(k, device="cuda", generator=g) < 0.8
        C[:, 0:1].masked_fill_(~mask[:, None], float("nan"))
        H[:, d - 1:d].masked_fill_((y < 0)[:, None], float("nan"))
    g_loss = (torch.rand(n, device="cuda", generator=g) + 0.5) / n
    return H, C, y, mask, g_loss, 3.0 / math.sqrt(d)


def _int8_inputs(case, seed):
    """Rows X with loud features, codes [outer, inner] of a quantised normal weight and a
    scale for each output."""
    g, n, inner, outer = _gen(seed), case["n"], case["inner"], case["outer"]
    codes = torch.empty((outer, inner), dtype=torch.int8, device="cuda")
    for r in range(0, outer, 16384):
        rows = min(16384, outer - r)
        v = torch.randn(rows, inner, device="cuda", generator=g).mul_(32).round_()
        codes[r:r + rows] = v.clamp_(-127, 127).to(torch.int8)
    scales = (torch.rand(outer, device="cuda", generator=g) * 0.5 + 0.75) * 0.001
    X = torch.randn(n, inner, device="cuda", generator=g)
    X = X * (1 + 20 * (torch.rand(inner, device="cuda", generator=g) < 0.01))
    return X.to(DTYPES[case["dtype"]]), codes, scales


def _dropout_inputs(case, seed):
    X = torch.randn(case["n"], case["d"], device="cuda", generator=_gen(seed))
    # a key and the step of a training run
    return X.to(DTYPES[case["dtype"]]), (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 64, 2 ** 33 + 7


# ---- what is measured ---------------------------------------------------------------------


def prepare(case, seed):
    op = case["op"]
    if own:
        import paper_2506_09282_amd as hd
    if op == "dropout":
        X, key, step = _dropout_inputs(case, seed)
        return {"case": case, "X": X, "key": key, "step": step}
    if op == "int8":
        X, codes, scales = _int8_inputs(case, seed)
        st = {"case": case, "X": X}
        if own:  # the model, laid out once
            st["w"] = hd.byte_pack(codes, scales)
        else:
            st.update(codes=codes, scales=scales)
        return st
    H, C, y, mask, g_loss, scale = _loss_inputs(case, seed)
    st = {"case": case, "H": H, "C": C, "y": y, "mask": mask, "g": g_loss, "scale": scale}
    if op == "class_loss_grad":  # the forward pass was before
        if own:
            st["cl"] = hd.class_loss(H, C, y, scale=scale, mask=mask)
        else:
            st["stats"] = _plain_loss(H, C, y, scale, mask)["stats"]
    return st


def _plain_scores(H, C, mask):
    s = H.float() @ C.float().t()
    return s if mask is None else torch.where(mask, s, torch.full_like(s, -math.inf))


def _plain_loss(H, C, y, scale, mask):
    k = C.shape[0]
    s = _plain_scores(H, C, mask)
    m = s.amax(1, keepdim=True)
    some = m != -math.inf  # rows that hold a class at all (or NaN)
    z = (s - torch.where(some, m, torch.zeros_like(m))) * scale
    total = torch.exp(z).sum(1, keepdim=True)
    logsum = torch.where(some, torch.log(total), torch.zeros_like(total))
    asked = (y >= 0) & (y < k)
    at = torch.where(asked, y, torch.zeros_like(y)).long()[:, None]
    loss = (logsum - z.gather(1, at))[:, 0]
    return {"loss": torch.where(asked, loss, torch.zeros_like(loss)),
            "stats": torch.cat((m, logsum), 1)}


def _plain_loss_grad(H, C, y, stats, g, scale, mask, wrt):
    dtype, k = H.dtype, C.shape[0]
    m, logsum = stats[:, :1], stats[:, 1:]
    t = _plain_scores(H, C, mask)
    t = (t - torch.where(m != -math.inf, m, torch.zeros_like(m))) * scale - logsum
    asked = (y >= 0) & (y < k)
    at = torch.where(asked, y, torch.zeros_like(y)).long()[:, None]
    live = t.gather(1, at) > -math.inf
    p = torch.exp(t)
    p.scatter_add_(1, at, torch.where(live, -torch.ones_like(m), torch.zeros_like(m)))
    p = p * (g * scale)[:, None]
    # rows that ask for no class, and closed classes, have no gradient and pass none on
    p = torch.where(asked[:, None], p, torch.zeros_like(p))
    if mask is not None:
        p = torch.where(mask, p, torch.zeros_like(p))
    H = H.float()
    out = {"dC": (p.t() @ torch.where(asked[:, None], H, torch.zeros_like(H))).to(dtype)}
    if wrt == "both":
        C = C.float()
        C = C if mask is None else torch.where(mask[:, None], C, torch.zeros_like(C))
        out["dH"] = (p @ C).to(dtype)
    return out


def _plain_int8(X, codes, scales):
    x = X.float()
    s = x.abs().amax(1, keepdim=True) * (1.0 / 127.0)
    r = torch.where(s > 0, torch.reciprocal(s), torch.zeros_like(s))
    q = torch.round(x * r).clamp_(-127, 127)
    return ((q @ codes.float().t()) * s * scales).to(X.dtype)


def _plain_dropout(X, p, key, step):
    n, d = X.shape
    low = 0xFFFFFFFF
    groups = -(-d // 4)  # four values of a row share a counter {group, row, step}
    c0 = torch.arange(groups, device=X.device).expand(n, groups)
    c1 = torch.arange(n, device=X.device)[:, None].expand(n, groups)
    c2, c3 = torch.full_like(c0, step & low), torch.full_like(c0, step >> 32)
    k0, k1 = key & low, key >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64
        c0, c1, c2, c3 = (((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1,
                          a & low)
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    r = torch.stack((c0, c1, c2, c3), 2).view(n, 4 * groups)[:, :d]
    kept = r >= round(p * 2 ** 32)
    x = X.float()
    return torch.where(kept, x * (1.0 / (1.0 - p)), torch.zeros_like(x)).to(X.dtype)


def run(state):
    c = state["case"]
    op = c["op"]
    if own:
        import paper_2506_09282_amd as hd
        if op == "dropout":
            return hd.dropout(state["X"], c["p"], state["key"], step=state["step"])
        if op == "int8":
            return hd.byte_product(state["X"], state["w"])
        if op == "class_loss":
            cl = hd.class_loss(state["H"], state["C"], state["y"], scale=state["scale"],
                               mask=state["mask"])
            return {"loss": cl.loss, "stats": cl.stats}
        dH, dC = hd.class_loss_grad(state["H"], state["C"], state["y"], state["cl"], state["g"],
                                    scale=state["scale"], mask=state["mask"], wrt=c["wrt"])
        return {"dC": dC} if dH is None else {"dC": dC, "dH": dH}
    if op == "dropout":
        return _plain_dropout(state["X"], c["p"], state["key"], state["step"])
    if op == "int8":
        return _plain_int8(state["X"], state["codes"], state["scales"])
    if op == "class_loss":
        return _plain_loss(state["H"], state["C"], state["y"], state["scale"], state["mask"])
    return _plain_loss_grad(state["H"], state["C"], state["y"], state["stats"], state["g"],
                            state["scale"], state["mask"], c["wrt"])


# ---- the definition in 64 bits ------------------------------------------------------------


def _mul32(a, b):
    """High and low half of a 32 x 32 bit product, from 16-bit pieces of b."""
    lo, hi = a * (b % 65536), a * (b // 65536)
    both = lo + (hi % 65536) * 65536
    return hi // 65536 + both // 2 ** 32, both % 2 ** 32


def exact(case, seed):
    op, n = case["op"], case["n"]
    if op == "dropout":
        X, key, step = _dropout_inputs(case, seed)
        p, parts = case["p"], []
        column = torch.arange(case["d"], device="cuda")
        for r in range(0, n, max(1, 2 ** 24 // case["d"])):
            x = X[r:r + max(1, 2 ** 24 // case["d"])].double()
            row = torch.arange(r, r + x.shape[0], device="cuda")[:, None]
            w = [(column // 4).expand(x.shape), row.expand(x.shape),
                 torch.full(x.shape, step % 2 ** 32, device="cuda"),
                 torch.full(x.shape, step // 2 ** 32, device="cuda")]
            ks = [key % 2 ** 32, key // 2 ** 32]
            for _ in range(10):
                (h0, l0), (h1, l1) = _mul32(w[0], 0xD2511F53), _mul32(w[2], 0xCD9E8D57)
                w = [h1 ^ w[1] ^ ks[0], l1, h0 ^ w[3] ^ ks[1], l0]
                ks = [(ks[0] + 0x9E3779B9) % 2 ** 32, (ks[1] + 0xBB67AE85) % 2 ** 32]
            place = column % 4
            u = torch.where(place < 2, torch.where(place == 0, w[0], w[1]),
                            torch.where(place == 2, w[2], w[3]))
            parts.append(x / (1 - p) * (u >= round(p * 2 ** 32)))
        return torch.cat(parts)
    if op == "int8":
        X, codes, scales = _int8_inputs(case, seed)
        # the rows' codes are what the rule's fp32 steps say; what follows is exact
        x = X.float()
        step = x.abs().max(1).values * torch.tensor(1 / 127, dtype=torch.float32, device="cuda")
        q = torch.round(x * (torch.ones_like(step) / step)[:, None]).double()
        parts = [q @ codes[r:r + 2048].double().t() for r in range(0, case["outer"], 2048)]
        return torch.cat(parts, 1) * step.double()[:, None] * scales.double()
    H, C, y, mask, g, scale = _loss_inputs(case, seed)
    k, d = case["k"], case["d"]
    open_ = torch.ones(k, dtype=torch.bool, device="cuda") if mask is None else mask
    C = C.double()
    parts, dC = [], torch.zeros((k, d), dtype=torch.float64, device="cuda")
    clean = C.masked_fill(~open_[:, None], 0.0)
    rows = max(1, 2 ** 28 // k)
    for r in range(0, n, rows):
        h, yr = H[r:r + rows].double(), y[r:r + rows].long()
        s = (h @ clean.t()).masked_fill(~open_, -math.inf)
        asked, at = yr >= 0, yr.clamp(min=0)[:, None]
        top = s.max(1, keepdim=True).values
        empty = top == -math.inf
        lse = torch.logsumexp(scale * s, 1, keepdim=True)
        logp = (scale * s - lse).masked_fill(empty, -math.inf)
        if op == "class_loss":
            parts.append(((-logp.gather(1, at)[:, 0]).masked_fill(~asked, 0.0),
                          torch.cat((top, (lse - scale * top).masked_fill(empty, 0.0)), 1)))
            continue
        one = torch.zeros_like(logp).scatter_(1, at, 1.0) * open_
        ds = ((logp.exp() - one) * (scale * g[r:r + rows].double())[:, None])
        ds = ds.masked_fill(~asked[:, None], 0.0)
        dC += ds.t() @ h.masked_fill(~asked[:, None], 0.0)
        if case["wrt"] == "both":
            parts.append((ds @ clean,))
    parts = [torch.cat(v) for v in zip(*parts)]
    if op == "class_loss":
        return {"loss": parts[0], "stats": parts[1]}
    return {"dC": dC, "dH": parts[0]} if parts else {"dC": dC}

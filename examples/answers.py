"""Learning from kept encodings and answering from a model in 4 bits.

    python examples/answers.py [--train 20000] [--steps 20]

1. Single-pass training gives the class hypervectors (bundling).
2. The encodings are kept once, in 8 bits; each refining step scores them, takes the log
   probabilities of the labels and their gradient, and reads the class vectors'
   gradient from the checkpoint.
3. Base and class vectors are laid out in 4 bits with group scales, and single readings are
   answered from them: label, its log probability, the entropy, the next best.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_09282_amd as hd  # noqa: E402


def readings(n: int, F: int, K: int, seed: int, device="cuda"):
    """Synthetic readings: class centres (the same for every seed) in strong noise."""
    centres = torch.randn(K, F, generator=torch.Generator().manual_seed(17))
    g = torch.Generator().manual_seed(seed)
    y = torch.randint(0, K, (n,), dtype=torch.int32, generator=g)
    X = centres[y.long()] + 6.0 * torch.randn(n, F, generator=g)
    return X.to(device), y.to(device)


def bundled(X, B, y, K: int):
    """Class hypervectors by single-pass training, [K, D] in -1 and +1."""
    return hd.class_hardsign(hd.bundle_classes_packed(X, hd.pack_model(B), y, K))


def refine(C, H, y, steps: int, rate: float, scale: float):
    """Gradient steps on the mean log probability of the labels, from encodings kept in
    8 bits. Returns the refined C and the loss before each step."""
    kept = hd.ckpt_store(H)
    C = C.clone()
    N, losses = H.shape[0], []
    g = torch.full((N,), -1.0 / N, dtype=torch.float32, device=H.device)
    for _ in range(steps):
        _, S = hd.similarity(hd.ckpt_load(kept), C, return_scores=True)
        lp = hd.logprobs(S, y, scale=scale)
        losses.append(-lp.logp.mean())
        dS = hd.logprobs_grad(S, y, lp, g, scale=scale, out=S)
        C -= rate * hd.ckpt_class_grad(dS, kept)
    return C, [float(v) for v in losses]


class FourBitModel:
    """Base and class hypervectors in 4 bits; answers with log probabilities."""

    def __init__(self, B, C, group: int = 64):
        self.B = hd.nibble_quantize(B, group=group, inner_rows=True)
        self.C = hd.nibble_quantize(C, group=group)

    def scores(self, X):
        H = hd.nibble_product(X, self.B, act="hardsign", dtype=torch.bfloat16)
        return hd.nibble_product(H, self.C, dtype=torch.float32)

    def answer(self, X, scale: float, top: int = 3):
        return hd.logprobs(self.scores(X), top=top, scale=scale)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--train", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    F, D, K = 561, 10240, 6
    B = torch.randn(F, D, generator=torch.Generator().manual_seed(1)).cuda()
    X, y = readings(a.train, F, K, seed=2)
    Xt, yt = readings(2000, F, K, seed=3)

    C = bundled(X, B, y, K)
    scale = 1.0 / D ** 0.5
    C2, losses = refine(C, hd.encode(X, B), y, a.steps, rate=200.0, scale=scale)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    for name, c in (("bundled", C), ("refined", C2)):
        full = float((hd.infer(Xt, B, c) == yt).float().mean())
        four = FourBitModel(B, c)
        lp = four.answer(Xt, scale)
        print(f"{name}: fp32 {full:.4f}, 4 bits {float((lp.ids[:, 0] == yt).float().mean()):.4f}, "
              f"mean entropy {float(lp.entropy.mean()):.3f}")
    one = four.answer(Xt[:1], scale)
    print("first reading:", [(int(k), round(float(p), 3))
                             for k, p in zip(one.ids[0], one.top_logp[0].exp())],
          "label", int(yt[0]))


if __name__ == "__main__":
    main()

"""A compressed output head from end to end: 4-bit weights, the rank-k compensation of what they leave, its fit to the
uncompressed head by distillation, and tokens drawn from its logits.

    python examples/compressed_head.py [--vocab 8192] [--hidden 1024] [--rank 33]

Weights and activations are synthetic: a decaying spectrum as trained projections have, normal activations."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_12969_amd import lrc  # noqa: E402


def synthetic_head(vocab, hidden, g):
    """vocab x hidden weights whose singular values fall like 1 / sqrt(i)."""
    left = torch.randn(vocab, hidden, generator=g, device="cuda")
    left *= torch.arange(1, hidden + 1, device="cuda") ** -0.5
    return left @ torch.randn(hidden, hidden, generator=g, device="cuda") / hidden ** 0.5


def compress(W, rank, group, g):
    """Codes and scales of W, and the rank-k compensation of W - W4 in binary32."""
    codes, scales, values = lrc.q4_quantize(W, group=group, values=True)
    omega = torch.randn(min(rank + 16, W.shape[1]), W.shape[1], generator=g, device="cuda", dtype=torch.float64)
    U, s, V = lrc.rsvd((W - values).double(), omega, rank, power_iters=1)
    factors = tuple(f.float() for f in (U, s, V))
    return codes, scales, values, factors


def fit(codes, scales, factors, X, ids, top, lse, group, steps=20, rate=0.5):
    """Gradient steps on U, the compensation's left factor: the loss before and after, and the factors."""
    U, s, V = factors
    U = U.clone()
    weight = torch.full((X.shape[0],), 1.0 / X.shape[0], device="cuda")
    T = (X @ V) * s
    rate = rate / float((T * T).sum(0).max()) * X.shape[0]
    first = last = None
    for step in range(steps + 1):
        logits = lrc.q4_apply(codes, scales, X, group=group, factors=(U, s, V))
        if step == steps:
            last, _ = lrc.distill_forward(logits, ids, top, teacher_lse=lse, weight=weight)
            break
        loss, grad = lrc.distill(logits, ids, top, teacher_lse=lse, weight=weight, grad=logits)
        first = loss if first is None else first
        U -= rate * (grad.t().contiguous() @ T)
    return float(first.sum()), float(last.sum()), (U, s, V)


def run(vocab=8192, hidden=1024, rank=33, group=128, tokens=512, top=64, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = synthetic_head(vocab, hidden, g)
    codes, scales, values, factors = compress(W, rank, group, g)
    U, s, V = factors
    plain = float((W - values).norm() / W.norm())
    compensated = float((W - values - (U * s) @ V.t()).norm() / W.norm())

    X = torch.randn(tokens, hidden, generator=g, device="cuda")
    teacher = X @ W.t()
    top_logits, ids = teacher.topk(top, dim=1)
    lse = teacher.logsumexp(dim=1)
    before, after, factors = fit(codes, scales, factors, X, ids, top_logits, lse, group)

    # what is stored and served: binary16 factors and activations
    stored = tuple(f.half() for f in factors)
    x = torch.randn(4, hidden, generator=g, device="cuda").half()
    logits = lrc.q4_apply(codes, scales, x, group=group, factors=stored, out_dtype=torch.float32)
    drawn = lrc.sample(logits, torch.rand(4, generator=g, device="cuda"),
                       temperature=torch.full((4,), 0.8, device="cuda"),
                       top_k=torch.full((4,), 50, dtype=torch.int64, device="cuda"),
                       top_p=torch.full((4,), 0.95, device="cuda"))
    dense = 2 * vocab * hidden
    held = lrc.q4_storage_bytes(vocab, hidden, group, "fp16") + 2 * rank * (vocab + hidden + 1)
    return dict(error_4bit=plain, error_compensated=compensated, loss_before=before, loss_after=after,
                bytes_of_16_bit=held / dense, tokens=drawn.tolist())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=8192)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--rank", type=int, default=33)
    a = ap.parse_args()
    for name, value in run(a.vocab, a.hidden, a.rank).items():
        print(f"{name}: {value if isinstance(value, list) else format(value, '.4g')}")

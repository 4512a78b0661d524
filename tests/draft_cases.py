"""Seeded trees and inputs of the speculative decoding tests, and their error bounds.

Bounds are derived, in units of the roundings that happen: bf16 2^-8, f16 2^-11 and fp32 2^-24
relative to the value rounded.
"""
import random

import numpy as np
import torch

BF16, F16, F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


def tree(kind, n, seed=0):
    rng = random.Random(f"{kind} {n} {seed}")
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "roots":          # no common root
        return [-1] * n
    if kind == "forest":
        return [-1 if i == 0 or rng.random() < 0.2 else rng.randint(0, i - 1) for i in range(n)]
    return [-1] + [rng.randint(max(0, i - 6), i - 1) if rng.random() < 0.6 else rng.randint(0, i - 1) for i in range(1, n)]


def bf16(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def worst(got, want, bound):
    """Largest error in units of its bound (at most 1 passes); not finite where the other is finite: infinite."""
    got, want = f64(got) if isinstance(got, torch.Tensor) else got, np.asarray(want)
    bound = np.broadcast_to(bound, want.shape)
    same = np.isnan(got) == np.isnan(want)
    if not same.all():
        return float("inf")
    fine = ~np.isnan(want)
    d = np.abs(got - want)[fine]
    return float((d / (bound[fine] + 1e-300)).max(initial=0.0))


def delta_inputs(rng, n, Hk, Hv, d):
    k = rng.standard_normal((n, Hk, d))
    k = torch.from_numpy(k / np.linalg.norm(k, axis=-1, keepdims=True)).to(torch.bfloat16)
    beta = torch.from_numpy(1 / (1 + np.exp(-rng.standard_normal((n, Hv))))).float()
    g = torch.from_numpy(np.exp(-np.log1p(np.exp(rng.standard_normal((n, Hv)) - 4)))).float()
    return dict(state=torch.from_numpy(0.1 * rng.standard_normal((Hv, d, d))).float(), q=bf16(rng, n, Hk, d), k=k,
                v=bf16(rng, n, Hv, d), beta=beta, g=g)


def rows_of(rng, n, V, peak=2.0):
    """n fp32 probability rows."""
    z = rng.standard_normal((n, V)) * peak
    p = np.exp(z - z.max(-1, keepdims=True))
    return (p / p.sum(-1, keepdims=True)).astype(np.float32)


def drafted(rng, parents, proposal, distinct=False):
    """Tokens of the nodes: drawn from their parents' rows, or the likeliest ones in order."""
    tok = np.zeros(len(parents), np.int32)
    for i, p in enumerate(parents):
        if p < 0:
            continue
        row = proposal[p].astype(np.float64)
        if distinct:
            rank = sum(parents[j] == p for j in range(i))
            tok[i] = np.argsort(-row, kind="stable")[min(rank, len(row) - 1)]
        else:
            tok[i] = rng.choice(len(row), p=row / row.sum())
    return tok

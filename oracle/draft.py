"""Speculative decoding of a hybrid context in float64 (test infrastructure only).

A drafter proposes a tree of tokens: node i continues node parents[i] < i, or the context
itself (-1). These are the definitions, node by node along each path: norms of queries and
keys with the rotation, attention over the cache and the ancestors, the recurrent layers from
the carried state, and recursive rejection sampling against the target's probabilities.
Inputs are float64 arrays (bf16 values widened by the caller).
"""
import numpy as np


def line(parents, i):
    """Ancestors of node i and itself, from the root on."""
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i]
    return out[::-1]


def depths(parents):
    return np.array([len(line(parents, i)) - 1 for i in range(len(parents))], dtype=np.int64)


def qk_norm_rope(x, pos, rotary, theta, kind="none", eps=0.0, weight=None, offset=0.0):
    """x [T][H][D], pos [T]."""
    x = np.array(x, dtype=np.float64)
    if kind == "rms":
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * (np.asarray(weight, np.float64) + offset)
    elif kind == "l2":
        x = x / np.sqrt((x * x).sum(-1, keepdims=True) + eps)
    half = rotary // 2
    ang = np.asarray(pos, np.float64)[:, None] * theta ** (-2.0 * np.arange(half) / max(1, rotary))
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = x.copy()
    y[..., :half] = x[..., :half] * c - x[..., half:rotary] * s
    y[..., half:rotary] = x[..., half:rotary] * c + x[..., :half] * s
    return y


def draft_attention(q, k, v, parents, scale):
    """q [n][Hq][D]; k, v [len + n][Hkv][D], the nodes' rows last. Returns (out [n][Hq][D], the same with |v|,
    the largest sum of |q k| scale of a row [n][Hq])."""
    n, Hq, _ = q.shape
    rows, G = k.shape[0] - n, Hq // k.shape[1]
    out, mag = np.zeros_like(q), np.zeros_like(q)
    most = np.zeros((n, Hq))
    for i in range(n):
        see = np.concatenate([np.arange(rows), rows + np.array(line(parents, i), dtype=np.int64)])
        for h in range(Hq):
            K, V = k[see, h // G], v[see, h // G]
            z = scale * (K @ q[i, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ V, p @ np.abs(V)
            most[i, h] = scale * (np.abs(K) @ np.abs(q[i, h])).max()
    return out, mag, most


def draft_short_conv(state, x, w, parents, silu):
    """state [W-1][C], x [n][C], w [C][W]. Returns (y [n][C], sum of |w x|)."""
    W = w.shape[1]
    y, mag = np.zeros(x.shape), np.zeros(x.shape)
    for i in range(x.shape[0]):
        rows = np.concatenate([state, x[line(parents, i)]])[-W:]
        y[i], mag[i] = (rows.T * w).sum(1), (np.abs(rows).T * np.abs(w)).sum(1)
    return (y / (1 + np.exp(-y)) if silu else y), mag


def delta_step(S, k, v, beta, g, sign=-1.0):
    """One token: S <- g S (I - beta k k^T) + beta v k^T; S [Hv][dv][dk], k [Hk][dk], v [Hv][dv]. sign 1 with
    magnitudes for everything bounds every intermediate."""
    k = np.repeat(k, S.shape[0] // k.shape[0], axis=0)
    b, g = beta[:, None, None], g[:, None, None]
    Sk = np.einsum("hij,hj->hi", S, k)
    return g * (S + sign * b * Sk[:, :, None] * k[:, None, :]) + b * v[:, :, None] * k[:, None, :]


def draft_delta_rule(S0, q, k, v, beta, g, parents, scale, sign=-1.0):
    states, out = [], np.zeros(v.shape)
    for i, p in enumerate(parents):
        S = delta_step(states[p] if p >= 0 else S0, k[i], v[i], beta[i], g[i], sign)
        states.append(S)
        out[i] = scale * np.einsum("hij,hj->hi", S, np.repeat(q[i], S.shape[0] // q.shape[1], axis=0))
    return out


def draft_verify(parents, tokens, target, u, proposal=None):
    """Returns (accepted path, next token)."""
    n, V = target.shape
    m, path = 0, [0]
    while True:
        p = target[m].copy()
        whole, left = 1.0, p          # `left` is `whole` times a distribution
        took = -1
        for c in [c for c in range(m + 1, n) if parents[c] == m]:
            x = int(tokens[c])
            inside = 0 <= x < V
            qx = 1.0 if proposal is None else (proposal[m, x] if inside else 1.0)
            if inside and u[c] * qx < left[x] / whole:
                took = c
                break
            if proposal is None:
                left = left.copy()
                if inside:
                    left[x] = 0.0
            else:
                left = np.maximum(left / whole - proposal[m], 0.0)
            whole = left.sum()
            if not whole > 0:
                whole = 1.0           # nothing is left: no later child passes either
                left = np.zeros(V)
        if took < 0:
            break
        m = took
        path.append(m)
    left = np.maximum(left, 0.0)
    if not left.sum() > 0:
        left = np.maximum(target[m], 0.0)
    total = left.sum()
    if not (total > 0 and np.isfinite(total)):
        return path, -1
    cdf = np.cumsum(left)
    over = np.nonzero(cdf > u[0] * cdf[-1])[0]
    return path, int(over[0]) if len(over) else int(np.nonzero(left)[0][-1])

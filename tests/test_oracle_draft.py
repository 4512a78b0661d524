"""The speculative decoding definitions (oracle.draft) against the rest of the oracle and
against what they stand for."""
import itertools

import numpy as np

import oracle
from oracle import draft as O
from draft_cases import drafted, f64, rows_of, delta_inputs, tree


def test_a_chain_is_the_ordinary_tail():
    rng = np.random.default_rng(0)
    n, rows, hq, hkv, D = 6, 9, 4, 2, 8
    chain = tree("chain", n)
    k, v, q = rng.standard_normal((rows + n, hkv, D)), rng.standard_normal((rows + n, hkv, D)), rng.standard_normal((n, hq, D))
    got, _, _ = O.draft_attention(q, k, v, chain, 0.3)
    assert np.allclose(got, oracle.causal_gqa_attention(q, k, v, rows, 0.3), atol=1e-12)
    c = {x: f64(t) for x, t in delta_inputs(rng, n, 1, 2, 4).items()}
    want, _ = oracle.gated_delta_tokens(c["state"], c["q"], c["k"], c["v"], c["beta"], c["g"], 0.5)
    assert np.allclose(O.draft_delta_rule(c["state"], c["q"], c["k"], c["v"], c["beta"], c["g"], chain, 0.5), want, atol=1e-13)
    assert list(O.depths(chain)) == list(range(n))


def test_every_path_of_a_tree_is_a_chain():
    rng = np.random.default_rng(1)
    parents = tree("forest", 14)
    n, W = len(parents), 4
    c = {x: f64(t) for x, t in delta_inputs(rng, n, 1, 2, 4).items()}
    x, state, w = rng.standard_normal((n, 5)), rng.standard_normal((W - 1, 5)), rng.standard_normal((5, W))
    o = O.draft_delta_rule(c["state"], c["q"], c["k"], c["v"], c["beta"], c["g"], parents, 1.0)
    y, _ = O.draft_short_conv(state, x, w, parents, True)
    for i in range(n):
        p = O.line(parents, i)
        want, _ = oracle.gated_delta_tokens(c["state"], c["q"][p], c["k"][p], c["v"][p], c["beta"][p], c["g"][p], 1.0)
        assert np.allclose(o[i], want[-1], atol=1e-13)
        rows = np.concatenate([state, x[p]])[-W:]
        z = (rows.T * w).sum(1)
        assert np.allclose(y[i], z / (1 + np.exp(-z)), atol=1e-13)


def test_the_norms():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 2, 8))
    y = O.qk_norm_rope(x, np.zeros(3), 8, 100.0, "rms", 0.0, np.full(8, 2.0), 1.0)
    assert np.allclose((y * y).mean(-1), 9.0)
    y = O.qk_norm_rope(x, np.array([0, 5, 77]), 4, 100.0, "l2")
    assert np.allclose((y * y).sum(-1), 1.0) and np.allclose(y[0], x[0] / np.linalg.norm(x[0], axis=-1, keepdims=True))


def _law(parents, target, proposal, V):
    """Distribution of (the accepted tokens, the next one): exact over tokens drawn from the proposals, by
    integrating each test's uniform number (its outcome has probability min(1, p'(x) / q(x)))."""
    law = {}

    def go(m, tok, prob, said):
        kids = [c for c in range(len(parents)) if parents[c] == m]
        left, weight = target[m].copy(), prob
        for c in kids:
            a = min(1.0, left[tok[c]] / proposal[m, tok[c]])
            if a > 0:
                go(c, tok, weight * a, said + (tok[c],))
            weight *= 1 - a
            if weight < 1e-15:
                return
            left = np.maximum(left - proposal[m], 0)
            left /= left.sum()
        for t in range(V):
            key = said + (t,)
            law[key] = law.get(key, 0.0) + weight * left[t]

    n = len(parents)
    for tok in itertools.product(range(V), repeat=n - 1):
        tok = (0,) + tok
        prob = np.prod([proposal[parents[i], tok[i]] for i in range(1, n)])
        go(0, tok, prob, ())
    return law


def test_the_first_token_follows_the_target():
    """Whatever the drafter proposes, the token behind the root has the target's distribution."""
    rng = np.random.default_rng(3)
    V = 3
    for parents in ([-1, 0], [-1, 0, 0], [-1, 0, 0, 0], [-1, 0, 0, 1]):
        target = rows_of(rng, len(parents), V).astype(np.float64)
        proposal = rows_of(rng, len(parents), V).astype(np.float64)
        target /= target.sum(-1, keepdims=True)
        proposal /= proposal.sum(-1, keepdims=True)
        first = np.zeros(V)
        for said, p in _law(parents, target, proposal, V).items():
            first[said[0]] += p
        assert np.allclose(first, target[0], atol=1e-12)


def test_verification_by_its_outcomes():
    """Frequencies over many random numbers agree with the law (five standard errors)."""
    rng = np.random.default_rng(4)
    parents, V, N = [-1, 0, 0, 1], 4, 20000
    target, proposal = rows_of(rng, 4, V).astype(np.float64), rows_of(rng, 4, V).astype(np.float64)
    count = np.zeros(V)
    for _ in range(N):
        tok = np.array([0] + [rng.choice(V, p=proposal[p] / proposal[p].sum()) for p in parents[1:]])
        path, nxt = O.draft_verify(parents, tok, target, rng.random(4), proposal)
        count[tok[path[1]] if len(path) > 1 else nxt] += 1
    p = target[0] / target[0].sum()
    assert (np.abs(count / N - p) <= 5 * np.sqrt(p * (1 - p) / N)).all()
    # chosen tokens: a child is accepted with the target's probability of its token
    tok = drafted(rng, parents, proposal, distinct=True)
    count = np.zeros(V)
    for _ in range(N):
        path, nxt = O.draft_verify(parents, tok, target, rng.random(4))
        count[tok[path[1]] if len(path) > 1 else nxt] += 1
    assert (np.abs(count / N - p) <= 5 * np.sqrt(p * (1 - p) / N)).all()


def test_closed_form_of_repeated_rejection():
    """max(.. - q, 0) normalised r times is max(p - b q, 0) normalised, b growing by its sum each time."""
    rng = np.random.default_rng(5)
    p, q = (x / x.sum() for x in rows_of(rng, 2, 50).astype(np.float64))
    left, b, F = p, 0.0, 1.0
    for _ in range(5):
        left = np.maximum(left - q, 0)
        left /= left.sum()
        b += F
        F = np.maximum(p - b * q, 0).sum()
        assert np.allclose(np.maximum(p - b * q, 0) / F, left, atol=1e-12)

"""Speculative decoding on the GPU against the float64 definitions (oracle.draft)."""
import numpy as np
import pytest
import torch

import paper_2609_18935_amd as tu
from oracle import draft as O
from draft_cases import BF16, F16, F32, bf16, delta_inputs, drafted, f64, rows_of, tree, worst

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 1.0e7


def dev(t):
    return t.to(DEV)


def _ctx(rows, n, cursor=None, spare=0):
    ctx = tu.Context(rows + n + spare, device=DEV)
    cursor = rows if cursor is None else cursor
    ctx.set_metadata([(cursor - rows, cursor)] if rows else [], cursor)
    return ctx


# ----------------------------------------------------------------------------- norms and rotation

def _norm_bound(x, want, kind, weight, offset, D):
    """One rounding to bf16 of a value whose fp32 error is a few rounding steps of the two normed components."""
    y = np.abs(x) if kind == "none" else np.abs(O.qk_norm_rope(x, np.zeros(x.shape[0]), 0, 1.0, kind, 1e-6, weight, offset))
    mag = np.abs(y).max(-1, keepdims=True)
    return BF16 * np.abs(want) + (D / 8 + 24) * F32 * 2 * mag + 2.0 ** -126


@pytest.mark.parametrize("hq,hkv,D,rotary", [(16, 2, 256, 256), (32, 8, 128, 64), (16, 4, 64, 64), (8, 8, 128, 20),
                                             (4, 1, 64, 0), (5, 5, 256, 2), (16, 2, 256, 64), (3, 1, 64, 62)])
@pytest.mark.parametrize("kind,T", [("rms", 1), ("rms", 67), ("l2", 5), ("none", 33)])
def test_norm_rope(hq, hkv, D, rotary, kind, T):
    rng = np.random.default_rng([hq, D, rotary, T])
    qkv = bf16(rng, T, hq + 2 * hkv, D, scale=3.0)
    x = dev(qkv)
    q, k = x[:, :hq], x[:, hq:hq + hkv]                 # rows of one projection's output
    wq, wk = bf16(rng, D), bf16(rng, D)
    offset = 1.0 if T == 67 else 0.0
    norm = tu.QkNorm(kind, 1e-6, dev(wq), dev(wk), weight_offset=offset)
    p = tu.attn_params(hq, hkv, D, rotary, THETA)
    qo = torch.zeros(T, hq, D, dtype=torch.bfloat16, device=DEV)
    ko = torch.zeros(T, hkv, D, dtype=torch.bfloat16, device=DEV)
    pos = np.arange(T) + 479547
    tu.qk_norm_rope(p, q, k, qo, ko, norm=norm, first_pos=479547)
    for got, src, w in ((qo, qkv[:, :hq], wq), (ko, qkv[:, hq:hq + hkv], wk)):
        w = f64(w) if kind == "rms" else None
        want = O.qk_norm_rope(f64(src), pos, rotary, THETA, kind, np.float64(np.float32(1e-6)), w, offset)
        assert worst(got, want, _norm_bound(f64(src), want, kind, w, offset, D)) <= 1
    # device positions, in place, queries alone
    some = torch.randint(0, 2 ** 31 - 1, (T,), dtype=torch.int32)
    qi = dev(qkv[:, :hq].contiguous())
    tu.qk_norm_rope(p, qi, None, qi, None, norm=norm, positions=dev(some))
    w = f64(wq) if kind == "rms" else None
    want = O.qk_norm_rope(f64(qkv[:, :hq]), f64(some), rotary, THETA, kind, np.float64(np.float32(1e-6)), w, offset)
    assert worst(qi, want, _norm_bound(f64(qkv[:, :hq]), want, kind, w, offset, D) +
                 2.0 ** 31 * 2.0 ** -50 * np.abs(want).max()) <= 1
    assert torch.equal(x, dev(qkv))


def test_norm_of_zero_and_non_finite_rows():
    p = tu.attn_params(2, 1, 64, 64, THETA)
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    q[1, 0, 5] = float("nan")
    q[2, 1, 7] = float("inf")
    out = torch.zeros_like(q)
    tu.qk_norm_rope(p, q, None, out, None, norm=tu.QkNorm("rms", 1e-6))
    assert (out[0] == 0).all() and out[1, 0].isnan().all() and (out[1, 1] == 0).all()
    assert out[2, 1].isnan().any() and (out[2, 0] == 0).all()


@pytest.mark.parametrize("hq,hkv,D,rotary,rows,n", [(16, 2, 256, 256, 37, 1), (32, 8, 128, 64, 0, 128), (16, 4, 64, 20, 5, 19)])
def test_append(hq, hkv, D, rotary, rows, n):
    rng = np.random.default_rng([hq, n])
    parents = tree("forest", n)
    qkv = bf16(rng, n, hq + 2 * hkv, D)
    x = dev(qkv)
    ctx = _ctx(rows, n, 300000, spare=2)
    kc, vc = dev(bf16(rng, 2, rows + n + 2, hkv, D))
    before = kc.clone(), vc.clone(), ctx.pos.clone()
    q_hat = torch.zeros(n, hq, D, dtype=torch.bfloat16, device=DEV)
    w = bf16(rng, D)
    tu.draft_append(ctx, kc, vc, tu.attn_params(hq, hkv, D, rotary, THETA), tu.Draft(parents), x[:, :hq],
                    x[:, hq:hq + hkv], x[:, hq + hkv:], q_hat, norm=tu.QkNorm("rms", 1e-6, None, dev(w)))
    pos = 300000 + O.depths(parents)
    for got, src, wt in ((q_hat, qkv[:, :hq], None), (kc[rows:rows + n], qkv[:, hq:hq + hkv], f64(w))):
        want = O.qk_norm_rope(f64(src), pos, rotary, THETA, "rms", np.float64(np.float32(1e-6)), wt)
        assert worst(got, want, _norm_bound(f64(src), want, "rms", wt, 0.0, D)) <= 1
    assert torch.equal(vc[rows:rows + n], x[:, hq + hkv:])
    for now, then in ((kc, before[0]), (vc, before[1])):      # other rows, behind the last node too
        assert torch.equal(now[:rows], then[:rows]) and torch.equal(now[rows + n:], then[rows + n:])
    assert torch.equal(ctx.pos, before[2]) and ctx.len == rows and ctx.next_pos == 300000


# ----------------------------------------------------------------------------- attention

def _attn(hq, hkv, D, rows, parents, seed=0, splits=0, scale=None, kv=None, spare=3):
    rng = np.random.default_rng([hq, hkv, D, rows, len(parents), seed])
    n = len(parents)
    k, v = bf16(rng, 2, rows + n + spare, hkv, D) if kv is None else kv
    q = bf16(rng, n, hq, D)
    p = tu.attn_params(hq, hkv, D, softmax_scale=scale, kv_splits=splits)
    ctx = _ctx(rows, n, spare=spare)
    out = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = tu.draft_attention(ctx, dev(k), dev(v), p, tu.Draft(parents), dev(q), out)
    want, mag, most = O.draft_attention(f64(q), f64(k)[:rows + n], f64(v)[:rows + n], parents, D ** -0.5 if scale is None else scale)
    # the output's rounding; P and the partial outputs in f16 (P below 2^-14 of the reference in its subnormals);
    # the scores' fp32 sums and the exponential, in numerator and denominator
    bound = BF16 * np.abs(want) + (2 * F16 + 2 * ((D + 8) * F32 * most[..., None] + 16 * F32)) * mag + \
        2.0 ** -24 * (rows + n) * np.abs(f64(v)[:rows + n]).max() * 2.0 ** -8
    return out, want, bound, ws


@pytest.mark.parametrize("hq,hkv,D", [(16, 2, 256), (32, 8, 128), (16, 4, 64), (4, 4, 128), (3, 1, 64), (40, 1, 256)])
@pytest.mark.parametrize("rows,kind,n", [(0, "chain", 1), (1, "star", 2), (31, "forest", 33), (203, "tree", 17),
                                         (517, "roots", 64), (1000, "tree", 128)])
def test_attention(hq, hkv, D, rows, kind, n):
    out, want, bound, ws = _attn(hq, hkv, D, rows, tree(kind, n))
    assert worst(out, want, bound) <= 1
    assert tu.workspace_faults(ws) == 0


@pytest.mark.parametrize("splits", [1, 2, 7, 64])
def test_attention_splits(splits):
    out, want, bound, _ = _attn(16, 2, 256, 301, tree("tree", 40), splits=splits)
    assert worst(out, want, bound) <= 1


def test_attention_large_scores_and_far_apart_maxima():
    # scores up to several hundred: the running maximum moves, most keys vanish
    out, want, bound, _ = _attn(16, 2, 128, 700, tree("tree", 30), scale=4.0)
    assert worst(out, want, bound) <= 1


def test_attention_ignores_rows_behind_the_draft_and_hidden_nodes():
    rng = np.random.default_rng(5)
    rows, n, hkv, D = 50, 40, 2, 256
    parents = tree("star", n)
    kv = bf16(rng, 2, rows + n + 3, hkv, D)
    kv[:, rows + n:] = float("nan")            # rows that hold nothing
    kv[0, rows + 7] = float("nan")             # a node's own key: hidden from its siblings
    out, want, bound, _ = _attn(16, hkv, D, rows, parents, kv=kv)
    others = [i for i in range(n) if i != 7]
    assert worst(out[others], want[others], bound[others]) <= 1
    assert out[7].isnan().all()


@pytest.mark.parametrize("hq,hkv,D,rows,splits", [(16, 2, 256, 50, 0), (8, 2, 128, 700, 0), (16, 4, 64, 90, 1),
                                                    (16, 2, 256, 150, 3), (16, 4, 64, 900, 0)])
def test_attention_keeps_a_nodes_non_finite_value_from_nodes_that_do_not_see_it(hq, hkv, D, rows, splits):
    rng = np.random.default_rng(D)
    parents = tree("tree", 70)
    n = len(parents)
    kv = bf16(rng, 2, rows + n + 3, hkv, D)
    clean = kv.clone()
    kv[1, rows + 3, 1, 7] = float("nan")
    kv[1, rows + 66, 0, 0] = float("inf")
    kv[1, rows + 40, 1, D - 1] = 3e38          # beyond f16: the same, and reported
    out, _, _, ws = _attn(hq, hkv, D, rows, parents, kv=kv, splits=splits)
    _, want, bound, _ = _attn(hq, hkv, D, rows, parents, kv=clean, splits=splits)
    spoilt = np.zeros(want.shape, bool)
    G = hq // hkv
    for i in range(n):
        line = O.line(parents, i)
        spoilt[i, G:2 * G, 7] |= 3 in line
        spoilt[i, :G, 0] |= 66 in line
        spoilt[i, G:2 * G, D - 1] |= 40 in line
    got = f64(out)
    assert spoilt.any() and not np.isfinite(got[spoilt]).any()
    assert worst(got[~spoilt], want[~spoilt], np.broadcast_to(bound, want.shape)[~spoilt]) <= 1
    assert tu.workspace_faults(ws) == 4
    # a cached row is seen by every node
    kv = clean.clone()
    kv[1, 5, 0, 2] = float("nan")
    out, _, _, _ = _attn(hq, hkv, D, rows, parents, kv=kv, splits=splits)
    got = f64(out)
    assert np.isnan(got[:, :G, 2]).all() and np.isfinite(np.delete(got, 2, axis=2)).all() and np.isfinite(got[:, G:]).all()


def test_attention_reports_values_beyond_f16():
    rng = np.random.default_rng(6)
    kv = bf16(rng, 2, 64, 2, 128)
    kv[1, 3, 1, 5] = 1e5
    _, _, _, ws = _attn(16, 2, 128, 50, tree("tree", 11), kv=kv)
    assert tu.workspace_faults(ws) == 4


def test_attention_over_a_long_cache():
    hq, hkv, D, rows = 16, 2, 256, 40000
    parents = tree("tree", 24)
    n, g = len(parents), torch.Generator(device=DEV).manual_seed(3)
    k, v = torch.randn(2, rows + n, hkv, D, device=DEV, generator=g).to(torch.bfloat16)
    q = torch.randn(n, hq, D, device=DEV, generator=g).to(torch.bfloat16)
    out = torch.empty_like(q)
    tu.draft_attention(_ctx(rows, n), k, v, tu.attn_params(hq, hkv, D), tu.Draft(parents), q, out)
    for i in (0, 5, n - 1):
        see = torch.cat([torch.arange(rows), rows + torch.tensor(O.line(parents, i))]).to(DEV)
        for h in (0, 9, 15):
            z = k[see, h // 8].double() @ q[i, h].double() / 16
            p = torch.softmax(z, 0)
            V = v[see, h // 8].double()
            want, mag = p @ V, p @ V.abs()
            err = (out[i, h].double() - want).abs()
            assert (err <= BF16 * want.abs() + (2 * F16 + 2 * (264 * F32 * 20 + 16 * F32)) * mag + 2.0 ** -18).all()


# ----------------------------------------------------------------------------- recurrent layers

@pytest.mark.parametrize("W", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("kind,n", [("chain", 1), ("tree", 9), ("forest", 128)])
def test_short_conv(W, kind, n):
    rng = np.random.default_rng([W, n])
    parents, items, host = tree(kind, n), [], []
    for C in (8, 24, 2056):
        st, x, w = bf16(rng, W - 1, C), bf16(rng, n, C), bf16(rng, C, W)
        host.append((st, x, w))
        items.append((dev(st), dev(x), dev(w), torch.full((n, C), 9.0, dtype=torch.bfloat16, device=DEV)))
    for act in ("silu", "none"):
        tu.draft_short_conv(tu.Draft(parents), items, activation=act)
        for (st, x, w), (sd, xd, wd, out) in zip(host, items):
            want, mag = O.draft_short_conv(f64(st), f64(x), f64(w), parents, act == "silu")
            assert worst(out, want, BF16 * np.abs(want) + (W + 24) * F32 * 1.1 * mag) <= 1
            assert torch.equal(sd.cpu(), st)


def _delta_bound(S0, c, parents, scale, d, n):
    """fp32 roundings of sums of d and n products, relative to what the same formulas give with magnitudes."""
    mag = O.draft_delta_rule(np.abs(S0), np.abs(f64(c["q"])), np.abs(f64(c["k"])), np.abs(f64(c["v"])), f64(c["beta"]),
                             f64(c["g"]), parents, abs(scale), sign=1.0)
    return (d + 2 * n + 40) * F32 * mag


@pytest.mark.parametrize("Hk,Hv,d", [(16, 32, 128), (2, 2, 64), (1, 3, 128), (8, 16, 64)])
@pytest.mark.parametrize("kind,n", [("chain", 1), ("chain", 16), ("star", 17), ("tree", 33), ("forest", 64), ("tree", 65),
                                    ("chain", 128)])
def test_delta_rule(Hk, Hv, d, kind, n):
    rng = np.random.default_rng([Hv, d, n])
    parents, c = tree(kind, n), delta_inputs(rng, n, Hk, Hv, d)
    x = {k: dev(t) for k, t in c.items()}
    out = torch.full((n, Hv, d), 7.0, device=DEV)
    p = tu.delta_params(Hk, Hv, d, d, 64)
    tu.draft_delta_rule(x["state"], x["q"], x["k"], x["v"], x["beta"], x["g"], p, tu.Draft(parents), out)
    args = [f64(c[k]) for k in ("state", "q", "k", "v", "beta", "g")]
    want = O.draft_delta_rule(*args, parents, d ** -0.5)
    assert worst(out, want, _delta_bound(args[0], c, parents, d ** -0.5, d, n)) <= 1
    assert torch.equal(x["state"].cpu(), c["state"])


def test_delta_rule_gates_at_their_ends():
    rng = np.random.default_rng(1)
    n, Hk, Hv, d = 40, 2, 4, 128
    parents, c = tree("tree", n), delta_inputs(rng, n, Hk, Hv, d)
    c["g"][::3] = 0.0            # computed as 2^-100
    c["g"][1::3] = 1.0
    c["beta"][::4] = 0.0
    c["beta"][1::4] = 1.0
    x = {k: dev(t) for k, t in c.items()}
    out = torch.zeros(n, Hv, d, device=DEV)
    tu.draft_delta_rule(x["state"], x["q"], x["k"], x["v"], x["beta"], x["g"], tu.delta_params(Hk, Hv, d, d, 16),
                        tu.Draft(parents), out)
    args = [f64(c[k]) for k in ("state", "q", "k", "v", "beta", "g")]
    want = O.draft_delta_rule(*args, parents, d ** -0.5)
    # 2^-100 of a state of unit size against zero is far below the bound's floor
    assert worst(out, want, _delta_bound(args[0], c, parents, d ** -0.5, d, n) + 2.0 ** -80) <= 1


def test_delta_rule_non_finite_nodes_stay_on_their_path():
    rng = np.random.default_rng(2)
    n, Hk, Hv, d = 50, 1, 2, 64
    parents, c = tree("tree", n), delta_inputs(rng, n, Hk, Hv, d)
    clean = {k: t.clone() for k, t in c.items()}
    c["k"][9, 0, 3] = float("nan")
    c["v"][20, 1, 5] = float("inf")
    c["q"][30, 0, 1] = float("nan")
    x = {k: dev(t) for k, t in c.items()}
    out = torch.zeros(n, Hv, d, device=DEV)
    tu.draft_delta_rule(x["state"], x["q"], x["k"], x["v"], x["beta"], x["g"], tu.delta_params(Hk, Hv, d, d, 16),
                        tu.Draft(parents), out)
    args = [f64(clean[k]) for k in ("state", "q", "k", "v", "beta", "g")]
    want = O.draft_delta_rule(*args, parents, d ** -0.5)
    bad = np.zeros((n, Hv, d), bool)
    for i in range(n):
        seen = O.line(parents, i)
        bad[i] |= 9 in seen or i == 30
        bad[i, 1, 5] |= 20 in seen
    got = out.cpu().numpy()
    assert not np.isfinite(got[bad]).any() and bad.any()
    bound = _delta_bound(args[0], clean, parents, d ** -0.5, d, n)
    assert worst(got[~bad], want[~bad], bound[~bad]) <= 1


# ----------------------------------------------------------------------------- verification

def _verify(parents, tok, target, u, proposal=None, pad=0, **kw):
    n, V = target.shape
    def rows(x):
        t = torch.full((n, V + pad), 9.0, device=DEV)
        t[:, :V] = torch.from_numpy(x)
        return t[:, :V]
    ws = torch.empty(tu.draft_verify_workspace_size(tu.Draft(parents), V), dtype=torch.uint8, device=DEV)
    r = tu.draft_verify(tu.Draft(parents), torch.from_numpy(tok).to(DEV), rows(target), torch.from_numpy(u).to(DEV),
                        proposal=None if proposal is None else rows(proposal), workspace=ws, **kw).cpu().tolist()
    assert tu.workspace_faults(ws) == 0
    return r


def _want(parents, tok, target, u, proposal=None):
    path, nxt = O.draft_verify(parents, tok, target.astype(np.float64), u.astype(np.float64),
                               None if proposal is None else proposal.astype(np.float64))
    return [len(path), nxt] + path + [-1] * (len(parents) - len(path))


@pytest.mark.parametrize("V,pad", [(1, 0), (2, 3), (63, 1), (4097, 0), (50001, 7), (300000, 0)])
@pytest.mark.parametrize("kind,n", [("chain", 1), ("chain", 7), ("star", 12), ("tree", 40), ("tree", 128)])
@pytest.mark.parametrize("drawn", [True, False])
def test_verify(V, pad, kind, n, drawn):
    if V * n > 8_000_000:
        n = max(1, 8_000_000 // V)
    parents = tree(kind, n)
    for seed in range(3 if V > 10000 else 8):
        rng = np.random.default_rng([V, n, seed, drawn])
        target = rows_of(rng, n, V)
        near = rows_of(rng, n, V, 0.7) if seed % 2 else target        # a poor and a perfect drafter
        proposal = (0.5 * near + 0.5 * rows_of(rng, n, V)).astype(np.float32)
        tok = drafted(rng, parents, proposal, distinct=not drawn)
        u = rng.random(n).astype(np.float32)
        if seed == 2:
            u[:] = 0.0
        q = proposal if drawn else None
        assert _verify(parents, tok, target, u, q, pad) == _want(parents, tok, target, u, q)


def test_verify_edges():
    parents, V = [-1, 0, 0, 1, 3], 5000
    rng = np.random.default_rng(0)
    target, proposal = rows_of(rng, 5, V), rows_of(rng, 5, V)
    tok, u = drafted(rng, parents, proposal), rng.random(5).astype(np.float32)
    # tokens outside the vocabulary are never accepted
    out = tok.copy()
    out[1], out[2] = -3, V
    for q in (proposal, None):
        assert _verify(parents, out, target, u, q) == _want(parents, out, target, u, q)
    # one-hot target: the child that holds the token, and it alone
    hot = np.zeros((5, V), np.float32)
    hot[0, tok[2]] = hot[2, 4999] = 1
    assert _verify(parents, tok, hot, u, proposal)[:4] == [2, 4999, 0, 2]
    # the drafter's rows are the target's: every first child is accepted
    assert _verify(parents, drafted(rng, parents, target), target, u, target)[0] == 4
    # u[0] just below 1, and a tail of zeros: the last token with a share
    zt = target.copy()
    zt[:, 4000:] = 0
    one = np.array([np.nextafter(np.float32(1), np.float32(0))], np.float32)
    assert _verify([-1], np.zeros(1, np.int32), zt[:1], one) == _want([-1], np.zeros(1, np.int32), zt[:1], one)
    # rows without a sum
    for bad in (0.0, float("nan")):
        t = np.full((1, V), bad, np.float32)
        assert _verify([-1], np.zeros(1, np.int32), t, np.array([0.3], np.float32)) == [1, -1, 0]
    # nothing is left after a rejection: the row itself is drawn from
    same = np.full((2, 4), 0.25, np.float32)
    same[0] = [0.5, 0.5, 0, 0]
    got = _verify([-1, 0], np.array([0, 2], np.int32), same, np.array([0.7, 0.5], np.float32), np.repeat(same[:1], 2, 0))
    assert got == [1, 1, 0, -1]
    # the same token twice among siblings
    dup = np.array([0, 7, 7, 7, 7], np.int32)
    star = [-1, 0, 0, 0, 0]
    for q in (proposal, None):
        for s in range(6):
            us = np.random.default_rng(s).random(5).astype(np.float32)
            assert _verify(star, dup, target, us, q) == _want(star, dup, target, us, q)


# ----------------------------------------------------------------------------- acceptance

@pytest.mark.parametrize("n_attn,n_delta,hkv,D,Hk,Hv,d,W", [(1, 1, 2, 256, 2, 4, 128, 4), (20, 40, 1, 64, 1, 1, 64, 3),
                                                             (2, 0, 4, 128, 1, 1, 64, 4), (0, 2, 1, 64, 1, 2, 128, 8)])
@pytest.mark.parametrize("path", [[0], [0, 1, 2, 3], [0, 2, 5, 6, 11, 19]])
def test_accept(n_attn, n_delta, hkv, D, Hk, Hv, d, W, path):
    rng = np.random.default_rng([n_attn, n_delta, len(path)])
    n, rows = 20, 41
    parents = [-1] + [max(0, i // 2 - 1) for i in range(1, n)]
    for a, b in zip(path, path[1:]):
        parents[b] = a
    kv = bf16(rng, 2 * n_attn, rows + n + 2, hkv, D)
    cs = [delta_inputs(rng, n, Hk, Hv, d) for _ in range(n_delta)]
    conv = [(bf16(rng, W - 1, 40), bf16(rng, n, 40)) for _ in range(n_delta)]
    kvd = dev(kv)
    xs = [{k: dev(t) for k, t in c.items()} for c in cs]
    cd = [(dev(a), dev(b)) for a, b in conv]
    layers = [tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[kvd[2 * l]], v_cache=[kvd[2 * l + 1]])
              for l in range(n_attn)]
    layers += [tu.LayerIO(tu.TU_LAYER_DELTA, None, x["k"], x["v"], None, state=[x["state"]], beta=x["beta"], g=x["g"])
               for x in xs]
    stack = tu.DraftStack(layers, tu.attn_params(hkv, hkv, D), tu.delta_params(Hk, Hv, d, d, 64), cd)
    ctx = _ctx(rows, n, 1000, spare=2)
    tu.draft_accept(ctx, tu.Draft(parents), path, stack)
    a = len(path)
    assert (ctx.len, ctx.next_pos, ctx.vt_rows) == (rows + a, 1000 + a, 0) and ctx.intervals() == [(1000 - rows, 1000 + a)]
    assert ctx.pos[rows:rows + a].tolist() == list(range(1000, 1000 + a))
    want = kv.clone()
    want[:, rows:rows + a] = kv[:, [rows + i for i in path]]
    assert torch.equal(kvd.cpu()[:, :rows + a], want[:, :rows + a])
    assert torch.equal(kvd.cpu()[:, rows + n:], kv[:, rows + n:])
    for c, x in zip(cs, xs):
        S, M = f64(c["state"]), np.abs(f64(c["state"]))
        for i in path:
            step = [f64(c[k][i]) for k in ("k", "v", "beta", "g")]
            S, M = O.delta_step(S, *step), O.delta_step(M, *[np.abs(t) for t in step], sign=1.0)
        assert worst(x["state"], S, (d + 8) * a * F32 * M) <= 1
    for (st, x), (sd, _) in zip(conv, cd):
        assert torch.equal(sd.cpu(), torch.cat([st, x[path]])[-(W - 1):])


# ----------------------------------------------------------------------------- a whole step

def _step_setup(seed=0, rows=300, n=21):
    rng = np.random.default_rng(seed)
    hq, hkv, D, Hk, Hv, d, W, V = 16, 2, 256, 2, 4, 128, 4, 1000
    c = delta_inputs(rng, n, Hk, Hv, d)
    s = dict(rows=rows, n=n, parents=tree("tree", n, seed), attn=tu.attn_params(hq, hkv, D, 64, THETA),
             delta=tu.delta_params(Hk, Hv, d, d, 64), ctx=_ctx(rows, n, 5000, spare=n))
    s["kc"], s["vc"] = dev(bf16(rng, 2, rows + 2 * n, hkv, D))
    s["qkv"] = dev(bf16(rng, n, hq + 2 * hkv, D))
    s["w"] = dev(bf16(rng, 2, D))
    s["x"] = {k: dev(t) for k, t in c.items()}
    s["conv"] = [dev(bf16(rng, W - 1, Hv * d)), dev(bf16(rng, n, Hv * d)), dev(bf16(rng, Hv * d, W)),
                 torch.zeros(n, Hv * d, dtype=torch.bfloat16, device=DEV)]
    target, proposal = rows_of(rng, n, V), rows_of(rng, n, V, 1.5)
    s["tok"] = torch.from_numpy(drafted(rng, s["parents"], proposal)).to(DEV)
    s["target"], s["proposal"] = torch.from_numpy(target).to(DEV), torch.from_numpy(proposal).to(DEV)
    s["u"] = torch.from_numpy(rng.random(n).astype(np.float32)).to(DEV)
    s["q_hat"] = torch.zeros(n, hq, D, dtype=torch.bfloat16, device=DEV)
    s["o"], s["od"] = torch.zeros_like(s["q_hat"]), torch.zeros(n, Hv, d, device=DEV)
    s["result"] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
    s["draft"] = tu.Draft(s["parents"])
    s["norm"] = tu.QkNorm("rms", 1e-6, s["w"][0], s["w"][1])
    s["ws"] = torch.empty(tu.draft_attention_workspace_size(s["ctx"], s["attn"], s["draft"]), dtype=torch.uint8, device=DEV)
    s["wv"] = torch.empty(tu.draft_verify_workspace_size(s["draft"], V), dtype=torch.uint8, device=DEV)
    return s


def _step(s, stream=None):
    hq, hkv = 16, 2
    x, q = s["x"], s["qkv"]
    tu.draft_append(s["ctx"], s["kc"], s["vc"], s["attn"], s["draft"], q[:, :hq], q[:, hq:hq + hkv], q[:, hq + hkv:],
                    s["q_hat"], norm=s["norm"], stream=stream)
    tu.draft_attention(s["ctx"], s["kc"], s["vc"], s["attn"], s["draft"], s["q_hat"], s["o"], workspace=s["ws"], stream=stream)
    tu.draft_short_conv(s["draft"], [s["conv"]], stream=stream)
    v = s["conv"][3].view(s["n"], 4, 128)
    tu.draft_delta_rule(x["state"], x["q"], x["k"], v, x["beta"], x["g"], s["delta"], s["draft"], s["od"], stream=stream)
    tu.draft_verify(s["draft"], s["tok"], s["target"], s["u"], s["result"], proposal=s["proposal"], workspace=s["wv"],
                    stream=stream)
    return [t.clone() for t in (s["o"], s["od"], s["result"])]


def test_a_step_and_what_it_leaves_equal_plain_decoding():
    """The path that a step accepts, run afterwards token by token through the package's own tail
    calls from the same context, gives the same outputs, cache rows and states."""
    s = _step_setup()
    kc0, vc0, S0, cs0 = s["kc"].clone(), s["vc"].clone(), s["x"]["state"].clone(), s["conv"][0].clone()
    o, od, result = _step(s)
    r = result.tolist()
    path = r[2:2 + r[0]]
    assert path[0] == 0
    v = s["conv"][3].view(s["n"], 4, 128).clone()
    layers = [tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[s["kc"]], v_cache=[s["vc"]]),
              tu.LayerIO(tu.TU_LAYER_DELTA, None, s["x"]["k"], v, None, state=[s["x"]["state"]], beta=s["x"]["beta"],
                         g=s["x"]["g"])]
    tu.draft_accept(s["ctx"], s["draft"], path, tu.DraftStack(layers, s["attn"], s["delta"], [tuple(s["conv"][:2])]))
    # the same tokens as a tail
    a, rows, P = len(path), s["rows"], torch.tensor(path, device=DEV)
    ctx = _ctx(rows, s["n"], 5000, spare=s["n"])
    ctx.pos.copy_(s["ctx"].pos)
    q = s["qkv"][P].contiguous()
    qn, kn = q[:, :16].contiguous(), q[:, 16:18].contiguous()
    tu.qk_norm_rope(s["attn"], qn, kn, qn, kn, norm=s["norm"], first_pos=5000)
    out = torch.zeros(a, 16, 256, device=DEV)
    plain = tu.attn_params(16, 2, 256, 0, THETA)
    tu.tail_prefill_attention(ctx, kc0, vc0, plain, qn, kn, q[:, 18:].contiguous(), out)
    tu.commit_tail(ctx, a)
    assert (o[P].float() - out).abs().max() <= 2 * BF16 * out.abs().max()
    assert torch.equal(kc0[:rows + a], s["kc"][:rows + a]) and torch.equal(vc0[:rows + a], s["vc"][:rows + a])
    assert (ctx.len, ctx.next_pos, ctx.intervals()) == (s["ctx"].len, s["ctx"].next_pos, s["ctx"].intervals())
    assert torch.equal(ctx.pos[rows:rows + a], s["ctx"].pos[rows:rows + a])
    x = s["x"]
    y = torch.zeros(a, 512, dtype=torch.bfloat16, device=DEV)
    tu.short_conv_continue(cs0, s["conv"][1][P].contiguous(), s["conv"][2], y)
    assert torch.equal(cs0, s["conv"][0])
    assert (y.float() - v.view(-1, 512)[P].float()).abs().max() <= 2 * BF16 * y.float().abs().max()
    od2 = torch.zeros(a, 4, 128, device=DEV)
    tu.delta_rule_continue(S0, x["q"][P].contiguous(), x["k"][P].contiguous(), v[P].contiguous(), x["beta"][P].contiguous(),
                           x["g"][P].contiguous(), s["delta"], od2)
    assert (od2 - od[P]).abs().max() <= 1e-3 * od2.abs().max()
    assert (S0 - x["state"]).abs().max() <= 1e-3 * S0.abs().max()


def test_a_step_again_on_a_stream_and_from_a_graph():
    s = _step_setup(1)
    want = _step(s)
    for got in (_step(s), ):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(s)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # two graphs that share the workspaces, replayed in turn with eager steps between
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = _step(s)
        graphs.append((g, outs))
    for _ in range(3):
        for g, outs in graphs:
            for t in (s["o"], s["od"], s["result"], *outs):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
            assert all(torch.equal(a, b) for a, b in zip(_step(s), want))

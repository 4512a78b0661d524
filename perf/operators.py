"""Operators of one speculative decoding step of a hybrid context: what is measured.

A drafter proposes a tree of tokens after the context's last token (node 0); the model runs
the whole tree at once, the target's probabilities accept one path of it, and the path is
kept. The operators, as a program calls them:

  1. queries and keys, normed for each head and rotated in one pass
       norm    qk_norm_rope over T tokens
       append  draft_append: the nodes of a draft, keys and values into the cache
  2. attention of the tree over the cache
       attn    draft_attention: each node sees the cache and its own ancestors
  3. the recurrent layers over the tree, the carried states untouched
       conv    draft_short_conv: the short convolution along each node's path
       delta   draft_delta_rule: the gated delta rule along each node's path
  4. verification against the target's probabilities
       verify  draft_verify: the accepted path and the next token, from given random numbers
  5. the accepted path is kept
       accept  draft_accept: its cache rows, delta states and convolution states

`own` False computes them in elementary torch operations, True through the package. Sizes
are the package's own (heads 16/2 of 256, 16-32 of 128, 12 + 36 layers, 12K to 64K rows)
and generic vocabularies.
"""
import math
import random

import torch

own = False   # set by the tools: True calls the package

DEV = "cuda"
THETA = 1.0e7
EPS = 1e-6

ATTN_SHAPES = [(16, 2, 256), (32, 8, 128), (16, 4, 64), (8, 8, 128)]      # query heads, KV heads, head dim
DELTA_SHAPES = [(16, 32, 128), (16, 16, 128), (8, 16, 64), (2, 2, 64)]    # key heads, value heads, d


def listed():
    a, d = dict(hq=16, hkv=2, dim=256), dict(hk=16, hv=32, d=128)
    return [
        # the queries and keys of one layer of a full refill
        dict(name="norm-refill", kind="norm", T=8191, rotary=256, **a),
        # a single token enters one layer: pure latency
        dict(name="append-token", kind="append", n=1, spine=1, rows=11907, rotary=256, **a),
        # plain decoding of one token over a 32K context
        dict(name="attn-token", kind="attn", n=1, spine=1, rows=32768, **a),
        # a usual draft of a speaking character: 24 nodes over a 12K context
        dict(name="attn-draft", kind="attn", n=24, spine=6, rows=11907, **a),
        # a wide tree over the long-lived character's 64K context
        dict(name="attn-tree", kind="attn", n=64, spine=8, rows=65536, **a),
        # the short convolutions (q, k, v) of one recurrent layer over a wide tree
        dict(name="conv-tree", kind="conv", n=64, spine=8, cq=2048, ck=2048, cv=4096, width=4, silu=True),
        # one recurrent layer over a short chain, and over the wide tree
        dict(name="delta-chain", kind="delta", n=7, spine=7, **d),
        dict(name="delta-tree", kind="delta", n=64, spine=8, **d),
        # a chain drawn from a drafter's distributions, and a tree of several drawn children a node
        dict(name="verify-chain", kind="verify", n=6, spine=6, vocab=131072, drawn=True),
        dict(name="verify-tree", kind="verify", n=64, spine=8, vocab=131072, drawn=True),
        # four layers keep a path of 3 tokens; the 48-layer stack keeps one of 6
        dict(name="accept-few", kind="accept", n=24, spine=3, rows=11907, n_attn=1, n_delta=3, width=4, **a, **d),
        dict(name="accept-stack", kind="accept", n=64, spine=6, rows=32768, n_attn=12, n_delta=36, width=4, **a, **d),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "attn", "attn", "attn", "conv", "delta", "delta", "verify", "verify", "accept"])
    hq, hkv, dim = ATTN_SHAPES[0] if rng.random() < 0.5 else rng.choice(ATTN_SHAPES[1:])
    hk, hv, d = DELTA_SHAPES[0] if rng.random() < 0.5 else rng.choice(DELTA_SHAPES[1:])
    a, dl = dict(hq=hq, hkv=hkv, dim=dim), dict(hk=hk, hv=hv, d=d)
    if kind == "norm":
        return dict(kind=kind, T=_log_int(rng, 1, 8191), rotary=rng.choice([dim, dim, dim // 2, dim // 4, 20, 0]), **a)
    n = _log_int(rng, 1, 64)
    tree = dict(kind=kind, n=n, spine=n if rng.random() < 0.2 else rng.randint(1, min(n, 10)))
    if kind == "append":
        return dict(tree, rows=_log_int(rng, 1, 65536), rotary=rng.choice([dim, dim, dim // 2, dim // 4, 20, 0]), **a)
    if kind == "attn":
        return dict(tree, rows=_log_int(rng, 16, 65536), **a)
    if kind == "conv":
        return dict(tree, cq=hk * d, ck=hk * d, cv=hv * d, width=rng.choice([2, 3, 4, 4]), silu=rng.random() < 0.8)
    if kind == "delta":
        return dict(tree, **dl)
    if kind == "verify":
        return dict(tree, vocab=_log_int(rng, 257, 131072), drawn=rng.random() < 0.6)
    few = rng.random() < 0.6
    return dict(tree, spine=min(tree["spine"], 10), rows=_log_int(rng, 256, 32768), n_attn=1 if few else 12,
                n_delta=rng.choice([0, 1, 3]) if few else 36, width=4, **a, **dl)


# ----------------------------------------------------------------------------- inputs

class _Inputs:
    """Seeded draws on the device, each tensor from a generator of its own."""

    def __init__(self, seed):
        self.seed, self.n = int(seed), 0

    def _gen(self):
        self.n += 1
        return torch.Generator(device=DEV).manual_seed((self.seed * 1000003 + self.n) & 0x7FFFFFFFFFFF)

    def f32(self, *shape):
        return torch.randn(shape, generator=self._gen(), device=DEV, dtype=torch.float32)

    def bf16(self, *shape):
        return self.f32(*shape).to(torch.bfloat16)

    def unit(self, *shape):   # in [0, 1)
        return torch.rand(shape, generator=self._gen(), device=DEV, dtype=torch.float32)

    def keys(self, *shape):   # L2-normalised keys of the delta rule
        x = self.f32(*shape)
        return (x / x.square().sum(-1, keepdim=True).sqrt()).to(torch.bfloat16)

    def beta(self, *shape):
        return torch.sigmoid(self.f32(*shape))

    def gate(self, *shape):
        return torch.exp(-torch.nn.functional.softplus(self.f32(*shape) - 4.0))


def _tree(c, seed):
    """Parents of a tree of c['n'] nodes that holds a path of c['spine'] nodes from node 0, and that path."""
    rng = random.Random("tree %d %d %d" % (seed, c["n"], c["spine"]))
    n = c["n"]
    path = [0] + sorted(rng.sample(range(1, n), c["spine"] - 1))
    parents = [-1] + [max(0, rng.randint(0, i - 1)) if rng.random() < 0.5 else max(0, i // 3) for i in range(1, n)]
    for j in range(1, len(path)):
        parents[path[j]] = path[j - 1]
    return parents, path


def _plan(parents, width=1, ranks=False):
    """What the plain forms index with: who is whose ancestor (or the node itself), depths, the
    convolution's rows, the children of each node by rank."""
    n = len(parents)
    seen = torch.eye(n, dtype=torch.bool)
    for i in range(n):
        if parents[i] >= 0:
            seen[i] |= seen[parents[i]]
    plan = {"seen": seen.to(DEV), "depth": (seen.sum(1) - 1).to(DEV)}
    rows = []
    for i in range(n):   # row of [state; x] under each tap of node i
        r, at = [], i
        for _ in range(width):
            r.append(width - 1 + at)
            at = parents[at] if at >= 0 else at - 1
        rows.append([max(0, x) for x in r[::-1]])
    plan["taps"] = torch.tensor(rows, device=DEV)
    if ranks:
        kids = [[j for j in range(n) if parents[j] == i] for i in range(n)]
        most = max(1, max(len(x) for x in kids))
        plan["kids"] = torch.tensor([[x[r] if r < len(x) else -1 for x in kids] for r in range(most)], device=DEV)
        plan["parents"] = torch.tensor([max(0, p) for p in parents], device=DEV)
    return plan


def _proposals(c, x, parents):
    """Target rows, drafter's rows, drafted tokens and random numbers."""
    n, V = c["n"], c["vocab"]
    z = x.f32(n, V) * 2.5
    target = torch.softmax(z, -1)
    proposal = torch.softmax(0.9 * z + 0.6 * x.f32(n, V), -1)
    par = torch.tensor([max(0, p) for p in parents], device=DEV)
    if c["drawn"]:      # each child drawn from its parent's row
        cdf = proposal.double().cumsum(-1)[par]
        tokens = torch.searchsorted(cdf, x.unit(n, 1).double() * cdf[:, -1:], right=True)[:, 0].clamp(max=V - 1)
    else:               # the drafter's most likely tokens, in order
        rank = [sum(parents[j] == parents[i] for j in range(i)) for i in range(n)]
        top = proposal.topk(max(rank) + 1, dim=-1).indices
        tokens = top[par, torch.tensor(rank, device=DEV)]
        proposal = None
    return {"target": target, "proposal": proposal, "tokens": tokens.to(torch.int32), "u": x.unit(n)}


def prepare(c, seed):
    x, s = _Inputs(seed), {"c": c}
    kind = c["kind"]
    if kind != "norm":
        s["parents"], s["path"] = _tree(c, seed)
        s["plan"] = _plan(s["parents"], c.get("width", 1), kind == "verify")
    if kind in ("norm", "append"):
        T = c["T"] if kind == "norm" else c["n"]
        qkv = x.bf16(T, c["hq"] + 2 * c["hkv"], c["dim"]) * 3   # one projection's output: rows of q, k and v heads
        s["q"], s["k"], s["v"] = qkv.split([c["hq"], c["hkv"], c["hkv"]], dim=1)
        s["wq"], s["wk"] = (1 + 0.2 * x.f32(2, c["dim"])).to(torch.bfloat16)
        s["first"] = 479547 if kind == "norm" else c["rows"] + 260000
        s["q_hat"] = torch.zeros((T, c["hq"], c["dim"]), dtype=torch.bfloat16, device=DEV)
        s["k_hat"] = torch.zeros((T, c["hkv"], c["dim"]), dtype=torch.bfloat16, device=DEV)
    if kind in ("append", "attn"):
        n, rows = c["n"], c["rows"]
        s["k_cache"], s["v_cache"] = x.bf16(2, rows + n + 3, c["hkv"], c["dim"])
        if kind == "attn":
            s["q_hat"] = x.bf16(n, c["hq"], c["dim"])
            s["out"] = torch.zeros_like(s["q_hat"])
    if kind == "conv":
        s["conv"] = [(x.bf16(c["width"] - 1, ch), x.bf16(c["n"], ch), (x.f32(ch, c["width"]) * 0.5).to(torch.bfloat16),
                      torch.zeros((c["n"], ch), dtype=torch.bfloat16, device=DEV)) for ch in (c["cq"], c["ck"], c["cv"])]
    if kind == "delta":
        n = c["n"]
        s.update(state=0.1 * x.f32(c["hv"], c["d"], c["d"]), q=x.bf16(n, c["hk"], c["d"]), k=x.keys(n, c["hk"], c["d"]),
                 v=x.bf16(n, c["hv"], c["d"]), beta=x.beta(n, c["hv"]), g=x.gate(n, c["hv"]),
                 out=torch.zeros((n, c["hv"], c["d"]), dtype=torch.float32, device=DEV))
    if kind == "verify":
        s.update(_proposals(c, x, s["parents"]))
    if kind == "accept":
        n, na, nd = c["n"], c["n_attn"], c["n_delta"]
        s["kv"] = x.bf16(2, na, c["rows"] + n, c["hkv"], c["dim"])
        s["S"] = 0.1 * x.f32(nd, c["hv"], c["d"], c["d"])
        s["k"], s["v"] = x.keys(nd, n, c["hk"], c["d"]), x.bf16(nd, n, c["hv"], c["d"])
        s["beta"], s["g"] = x.beta(nd, n, c["hv"]), x.gate(nd, n, c["hv"])
        ch = (2 * c["hk"] + c["hv"]) * c["d"]
        s["cs"], s["cx"] = x.bf16(nd, c["width"] - 1, ch), x.bf16(nd, n, ch)
        s["path_d"] = torch.tensor(s["path"], device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """The package's handles that a program keeps."""
    import paper_2609_18935_amd as tu
    c = s["c"]
    if "hq" in c:
        s["attn"] = tu.attn_params(c["hq"], c["hkv"], c["dim"], c.get("rotary", c["dim"]), THETA)
    if "hk" in c:
        s["delta"] = tu.delta_params(c["hk"], c["hv"], c["d"], c["d"], 64)
    if "wq" in s:
        s["norm"] = tu.QkNorm("rms", EPS, s["wq"], s["wk"])
    if c["kind"] != "norm":
        s["draft"] = tu.Draft(s["parents"])
    if "rows" in c:
        s["ctx"] = tu.Context(c["rows"] + c["n"], device=DEV)
        s["live"], s["cursor"] = [(260000, 260000 + c["rows"])], 260000 + c["rows"]
        s["ctx"].set_metadata(s["live"], s["cursor"])
    if c["kind"] == "attn":
        s["ws"] = torch.empty(tu.draft_attention_workspace_size(s["ctx"], s["attn"], s["draft"]), dtype=torch.uint8,
                              device=DEV)
    if c["kind"] == "verify":
        s["ws"] = torch.empty(tu.draft_verify_workspace_size(s["draft"], c["vocab"]), dtype=torch.uint8, device=DEV)
        s["result"] = torch.zeros(c["n"] + 2, dtype=torch.int32, device=DEV)
    if c["kind"] == "accept":
        layers = [tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[s["kv"][0, l]], v_cache=[s["kv"][1, l]])
                  for l in range(c["n_attn"])]
        layers += [tu.LayerIO(tu.TU_LAYER_DELTA, None, s["k"][l], s["v"][l], None, state=[s["S"][l]],
                              beta=s["beta"][l], g=s["g"][l]) for l in range(c["n_delta"])]
        s["stack"] = tu.DraftStack(layers, s["attn"], s["delta"], [(s["cs"][l], s["cx"][l]) for l in range(c["n_delta"])])


# ----------------------------------------------------------------------------- one pass

def run(s):
    return _own(s) if own else _PLAIN[s["c"]["kind"]](s)


def _own(s):
    import paper_2609_18935_amd as tu
    c = s["c"]
    kind = c["kind"]
    if kind == "norm":
        tu.qk_norm_rope(s["attn"], s["q"], s["k"], s["q_hat"], s["k_hat"], norm=s["norm"], first_pos=s["first"])
        return s["q_hat"], s["k_hat"]
    if kind == "append":
        tu.draft_append(s["ctx"], s["k_cache"], s["v_cache"], s["attn"], s["draft"], s["q"], s["k"], s["v"], s["q_hat"],
                        norm=s["norm"])
        at = slice(c["rows"], c["rows"] + c["n"])
        return s["q_hat"], s["k_cache"][at], s["v_cache"][at]
    if kind == "attn":
        tu.draft_attention(s["ctx"], s["k_cache"], s["v_cache"], s["attn"], s["draft"], s["q_hat"], s["out"],
                           workspace=s["ws"])
        return s["out"]
    if kind == "conv":
        tu.draft_short_conv(s["draft"], s["conv"], activation="silu" if c["silu"] else "none")
        return [o for _, _, _, o in s["conv"]]
    if kind == "delta":
        tu.draft_delta_rule(s["state"], s["q"], s["k"], s["v"], s["beta"], s["g"], s["delta"], s["draft"], s["out"])
        return s["out"]
    if kind == "verify":
        tu.draft_verify(s["draft"], s["tokens"], s["target"], s["u"], s["result"], proposal=s["proposal"],
                        workspace=s["ws"])
        return s["result"]
    s["ctx"].set_metadata(s["live"], s["cursor"])   # every pass keeps the path at the same length
    tu.draft_accept(s["ctx"], s["draft"], s["path"], s["stack"])
    return _kept(s)


def _kept(s):
    c = s["c"]
    return s["kv"][:, :, c["rows"]:c["rows"] + len(s["path"])], s["S"], s["cs"]


def _norm_rope(x, w, pos, rotary):
    """RMS norm of each head's row, times the weight, then rotate-half pairs (j, j + rotary / 2)."""
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    half = rotary // 2
    j = torch.arange(half, device=DEV, dtype=torch.float64)
    angle = pos.double()[:, None] * THETA ** (-2.0 * j / max(1, rotary))
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., :half], x[..., half:rotary]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rotary:]], -1).to(torch.bfloat16)


def _plain_norm(s):
    c = s["c"]
    pos = s["first"] + torch.arange(c["T"], device=DEV)
    return _norm_rope(s["q"], s["wq"], pos, c["rotary"]), _norm_rope(s["k"], s["wk"], pos, c["rotary"])


def _plain_append(s):
    c = s["c"]
    pos, at = s["first"] + s["plan"]["depth"], slice(c["rows"], c["rows"] + c["n"])
    s["k_cache"][at] = _norm_rope(s["k"], s["wk"], pos, c["rotary"])
    s["v_cache"][at] = s["v"]
    return _norm_rope(s["q"], s["wq"], pos, c["rotary"]), s["k_cache"][at], s["v_cache"][at]


def _plain_attn(s):
    c = s["c"]
    n, rows, G = c["n"], c["rows"], c["hq"] // c["hkv"]
    q = s["q_hat"].float().view(n, c["hkv"], G, c["dim"]).permute(1, 0, 2, 3).reshape(c["hkv"], n * G, c["dim"])
    k = s["k_cache"][:rows + n].float().permute(1, 2, 0).contiguous()
    v = s["v_cache"][:rows + n].float().permute(1, 0, 2).contiguous()
    z = (q @ k).view(c["hkv"], n, G, rows + n) * c["dim"] ** -0.5
    z[..., rows:].masked_fill_(~s["plan"]["seen"][None, :, None, :], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    o = (p.view(c["hkv"], n * G, rows + n) @ v).view(c["hkv"], n, G, c["dim"]) / p.sum(-1, keepdim=True)
    return o.permute(1, 0, 2, 3).reshape(n, c["hq"], c["dim"]).to(torch.bfloat16)


def _plain_conv(s):
    out = []
    for state, x, w, _ in s["conv"]:
        rows = torch.cat([state, x]).float()[s["plan"]["taps"]]       # [n, width, channels]
        y = (rows * w.float().t()).sum(1)
        out.append((y * torch.sigmoid(y) if s["c"]["silu"] else y).to(torch.bfloat16))
    return out


def _pseudo(S, k, v, beta, g, seen):
    """The pseudo-values u of nodes along their paths and the decays between them, in 64 bits:
    u_i = beta_i (v_i - gamma_i S k_i) - sum_{j before i} beta_i (gamma_i / gamma_j) (k_i . k_j) u_j.
    S [.., h, dv, dk], k [.., h, n, dk], v [.., h, n, dv], beta, g [.., h, n]."""
    lg = (seen.double() @ g.double().log().unsqueeze(-1)).squeeze(-1)                 # log of gamma
    ratio = torch.where(seen, (lg.unsqueeze(-1) - lg.unsqueeze(-2)), -math.inf).exp()
    M = beta.unsqueeze(-1) * ratio * (k @ k.transpose(-1, -2).contiguous())
    M = M - torch.diag_embed(M.diagonal(dim1=-2, dim2=-1))
    b = beta.unsqueeze(-1) * (v - lg.exp().unsqueeze(-1) * (k @ S.transpose(-1, -2).contiguous()))
    eye = torch.eye(k.shape[-2], device=DEV, dtype=torch.float64)
    return torch.linalg.solve_triangular(eye + M, b, upper=False), ratio, lg


def _plain_delta(s):
    c = s["c"]
    G = c["hv"] // c["hk"]
    q, k = (s[x].double().permute(1, 0, 2).repeat_interleave(G, 0) for x in ("q", "k"))
    S, v, beta, g = s["state"].double(), s["v"].double().permute(1, 0, 2), s["beta"].double().t(), s["g"].double().t()
    u, ratio, lg = _pseudo(S, k, v, beta, g, s["plan"]["seen"])
    o = lg.exp().unsqueeze(-1) * (q @ S.transpose(-1, -2).contiguous()) + (ratio * (q @ k.transpose(-1, -2).contiguous())) @ u
    return (c["d"] ** -0.5 * o).permute(1, 0, 2).float().contiguous()


def _plain_verify(s):
    c, plan = s["c"], s["plan"]
    n, V = c["n"], c["vocab"]
    p, u = s["target"].double(), s["u"].double()
    q = s["proposal"].double() if c["drawn"] else None
    node, tokens = torch.arange(n, device=DEV), s["tokens"].long()
    beta, total = torch.zeros(n, device=DEV, dtype=torch.float64), torch.ones(n, device=DEV, dtype=torch.float64)
    chosen, left = torch.full((n,), -1, device=DEV), p
    for kid in plan["kids"]:      # the children of a node are tried one after the other
        has = (kid >= 0) & (chosen < 0)
        x = tokens[kid.clamp(min=0)]
        px, qx = left[node, x], q[node, x] if c["drawn"] else 1.0
        yes = has & (u[kid.clamp(min=0)] * qx * total < px)
        chosen, no = torch.where(yes, kid, chosen), has & ~yes
        if c["drawn"]:            # what is left of the target: max(p - beta q, 0), unnormalised
            beta = torch.where(no, beta + total, beta)
            left = (p - beta[:, None] * q).clamp(min=0)
        else:
            left = torch.where(no[:, None] & (torch.arange(V, device=DEV) == x[:, None]), 0.0, left)
        total = torch.where(no, left.sum(-1), total)
    took = chosen[plan["parents"]] == node
    took[0] = True
    on = (plan["seen"] & ~took).sum(1) == 0
    path, last = torch.where(on, node, n).sort().values, torch.where(on, node, 0).max()
    row = left[last]
    row = torch.where(row.sum() > 0, row, p[last])
    cdf = row.cumsum(0)
    nxt = torch.searchsorted(cdf, (u[0] * cdf[-1]).view(1), right=True)
    return torch.cat([on.sum().view(1), nxt, torch.where(path < n, path, -1)]).to(torch.int32)


def _plain_accept(s):
    c, path, rows = s["c"], s["path_d"], s["c"]["rows"]
    a = path.numel()
    s["kv"][:, :, rows:rows + a] = s["kv"][:, :, rows + path]
    if c["n_delta"]:
        G = c["hv"] // c["hk"]
        k = s["k"][:, path].double().permute(0, 2, 1, 3).repeat_interleave(G, 1)
        v = s["v"][:, path].double().permute(0, 2, 1, 3)
        beta, g = (s[x][:, path].double().permute(0, 2, 1) for x in ("beta", "g"))
        S = s["S"].double()
        u, ratio, lg = _pseudo(S, k, v, beta, g, torch.ones((a, a), dtype=torch.bool, device=DEV).tril())
        keep = ratio[..., -1, :].unsqueeze(-1) * k
        s["S"].copy_(lg[..., -1].exp()[..., None, None] * S + u.transpose(-1, -2).contiguous() @ keep)
        s["cs"].copy_(torch.cat([s["cs"], s["cx"][:, path]], 1)[:, a:])
    return _kept(s)


_PLAIN = {"norm": _plain_norm, "append": _plain_append, "attn": _plain_attn, "conv": _plain_conv,
          "delta": _plain_delta, "verify": _plain_verify, "accept": _plain_accept}


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(c):
    kind, n = c["kind"], c.get("n", 0)
    if kind in ("norm", "append"):
        T = c["T"] if kind == "norm" else n
        heads = c["hq"] + c["hkv"] * (1 if kind == "norm" else 2)
        return {"bytes": 4 * T * heads * c["dim"] + 4 * c["dim"], "flops": 8 * T * (c["hq"] + c["hkv"]) * c["dim"]}
    if kind == "attn":
        rows = c["rows"] + n
        return {"bytes": 4 * rows * c["hkv"] * c["dim"] + 4 * n * c["hq"] * c["dim"], "flops": 4 * rows * n * c["hq"] * c["dim"]}
    if kind == "conv":
        ch = c["cq"] + c["ck"] + c["cv"]
        return {"bytes": 2 * ch * (2 * n + 2 * c["width"] - 1), "flops": 2 * ch * n * c["width"]}
    if kind == "delta":
        d, state = c["d"], c["hv"] * c["d"] * c["d"]
        return {"bytes": 4 * state + n * (4 * c["hk"] * d + 6 * c["hv"] * d + 8 * c["hv"]),
                "flops": 4 * n * state + 2 * n * n * c["hv"] * 2 * d}
    if kind == "verify":   # at least the row that the next token is drawn from
        return {"bytes": 4 * c["vocab"] * (2 if c["drawn"] else 1) + 16 * n, "flops": 3 * c["vocab"]}
    d, a = c["d"], c["spine"]
    kv = 8 * c["n_attn"] * a * c["hkv"] * c["dim"]
    state = c["n_delta"] * c["hv"] * d * d
    ch = c["n_delta"] * (2 * c["hk"] + c["hv"]) * d
    return {"bytes": kv + 8 * state + c["n_delta"] * a * (2 * c["hk"] * d + 2 * c["hv"] * d + 8 * c["hv"]) +
            4 * ch * (c["width"] - 1), "flops": 6 * a * state}


# ----------------------------------------------------------------------------- 64-bit results, from the definitions

def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind in ("norm", "append"):
        T = c["T"] if kind == "norm" else c["n"]
        steps = torch.arange(T, device=DEV) if kind == "norm" else _depths(s["parents"])
        pos = (s["first"] + steps).double()
        q, k = (_exact_norm(s[x], s[w], pos, c["rotary"]) for x, w in (("q", "wq"), ("k", "wk")))
        return (q, k) if kind == "norm" else (q, k, s["v"].double())
    if kind == "attn":
        return _exact_attn(s)
    if kind == "conv":
        return [_exact_conv(s["parents"], *item[:3], c) for item in s["conv"]]
    if kind == "delta":
        return _exact_delta(s)
    if kind == "verify":
        return None
    kv = s["kv"][:, :, [c["rows"] + i for i in s["path"]]].double()
    S = s["S"].double()
    for i in s["path"] if c["n_delta"] else []:
        S = _exact_step(S, s["k"][:, i], s["v"][:, i], s["beta"][:, i], s["g"][:, i])[0]
    cs = torch.cat([s["cs"], s["cx"][:, s["path"]]], 1)[:, len(s["path"]):].double()
    return kv, S, cs


def _depths(parents):
    d = []
    for p in parents:
        d.append(d[p] + 1 if p >= 0 else 0)
    return torch.tensor(d, device=DEV)


def _exact_norm(x, w, pos, rotary):
    x = x.double()
    x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
    y, half = x.clone(), rotary // 2
    for j in range(half):
        ang = (pos * math.pow(THETA, -2.0 * j / rotary))[:, None]
        y[..., j] = x[..., j] * ang.cos() - x[..., j + half] * ang.sin()
        y[..., j + half] = x[..., j + half] * ang.cos() + x[..., j] * ang.sin()
    return y


def _exact_attn(s):
    c = s["c"]
    n, rows, G = c["n"], c["rows"], c["hq"] // c["hkv"]
    out = torch.zeros((n, c["hq"], c["dim"]), dtype=torch.float64, device=DEV)
    lines = []
    for i in range(n):
        line, at = [], i
        while at >= 0:
            line.append(rows + at)
            at = s["parents"][at]
        lines.append(torch.tensor(line, device=DEV))
    for h in range(c["hq"]):
        K, V = (s[x][:rows + n, h // G].double() for x in ("k_cache", "v_cache"))
        q = s["q_hat"][:, h].double() * c["dim"] ** -0.5
        z = q @ K[:rows].t().contiguous()
        for i in range(n):
            zi = torch.cat([z[i], K[lines[i]] @ q[i]])
            p = torch.softmax(zi, 0)
            out[i, h] = p[:rows] @ V[:rows] + p[rows:] @ V[lines[i]]
    return out


def _exact_conv(parents, state, x, w, c):
    W, y = c["width"], torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    for i in range(c["n"]):
        at, back = i, W - 2          # back: the state row that comes next once the path is behind us
        for t in range(W - 1, -1, -1):
            if at >= 0:
                y[i] += w[:, t].double() * x[at].double()
                at = parents[at]
            else:
                y[i] += w[:, t].double() * state[back].double()
                back -= 1
    return y / (1 + torch.exp(-y)) if c["silu"] else y


def _exact_step(S, k, v, beta, g):
    """One token of S <- g S (I - beta k k^T) + beta v k^T; heads in the third dimension from the end."""
    k = k.double().repeat_interleave(v.shape[-2] // k.shape[-2], -2)
    b, g = beta.double()[..., None, None], g.double()[..., None, None]
    Sk = (S * k.unsqueeze(-2)).sum(-1, keepdim=True)
    return g * (S - b * Sk * k.unsqueeze(-2)) + b * v.double().unsqueeze(-1) * k.unsqueeze(-2), k


def _exact_delta(s):
    c, states = s["c"], []
    out = torch.zeros((c["n"], c["hv"], c["d"]), dtype=torch.float64, device=DEV)
    for i, p in enumerate(s["parents"]):
        S, _ = _exact_step(states[p] if p >= 0 else s["state"].double(), s["k"][i], s["v"][i], s["beta"][i], s["g"][i])
        states.append(S)
        q = s["q"][i].double().repeat_interleave(c["hv"] // c["hk"], 0)
        out[i] = c["d"] ** -0.5 * (S * q[:, None, :]).sum(-1)
    return out

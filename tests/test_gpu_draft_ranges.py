"""Speculative decoding on the GPU beyond the single calls: batches that change the launches'
shape, stacks of several launches, calls beside each other, drawn shapes, and what the other
calls of the package read of an accepted path."""
import threading

import numpy as np
import pytest
import torch

import paper_2609_18935_amd as tu
from oracle import draft as O
from draft_cases import BF16, F32, bf16, delta_inputs, drafted, f64, rows_of, tree, worst
from test_gpu_draft import DEV, THETA, _attn, _ctx, _delta_bound, _norm_bound, _step, _step_setup, _verify, _want, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,D,rotary", [(3, 1, 64, 64), (2, 2, 128, 32), (5, 1, 256, 256), (1, 1, 64, 6)])
@pytest.mark.parametrize("T", [255, 1025, 2049, 2051, 6145, 6147])     # 1, 2 and 4 tokens a workgroup, the last one short
def test_norm_of_many_tokens(hq, hkv, D, rotary, T):
    rng = np.random.default_rng([hq, D, T])
    q, k, w = bf16(rng, T, hq, D, scale=2.0), bf16(rng, T, hkv, D), bf16(rng, D)
    qo, ko = (torch.full((T + 1, h, D), 9.0, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
    tu.qk_norm_rope(tu.attn_params(hq, hkv, D, rotary, THETA), dev(q), dev(k), qo[:T], ko[:T],
                    norm=tu.QkNorm("rms", 1e-6, dev(w), dev(w)), first_pos=1000)
    pos, eps = 1000 + np.arange(T), np.float64(np.float32(1e-6))
    for got, src in ((qo, q), (ko, k)):
        want = O.qk_norm_rope(f64(src), pos, rotary, THETA, "rms", eps, f64(w), 0.0)
        assert worst(got[:T], want, _norm_bound(f64(src), want, "rms", f64(w), 0.0, D)) <= 1
        assert (got[T] == 9).all()


@pytest.mark.parametrize("hq,hkv,D", [(16, 4, 64), (32, 8, 128), (12, 3, 128)])
@pytest.mark.parametrize("splits", [1, 2, 5, 64])
def test_attention_splits_of_narrow_heads(hq, hkv, D, splits):
    out, want, bound, _ = _attn(hq, hkv, D, 419, tree("tree", 50), splits=splits)
    assert worst(out, want, bound) <= 1


@pytest.mark.parametrize("seed", range(16))
def test_attention_of_drawn_shapes(seed):
    rng = np.random.default_rng([77, seed])
    D, hkv = int(rng.choice([64, 128, 256])), int(rng.integers(1, 6))
    hq = hkv * int(rng.integers(1, 6))
    n, rows = int(rng.integers(1, 129)), int(rng.choice([0, 1, 31, 32, 33, 63, 64, 65, 127, 400, 777]))
    kind = str(rng.choice(["chain", "star", "roots", "forest", "tree"]))
    print(f"[case] {hq}/{hkv}x{D} n={n} rows={rows} {kind}", flush=True)
    out, want, bound, ws = _attn(hq, hkv, D, rows, tree(kind, n, seed), seed=seed, splits=int(rng.choice([0, 0, 1, 3, 40])))
    assert worst(out, want, bound) <= 1
    assert tu.workspace_faults(ws) == 0


@pytest.mark.parametrize("seed", range(12))
def test_delta_rule_of_drawn_shapes(seed):
    rng = np.random.default_rng([78, seed])
    d, Hk = int(rng.choice([64, 128])), int(rng.integers(1, 5))
    Hv, n = Hk * int(rng.integers(1, 4)), int(rng.integers(1, 129))
    kind = str(rng.choice(["chain", "star", "roots", "forest", "tree"]))
    print(f"[case] {Hk}-{Hv}/{d} n={n} {kind}", flush=True)
    parents, c = tree(kind, n, seed), delta_inputs(rng, n, Hk, Hv, d)
    x = {k: dev(t) for k, t in c.items()}
    out = torch.full((n + 1, Hv, d), 7.0, device=DEV)
    tu.draft_delta_rule(x["state"], x["q"], x["k"], x["v"], x["beta"], x["g"], tu.delta_params(Hk, Hv, d, d, 64),
                        tu.Draft(parents), out[:n])
    want = O.draft_delta_rule(f64(c["state"]), *[f64(c[k]) for k in ("q", "k", "v", "beta", "g")], parents, d ** -0.5)
    assert worst(out[:n], want, _delta_bound(f64(c["state"]), c, parents, d ** -0.5, d, n)) <= 1
    assert (out[n] == 7).all() and torch.equal(x["state"].cpu(), c["state"])


def test_accept_of_more_layers_than_a_launch_takes():
    rng = np.random.default_rng(9)
    n, rows, path, hkv, D, d, W = 7, 11, [0, 2, 4, 6], 1, 64, 64, 3
    parents = [-1, 0, 0, 1, 2, 1, 4]
    n_attn, n_delta = 35, 101
    kv = bf16(rng, 2 * n_attn, rows + n, hkv, D)
    kvd = dev(kv)
    cs = [delta_inputs(rng, n, 1, 1, d) for _ in range(n_delta)]
    xs = [{k: dev(t) for k, t in c.items()} for c in cs]
    conv = [(bf16(rng, W - 1, 8 * (1 + i % 3)), bf16(rng, n, 8 * (1 + i % 3))) for i in range(n_delta)]
    cd = [(dev(a), dev(b)) for a, b in conv]
    attn = [tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[kvd[2 * l]], v_cache=[kvd[2 * l + 1]])
            for l in range(n_attn)]
    delta = [tu.LayerIO(tu.TU_LAYER_DELTA, None, x["k"], x["v"], None, state=[x["state"]], beta=x["beta"], g=x["g"])
             for x in xs]
    layers = [L for pair in zip(delta, attn) for L in pair] + delta[n_attn:]     # mixed, a tail of one kind
    ctx = _ctx(rows, n, 50)
    tu.draft_accept(ctx, tu.Draft(parents), path, tu.DraftStack(layers, tu.attn_params(1, 1, D), tu.delta_params(1, 1, d, d, 64), cd))
    a = len(path)
    assert torch.equal(kvd.cpu()[:, rows:rows + a], kv[:, [rows + i for i in path]])
    assert torch.equal(kvd.cpu()[:, :rows], kv[:, :rows])
    assert ctx.pos[rows:rows + a].tolist() == [50, 51, 52, 53] and ctx.len == rows + a
    for c, x in zip(cs, xs):
        S, M = f64(c["state"]), np.abs(f64(c["state"]))
        for i in path:
            step = [f64(c[k][i]) for k in ("k", "v", "beta", "g")]
            S, M = O.delta_step(S, *step), O.delta_step(M, *[np.abs(t) for t in step], sign=1.0)
        assert worst(x["state"], S, (d + 8) * a * F32 * M) <= 1
    for (st, x), (sd, _) in zip(conv, cd):
        assert torch.equal(sd.cpu(), torch.cat([st, x[path]])[-(W - 1):])


def test_conv_of_more_tensors_than_a_launch_takes():
    rng = np.random.default_rng(10)
    n, W = 9, 4
    parents = tree("tree", n)
    items = [(bf16(rng, W - 1, C), bf16(rng, n, C), bf16(rng, C, W)) for C in [8 * (1 + i % 5) for i in range(37)]]
    outs = [torch.zeros(n, x.shape[1], dtype=torch.bfloat16, device=DEV) for _, x, _ in items]
    tu.draft_short_conv(tu.Draft(parents), [(*map(dev, it), o) for it, o in zip(items, outs)], "none")
    for (st, x, w), o in zip(items, outs):
        want, mag = O.draft_short_conv(f64(st), f64(x), f64(w), parents, False)
        assert worst(o, want, BF16 * np.abs(want) + 2 * W * F32 * mag) <= 1


def test_steps_of_two_contexts_beside_each_other():
    """Two streams, each with its own context, tensors and workspaces, their calls interleaved."""
    setups = [_step_setup(2), _step_setup(3, rows=901, n=60)]
    want = [_step(s) for s in setups]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in setups]
    for _ in range(8):
        got = []
        for s, st in zip(setups, streams):
            with torch.cuda.stream(st):
                got.append(_step(s))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_a_stream_given_by_name():
    s = _step_setup(4)
    want = _step(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for t in (s["o"], s["od"], s["result"]):
        t.zero_()
    torch.cuda.synchronize()
    _step(s, stream=side)              # its copies of the results are made on the current stream: not used
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((s["o"], s["od"], s["result"]), want))


def test_an_accepted_path_under_an_update_with_a_vt_copy():
    """A context whose value cache has a V^T copy decodes a draft and keeps a path; the next
    stack update (a removal and a tail) reads the accepted rows as one without the copy does."""
    hq, hkv, D, rows, n, T = 16, 2, 256, 700, 21, 90
    rng = np.random.default_rng(12)
    parents, path = tree("tree", n), [0]
    while any(p == path[-1] for p in parents):
        path.append(max(i for i, p in enumerate(parents) if p == path[-1]))
    cap = rows + n + T
    kv, qkv, tail = bf16(rng, 2, cap, hkv, D), bf16(rng, n, hq + 2 * hkv, D), bf16(rng, T, hq + 2 * hkv, D)
    p = tu.attn_params(hq, hkv, D, 64, THETA)
    got = []
    for copy in (False, True):
        kc, vc = dev(kv)
        ctx = _ctx(rows, n, rows, spare=T)
        ctx.pos[:rows] = torch.arange(rows, dtype=torch.int32, device=DEV)
        vt = None
        if copy:
            vt = tu.new_vt_cache(cap, hkv, D, DEV)
            tu.refresh_vt_cache(ctx, [vc], [vt])
            assert ctx.vt_rows == rows
        x = dev(qkv)
        draft, q_hat = tu.Draft(parents), torch.zeros(n, hq, D, dtype=torch.bfloat16, device=DEV)
        tu.draft_append(ctx, kc, vc, p, draft, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q_hat)
        layer = tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[kc], v_cache=[vc])
        tu.draft_accept(ctx, draft, path, tu.DraftStack([layer], p))
        t = dev(tail)
        q, k, v = t[:, :hq].contiguous(), t[:, hq:hq + hkv].contiguous(), t[:, hq + hkv:].contiguous()
        out = torch.zeros(T, hq, D, device=DEV)
        up = tu.LayerIO(tu.TU_LAYER_ATTN, q, k, v, out, k_cache=[kc], v_cache=[vc], vt_cache=[vt] if copy else None)
        tu.update_layer_stack([ctx], [np.array([[650, 660]])], [T], [up], p)
        got.append((out, kc[:ctx.len], vc[:ctx.len], ctx.pos[:ctx.len], ctx.intervals()))
    assert len(path) > 2
    for a, b in zip(*got):
        assert a == b if isinstance(a, list) else torch.equal(a, b)
    out, kc, _, pos, runs = got[0]
    assert runs == [(0, 650), (660, rows + len(path) + T)] and pos.tolist() == [*range(650), *range(660, runs[-1][1])]
    K, V = f64(kc), f64(got[0][2])
    L = len(K) - T
    qh = O.qk_norm_rope(f64(tail[:, :hq]), rows + len(path) + np.arange(T), 64, THETA)
    qh = f64(torch.from_numpy(qh).to(torch.bfloat16))
    want, _, _ = O.draft_attention(qh, K, V, [i - 1 for i in range(T)], D ** -0.5)
    assert np.abs(f64(out) - want).max() <= 2e-2 and L == rows - 10 + len(path)


@pytest.mark.parametrize("seed", range(8))
def test_verify_of_drawn_trees(seed):
    """Large trees over small vocabularies (every kind of walk: several rejections, duplicates)."""
    rng = np.random.default_rng([79, seed])
    n, V = int(rng.integers(1, 129)), int(rng.choice([2, 3, 8, 40, 700, 5000]))
    parents = tree(str(rng.choice(["chain", "star", "tree"])), n, seed)
    target, proposal = rows_of(rng, n, V, 1.0), rows_of(rng, n, V, 1.0)
    for drawn in (True, False):
        tok = drafted(rng, parents, proposal, distinct=not drawn)
        for _ in range(6):
            u = rng.random(n).astype(np.float32)
            assert _verify(parents, tok, target, u, proposal if drawn else None) == \
                _want(parents, tok, target, u, proposal if drawn else None)


def test_offsets_beyond_32_bits():
    """A cache of more than 2 GB a buffer: append, attention in one split if the split could, acceptance."""
    hkv, D, rows, n = 32, 256, 150_000, 3
    g = torch.Generator(device=DEV).manual_seed(5)
    kc, vc = (torch.empty(rows + n, hkv, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    assert kc.numel() * 2 > 2 ** 31
    qkv = torch.randn(n, 3 * hkv, D, device=DEV, generator=g).to(torch.bfloat16)
    p = tu.attn_params(hkv, hkv, D, 0, kv_splits=1)
    ctx, draft = _ctx(rows, n), tu.Draft([-1, 0, 0])
    q_hat, out = torch.zeros(2, n, hkv, D, dtype=torch.bfloat16, device=DEV)
    tu.draft_append(ctx, kc, vc, p, draft, qkv[:, :hkv], qkv[:, hkv:2 * hkv], qkv[:, 2 * hkv:], q_hat)
    assert torch.equal(q_hat, qkv[:, :hkv]) and torch.equal(kc[rows:], qkv[:, hkv:2 * hkv]) and torch.equal(vc[rows:], qkv[:, 2 * hkv:])
    ws = tu.draft_attention(ctx, kc, vc, p, draft, q_hat, out)
    assert ws.numel() > 256 and tu.workspace_faults(ws) == 0          # two splits: one's rows would span 2 GB
    for i, see in ((0, [0]), (2, [0, 2])):
        rowset = torch.cat([torch.arange(rows), rows + torch.tensor(see)]).to(DEV)
        for h in (0, 17, 31):
            pr = torch.softmax(kc[rowset, h].double() @ q_hat[i, h].double() / 16, 0)
            V = vc[rowset, h].double()
            want, mag = pr @ V, pr @ V.abs()
            err = (out[i, h].double() - want).abs()
            # output rounding; P and partial outputs in f16, P's subnormals; fp32 scores (|q| |k| <= 20 here) and exponentials
            assert (err <= BF16 * want.abs() + (2 * 2.0 ** -11 + 2 * (264 * F32 * 20 + 16 * F32)) * mag + 2.0 ** -18).all()
    layer = tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[kc], v_cache=[vc])
    tu.draft_accept(ctx, draft, [0, 2], tu.DraftStack([layer], p))
    assert torch.equal(kc[rows + 1], qkv[2, hkv:2 * hkv]) and torch.equal(vc[rows + 1], qkv[2, 2 * hkv:])
    assert ctx.pos[rows:rows + 2].tolist() == [rows, rows + 1]


def test_probability_rows_that_lie_far_apart():
    rng = np.random.default_rng(6)
    V, step, parents = 700, 1 << 30, [-1, 0, 0]
    target = rows_of(rng, 3, V, 1.0)
    far = torch.empty(2 * step + V, device=DEV).as_strided((3, V), (step, 1))
    far.copy_(torch.from_numpy(target))
    tok = drafted(rng, parents, target, distinct=True)
    for s in range(4):
        u = np.random.default_rng(s).random(3).astype(np.float32)
        got = tu.draft_verify(tu.Draft(parents), torch.from_numpy(tok).to(DEV), far, torch.from_numpy(u).to(DEV))
        assert got.tolist() == _want(parents, tok, target, u)


def test_steps_from_two_threads():
    setups = [_step_setup(5), _step_setup(6, rows=77, n=40)]
    want = [_step(s) for s in setups]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                got = _step(setups[i])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_kernel_times_carry_the_calls_names():
    s = _step_setup(7)
    tu.profile_enable(True)
    try:
        _step(s)
        names = set(tu.profile_collect())
    finally:
        tu.profile_enable(False)
    assert {"qk_norm_rope", "draft_attention", "draft_merge", "draft_conv", "draft_delta", "draft_verify"} <= names


@pytest.mark.parametrize("hq,hkv,D,rows,n", [(16, 2, 256, 40000, 64), (16, 2, 256, 40000, 27), (16, 2, 256, 30000, 40),
                                             (32, 8, 128, 25000, 61), (16, 4, 64, 60000, 128), (8, 1, 64, 50000, 33)])
def test_attention_with_many_rows_a_workgroup(hq, hkv, D, rows, n):
    """Long caches, where a workgroup takes five to eight waves of rows."""
    parents = tree("tree", n, 3)
    g = torch.Generator(device=DEV).manual_seed(n)
    k, v = torch.randn(2, rows + n, hkv, D, device=DEV, generator=g).to(torch.bfloat16)
    q = torch.randn(n, hq, D, device=DEV, generator=g).to(torch.bfloat16)
    out = torch.full((n + 1, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    tu.draft_attention(_ctx(rows, n), k, v, tu.attn_params(hq, hkv, D), tu.Draft(parents), q, out[:n])
    assert (out[n] == 7).all()
    for i in (0, n // 2, n - 1):
        see = torch.cat([torch.arange(rows), rows + torch.tensor(O.line(parents, i))]).to(DEV)
        for h in range(hq):
            pr = torch.softmax(k[see, h * hkv // hq].double() @ q[i, h].double() * D ** -0.5, 0)
            V = v[see, h * hkv // hq].double()
            want, mag = pr @ V, pr @ V.abs()
            err = (out[i, h].double() - want).abs()
            # as over 150,000 rows above
            assert (err <= BF16 * want.abs() + (2 * 2.0 ** -11 + 2 * ((D + 8) * F32 * 20 + 16 * F32)) * mag + 2.0 ** -18).all()

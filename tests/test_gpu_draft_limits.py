"""Speculative decoding on the GPU at the limits of its inputs, against the float64 definitions: rows
behind a short split, scores far apart, queries that are not finite, a kept workspace,
waits that expire."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2609_18935_amd as tu
from oracle import draft as O
from paper_2609_18935_amd import binding as B
from draft_cases import BF16, F16, F32, bf16, f64, rows_of, tree, worst
from test_gpu_draft import DEV, _attn, _ctx, _want, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,D,rows,n,splits", [(16, 2, 256, 0, 1, 0), (16, 2, 256, 2976, 1, 0), (16, 2, 256, 65, 3, 3),
                                                    (8, 2, 128, 0, 1, 0), (8, 2, 128, 0, 7, 1), (8, 2, 128, 130, 1, 3),
                                                    (16, 4, 64, 0, 1, 0), (16, 4, 64, 130, 1, 3)])
def test_attention_ignores_rows_behind_a_split_shorter_than_a_stage(hq, hkv, D, rows, n, splits):
    """The last split (or the only one) holds fewer rows than one load of a workgroup takes (16 of 256 dims, 32 of
    128): the rows behind it, which belong to no node, are not read as values."""
    rng = np.random.default_rng([D, rows, n])
    spare = 160
    kv = bf16(rng, 2, rows + n + spare, hkv, D)
    kv[:, rows + n:] = float("nan")
    out, want, bound, _ = _attn(hq, hkv, D, rows, tree("tree", n), kv=kv, spare=spare, splits=splits)
    assert worst(out, want, bound) <= 1


@pytest.mark.parametrize("hq,hkv,D", [(16, 2, 256), (8, 2, 128), (16, 4, 64)])
@pytest.mark.parametrize("rows,splits", [(4000, 1), (4000, 0), (700, 1), (12000, 3)])
@pytest.mark.parametrize("gap", [14.0, 16.0, 17.5, 18.0])
def test_attention_beside_a_sink(hq, hkv, D, rows, splits, gap):
    """The first key's score lies `gap` above all others' (in units of e) and its value is zero: the output is what
    the many small probabilities leave."""
    rng = np.random.default_rng([D, rows, int(2 * gap)])
    n = 5
    k, v = bf16(rng, 2, rows + n + 3, hkv, D)
    q = bf16(rng, n, hq, D, scale=0.5)
    k[..., 0], q[..., 0] = 0, gap * D ** 0.5 / 8
    k[0], k[0, :, 0] = 0, 8
    v = v.abs()
    v[0] = 0
    parents = tree("tree", n)
    out = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = tu.draft_attention(_ctx(rows, n, spare=3), dev(k), dev(v), tu.attn_params(hq, hkv, D, kv_splits=splits), tu.Draft(parents),
                            dev(q), out)
    want, mag, most = O.draft_attention(f64(q), f64(k)[:rows + n], f64(v)[:rows + n], parents, D ** -0.5)
    assert want.max() < 2e-2 and want.min() > 1e-6
    # the output's rounding; P and the partial outputs in f16; the scores' fp32 sums and the exponential, in numerator and
    # denominator. Below f16's normal range: P, at most 2^-25 of 2^11 times the largest key's; partial outputs, 2^-25
    bound = BF16 * np.abs(want) + (2 * F16 + 2 * ((D + 8) * F32 * most[..., None] + 16 * F32)) * mag + \
        2.0 ** -36 * (rows + n) * f64(v).max() + 2.0 ** -25
    assert worst(out, want, bound) <= 1
    assert tu.workspace_faults(ws) == 0


@pytest.mark.parametrize("hq,hkv,D", [(16, 2, 256), (8, 2, 128), (16, 4, 64)])
@pytest.mark.parametrize("exponent", [10, 12, 13, 14, 15])
@pytest.mark.parametrize("splits", [1, 4])
def test_attention_of_scores_of_millions(hq, hkv, D, exponent, splits):
    """Scores up to 2^27 that rise from key to key by far more than any rounding: the last cached key takes all."""
    rows, n, rng = 300, 3, np.random.default_rng(exponent)
    k, v = torch.zeros(rows + n, hkv, D, dtype=torch.bfloat16), bf16(rng, rows + n, hkv, D)
    q = torch.zeros(n, hq, D, dtype=torch.bfloat16)
    q[..., 0] = 2.0 ** exponent
    k[:rows, :, 0] = ((1 + torch.arange(rows) % 128 / 128) * 2.0 ** (exponent + torch.arange(rows) // 128 - 2)).to(torch.bfloat16)[:, None]
    out = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    tu.draft_attention(_ctx(rows, n), dev(k), dev(v), tu.attn_params(hq, hkv, D, kv_splits=splits), tu.Draft([-1, 0, 0]), dev(q), out)
    want = f64(v)[rows - 1].repeat(hq // hkv, axis=0)[None].repeat(n, axis=0)
    steps = np.diff(f64(k)[:rows, 0, 0]) * 2.0 ** exponent * D ** -0.5
    assert (steps > 0).all() and steps[-1] > 500       # exp(-500) is nothing
    # P and the partial output in f16, the sum of P in fp32, the output in bf16
    assert worst(out, want, (BF16 + 2 * F16 + 4 * F32) * np.abs(want)) <= 1


@pytest.mark.parametrize("hq,hkv,D,rows,n,splits", [(16, 2, 256, 0, 1, 0), (16, 2, 256, 40, 9, 1), (16, 2, 256, 900, 9, 0),
                                                    (8, 2, 128, 40, 9, 1), (8, 2, 128, 500, 9, 4), (16, 4, 64, 0, 1, 0),
                                                    (16, 4, 64, 300, 9, 1)])
def test_attention_of_queries_that_are_not_finite(hq, hkv, D, rows, n, splits):
    """Scores of -infinity alone, of both infinities, and NaN: softmax is NaN in each, whatever the splits, and
    the other queries do not notice."""
    rng = np.random.default_rng([D, rows])
    k, v = bf16(rng, 2, rows + n + 3, hkv, D)
    q, parents = bf16(rng, n, hq, D), tree("tree", n)
    k[..., 3] = 1
    clean, last = q.clone(), n - 1
    q[last, 0, 3], q[last, 1, 3], q[last, hq - 1, 5] = -float("inf"), float("inf"), float("nan")
    out = torch.full((n, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    tu.draft_attention(_ctx(rows, n, spare=3), dev(k), dev(v), tu.attn_params(hq, hkv, D, kv_splits=splits), tu.Draft(parents),
                       dev(q), out)
    want, mag, most = O.draft_attention(f64(clean), f64(k)[:rows + n], f64(v)[:rows + n], parents, D ** -0.5)
    want[last, [0, 1, hq - 1]] = np.nan
    bound = BF16 * np.abs(want) + (2 * F16 + 2 * ((D + 8) * F32 * most[..., None] + 16 * F32)) * mag + 2.0 ** -25
    assert worst(out, want, bound) <= 1


def test_a_workspace_kept_over_steps_of_other_sizes():
    hq, hkv, D, rng = 16, 2, 256, np.random.default_rng(8)
    p = tu.attn_params(hq, hkv, D)
    ws = torch.empty(tu.draft_attention_workspace_bound(p, 40, 2200), dtype=torch.uint8, device=DEV)
    for rows, n in ((2200, 40), (2100, 24), (2150, 24), (31, 40), (700, 1)):
        k, v = bf16(rng, 2, rows + n, hkv, D)
        q, parents = bf16(rng, n, hq, D), tree("tree", n)
        out = torch.zeros(n, hq, D, dtype=torch.bfloat16, device=DEV)
        tu.draft_attention(_ctx(rows, n), dev(k), dev(v), p, tu.Draft(parents), dev(q), out, workspace=ws)
        want, mag, most = O.draft_attention(f64(q), f64(k), f64(v), parents, D ** -0.5)
        bound = BF16 * np.abs(want) + (2 * F16 + 2 * ((D + 8) * F32 * most[..., None] + 16 * F32)) * mag + 2.0 ** -25
        assert worst(out, want, bound) <= 1 and tu.workspace_faults(ws) == 0


def _record(name):
    """The launch record `name` as the library's headers declare it."""
    src = ""
    for header in ("common.h", "draft.h"):
        with open(os.path.join(os.path.dirname(tu.__file__), "csrc", header)) as f:
            src += f.read()
    body = re.search(r"struct %s \{\n(.*?)\n\};" % name, src, re.S).group(1)
    assert "constexpr int kMaxDraft = 128;" in src and "struct DraftMasks {\n  uint64_t m[kMaxDraft][2];\n};" in src
    assert "struct CallStatus {\n  unsigned long long* word;\n  uint32_t* last;\n  uint32_t call;\n  uint32_t pad;\n};" in src

    class CallStatus(ctypes.Structure):
        _fields_ = [("word", ctypes.c_void_p), ("last", ctypes.c_void_p), ("call", ctypes.c_uint32)]

    plain = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "uint64_t": ctypes.c_uint64, "uint8_t": ctypes.c_uint8,
             "CallStatus": CallStatus, "DraftMasks": ctypes.c_uint64 * 2 * 128}
    fields = []
    for line in body.splitlines():
        kind, star, field, count = re.fullmatch(r"\s*(?:const )?([\w ]+?)(\*?) (\w+)(?:\[(\w+)\])?;.*", line).groups()
        t = ctypes.c_void_p if star else plain[kind]
        fields.append((field, t * (128 if count == "kMaxDraft" else int(count)) if count else t))
    return type(name, (ctypes.Structure,), {"_fields_": fields}), CallStatus


def test_a_verification_whose_waits_expire_leaves_no_half_result():
    """Each workgroup looks for the others' sums a few times only: those that come early give up, later ones see them
    all. The result is whole or empty, and empty only with TU_FAULT_WAIT."""
    V, lib = 300000, B.lib()
    target = rows_of(np.random.default_rng(20), 1, V)
    Args, CallStatus = _record("DraftVerifyArgs")
    x, t = torch.zeros(1, dtype=torch.int32, device=DEV), torch.from_numpy(target).to(DEV)
    ws = torch.zeros(tu.draft_verify_workspace_size(tu.Draft([-1]), V), dtype=torch.uint8, device=DEV)
    result = torch.zeros(3, dtype=torch.int32, device=DEV)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    us = np.linspace(0, 0.999, 25).astype(np.float32)
    want = [_want([-1], np.zeros(1, np.int32), target, u[None]) for u in us]
    seen = []
    for polls in (0, 1, 2, 3, 4, 6, 8, 12, 16):
        for i, u in enumerate(us):
            ud = torch.from_numpy(u[None]).to(DEV)
            a = Args(tokens=x.data_ptr(), target=t.data_ptr(), proposal=None, u=ud.data_ptr(), result=result.data_ptr(),
                     target_stride=V, proposal_stride=0, vocab=V, part=ws.data_ptr() + 256,
                     status=CallStatus(ws.data_ptr(), ws.data_ptr() + 64, 0xF0000000 + len(seen)), n=1, n_blocks=37,
                     slice=8192, wide=1, polls=polls)
            a.seen[0][0] = 1
            assert 36 * a.slice < V <= 37 * a.slice
            assert lib._ZN2tu18launch_draft_clearERKNS_15DraftVerifyArgsEP12ihipStream_t(ctypes.byref(a), stream) == 0
            assert lib._ZN2tu17launch_draft_drawERKNS_15DraftVerifyArgsEP12ihipStream_t(ctypes.byref(a), stream) == 0
            r, fault = result.tolist(), tu.workspace_faults(ws)
            seen.append((polls, r[0], fault))
            assert r == want[i] or (r == [0, -1, -1] and fault == tu.TU_FAULT_WAIT), (polls, float(u), r, fault)
    print("polls, whole results, whole ones beside an expired wait:",
          [(p, sum(s[1] for s in seen if s[0] == p), sum(s[1] for s in seen if s[0] == p and s[2])) for p in sorted({s[0] for s in seen})])

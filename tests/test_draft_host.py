"""What the speculative decoding calls refuse (host only: nothing is enqueued and no device
address is read), and what a refusal leaves."""
import ctypes

import pytest
import torch

import paper_2609_18935_amd as tu
from paper_2609_18935_amd import binding as B

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host addresses stand in for device addresses")
bf, f32 = torch.bfloat16, torch.float32
ATTN = tu.attn_params(4, 2, 64)
DELTA = tu.delta_params(2, 4, 64, 64, 16)


def _ctx(rows=10, capacity=20, cursor=50, live_cap=8):
    c = tu.Context(capacity, device="cpu", live_cap=live_cap)
    c.set_metadata([(0, rows)] if rows else [], cursor)
    return c


def _raises(code, call):
    with pytest.raises(tu.TailUpdateError) as e:
        call()
    assert e.value.code == code, e.value


def z(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


def test_trees():
    n = 3
    ok = (z(n, 4, 64), z(n, 4, 64))
    c = _ctx()
    kc = z(20, 2, 64)
    for parents in ([0, 0, 1], [-2, 0, 1], [-1, 1, 0], [-1, 0, 3]):
        d = tu.Draft(parents)
        ws = z(1 << 16, dtype=torch.uint8)
        _raises(B.TU_ERR_ARG, lambda: tu.draft_attention(c, kc, kc, ATTN, d, *ok, workspace=ws))
        _raises(B.TU_ERR_ARG, lambda: tu.draft_delta_rule(z(4, 64, 64, dtype=f32), z(3, 2, 64), z(3, 2, 64), z(3, 4, 64),
                                                          z(3, 4, dtype=f32), z(3, 4, dtype=f32), DELTA, d, z(3, 4, 64, dtype=f32)))
        _raises(B.TU_ERR_ARG, lambda: tu.draft_short_conv(d, [(z(1, 8), z(3, 8), z(8, 2), z(3, 8))]))
        _raises(B.TU_ERR_ARG, lambda: tu.draft_append(c, kc, kc, ATTN, d, z(3, 4, 64), z(3, 2, 64), z(3, 2, 64), ok[0]))
        _raises(B.TU_ERR_ARG, lambda: tu.draft_accept(c, d, [0], tu.DraftStack([])))
    big = tu.Draft([i - 1 for i in range(129)])
    _raises(B.TU_ERR_ARG, lambda: tu.draft_short_conv(big, [(z(1, 8), z(129, 8), z(8, 2), z(129, 8))]))
    assert B.lib().draft_attention_workspace_size(ctypes.byref(ATTN), 129, 10) == 0
    assert (c.len, c.next_pos) == (10, 50)


def test_an_empty_draft_does_nothing():
    d, c = tu.Draft([]), _ctx()
    kc = z(20, 2, 64)
    tu.draft_append(c, kc, kc, ATTN, d, z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), z(0, 4, 64))
    tu.draft_attention(c, kc, kc, ATTN, d, z(0, 4, 64), z(0, 4, 64))
    tu.draft_short_conv(d, [(z(1, 8), z(0, 8), z(8, 2), z(0, 8))])
    tu.draft_accept(c, d, [], tu.DraftStack([]))
    tu.qk_norm_rope(ATTN, z(0, 4, 64), None, z(0, 4, 64), None)
    _raises(B.TU_ERR_ARG, lambda: tu.draft_verify(d, z(0, dtype=torch.int32), z(0, 5, dtype=f32), z(0, dtype=f32)))


def test_capacity_and_positions():
    d = tu.Draft([-1, 0, 0])
    q, kv = z(3, 4, 64), z(3, 2, 64)
    full = _ctx(18, 20)
    kc = z(20, 2, 64)
    _raises(B.TU_ERR_CAPACITY, lambda: tu.draft_append(full, kc, kc, ATTN, d, q, kv, kv, q))
    _raises(B.TU_ERR_CAPACITY, lambda: tu.draft_attention(full, kc, kc, ATTN, d, q, q))
    _raises(B.TU_ERR_CAPACITY, lambda: tu.draft_accept(full, d, [0], tu.DraftStack([])))
    late = _ctx(5, 20, cursor=2 ** 31 - 3)
    _raises(B.TU_ERR_ARG, lambda: tu.draft_append(late, kc, kc, ATTN, d, q, kv, kv, q))
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, q, None, q, None, first_pos=2 ** 31 - 3))
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, q, None, q, None, first_pos=-1))
    runs = _ctx(5, 20, cursor=50, live_cap=1)
    _raises(B.TU_ERR_CAPACITY, lambda: tu.draft_accept(runs, d, [0], tu.DraftStack([])))
    assert runs.intervals() == [(0, 5)] and runs.next_pos == 50


def test_norms():
    q = z(3, 4, 64)
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(weight_offset=float("inf"))):
        _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, q, None, q, None, norm=tu.QkNorm("rms", **kw)))
    bad = tu.QkNorm("rms")
    bad.c.kind = 7
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, q, None, q, None, norm=bad))
    with pytest.raises(ValueError):
        tu.QkNorm("rms", 1e-6, z(64, dtype=f32))
    with pytest.raises(ValueError):
        tu.qk_norm_rope(ATTN, q, None, q, None, norm=tu.QkNorm("rms", 1e-6, z(128)))
    with pytest.raises(ValueError):
        tu.qk_norm_rope(ATTN, None, None, None, None)
    # strides of tokens: not a multiple of 8, misaligned, overlapping
    wide = torch.zeros(3, 4 * 64 + 4, dtype=bf)
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, wide[:, :256].view(3, 4, 64), None, q, None))
    flat = torch.zeros(3 * 256 + 8, dtype=bf)
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, flat[1:769].view(3, 4, 64), None, q, None))
    one = torch.zeros(1, 4, 64, dtype=bf).expand(3, 4, 64)
    _raises(B.TU_ERR_ARG, lambda: tu.qk_norm_rope(ATTN, one, None, q, None))
    with pytest.raises(ValueError):
        tu.qk_norm_rope(ATTN, z(3, 64, 4).transpose(1, 2), None, q, None)


@pytest.mark.parametrize("what", ["dtype", "shape", "contiguous"])
def test_tensors(what):
    d, c = tu.Draft([-1, 0, 0]), _ctx()
    wrong = {"dtype": lambda *s: z(*s, dtype=torch.float16), "shape": lambda *s: z(s[0] + 1, *s[1:]),
             "contiguous": lambda *s: z(s[0], *s[1:-1], 2 * s[-1])[..., ::2]}[what]
    kc = z(20, 2, 64)
    calls = [lambda: tu.draft_attention(c, kc, kc, ATTN, d, wrong(3, 4, 64), z(3, 4, 64)),
             lambda: tu.draft_attention(c, kc, kc, ATTN, d, z(3, 4, 64), wrong(3, 4, 64)),
             lambda: tu.draft_append(c, kc, kc, ATTN, d, z(3, 4, 64), z(3, 2, 64), wrong(3, 2, 64), z(3, 4, 64)),
             lambda: tu.draft_short_conv(d, [(z(1, 8), wrong(3, 8), z(8, 2), z(3, 8))]),
             lambda: tu.draft_delta_rule(wrong(4, 64, 64), z(3, 2, 64), z(3, 2, 64), z(3, 4, 64), z(3, 4, dtype=f32),
                                         z(3, 4, dtype=f32), DELTA, d, z(3, 4, 64, dtype=f32)),
             lambda: tu.draft_verify(d, wrong(3), z(3, 9, dtype=f32), z(3, dtype=f32)),
             lambda: tu.draft_verify(d, z(3, dtype=torch.int32), z(3, 9, dtype=f32), z(3, dtype=f32), proposal=wrong(3, 9)),
             lambda: tu.DraftStack([tu.LayerIO(tu.TU_LAYER_DELTA, None, z(3, 2, 64), wrong(3, 4, 64), None,
                                               state=[z(4, 64, 64, dtype=f32)], beta=z(3, 4, dtype=f32),
                                               g=z(3, 4, dtype=f32))], None, DELTA)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    for short in (z(19, 2, 64), z(20, 2, 128), z(20, 1, 64)):
        with pytest.raises(ValueError):
            tu.draft_attention(c, short, kc, ATTN, d, z(3, 4, 64), z(3, 4, 64))


def test_workspaces():
    d, c = tu.Draft([-1, 0, 0]), _ctx(1000, 1010, 1000)
    kc = z(1010, 2, 64)
    need = tu.draft_attention_workspace_size(c, ATTN, d)
    assert need > 256
    _raises(B.TU_ERR_WORKSPACE, lambda: tu.draft_attention(c, kc, kc, ATTN, d, z(3, 4, 64), z(3, 4, 64),
                                                           workspace=z(need - 1, dtype=torch.uint8)))
    need = tu.draft_verify_workspace_size(d, 9)
    _raises(B.TU_ERR_WORKSPACE, lambda: tu.draft_verify(d, z(3, dtype=torch.int32), z(3, 9, dtype=f32), z(3, dtype=f32),
                                                        workspace=z(need - 1, dtype=torch.uint8)))


def test_verification():
    t = (z(3, dtype=torch.int32), z(3, 9, dtype=f32), z(3, dtype=f32))
    _raises(B.TU_ERR_ARG, lambda: tu.draft_verify(tu.Draft([-1, -1, 0]), *t))      # two roots
    _raises(B.TU_ERR_ARG, lambda: tu.draft_verify(tu.Draft([-1, 0, 0]), t[0], z(3, 0, dtype=f32), t[2]))
    with pytest.raises(ValueError):
        tu.draft_verify(tu.Draft([-1, 0, 0]), t[0], z(3, 18, dtype=f32)[:, ::2], t[2])


def test_paths_and_stacks():
    d, c = tu.Draft([-1, 0, 0, 2]), _ctx()
    for path in ([1], [0, 3], [0, 2, 2], [0, 4], [-1], [0, 1, 3]):
        _raises(B.TU_ERR_ARG, lambda: tu.draft_accept(c, d, path, tu.DraftStack([])))
    assert (c.len, c.next_pos, c.intervals()) == (10, 50, [(0, 10)])
    layer = tu.LayerIO(tu.TU_LAYER_DELTA, None, z(3, 2, 64), z(3, 4, 64), None, state=[z(4, 64, 64, dtype=f32)],
                       beta=z(3, 4, dtype=f32), g=z(3, 4, dtype=f32))
    with pytest.raises(ValueError):     # 3 rows, 4 nodes
        tu.draft_accept(c, d, [0], tu.DraftStack([layer], None, DELTA))
    with pytest.raises(ValueError):
        tu.DraftStack([layer])
    cache = tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[z(19, 2, 64)], v_cache=[z(19, 2, 64)])
    with pytest.raises(ValueError):     # shorter than the context's capacity
        tu.draft_accept(c, d, [0], tu.DraftStack([cache], ATTN))
    with pytest.raises(ValueError):     # widths differ
        tu.DraftStack([], convs=[(z(3, 8), z(4, 8)), (z(2, 8), z(4, 8))])


def test_conv_widths_and_channels():
    d = tu.Draft([-1, 0])
    _raises(B.TU_ERR_ARG, lambda: tu.draft_short_conv(d, [(z(1, 12), z(2, 12), z(12, 2), z(2, 12))]))
    _raises(B.TU_ERR_ARG, lambda: tu.draft_short_conv(d, [(z(8, 8), z(2, 8), z(8, 9), z(2, 8))]))
    _raises(B.TU_ERR_ARG, lambda: tu.draft_short_conv(d, [(None, z(2, 8), z(8, 2), z(2, 8))]))
    with pytest.raises(ValueError):
        tu.draft_short_conv(d, [(z(1, 8), z(2, 8), z(8, 2), z(2, 8)), (z(2, 8), z(2, 8), z(8, 3), z(2, 8))])


def test_head_and_channel_counts_beyond_the_launches_offsets():
    """The counts alone are refused, before any address matters (no such tensor exists here)."""
    one = z(64)
    p = ctypes.byref
    many = tu.attn_params(1 << 17, 1, 64)
    d = tu.Draft([i - 1 for i in range(128)])
    c = _ctx(10, 200)
    ws = z(1 << 12, dtype=torch.uint8)
    assert B.lib().draft_attention(p(c.c), one.data_ptr(), one.data_ptr(), p(many), d._ref, one.data_ptr(), one.data_ptr(),
                                   ws.data_ptr(), 1 << 40, None) == B.TU_ERR_ARG
    assert b"too many heads" in B.lib().tu_last_error()
    wide = tu.delta_params(1, 1 << 16, 64, 64, 16)
    f = z(64, dtype=f32)
    assert B.lib().draft_delta_rule(f.data_ptr(), one.data_ptr(), one.data_ptr(), one.data_ptr(), f.data_ptr(), f.data_ptr(),
                                    p(wide), d._ref, f.data_ptr(), None) == B.TU_ERR_ARG
    assert b"too many heads" in B.lib().tu_last_error()
    t = (B.tu_conv_tensor * 1)(B.tu_conv_tensor(one.data_ptr(), one.data_ptr(), one.data_ptr(), one.data_ptr(), 128, 1 << 24, 0))
    assert B.lib().draft_short_conv(d._ref, t, 1, 4, 0, None) == B.TU_ERR_ARG
    assert b"too many channels" in B.lib().tu_last_error()
    path = (ctypes.c_int32 * 1)(0)
    assert B.lib().draft_accept(p(c.c), d._ref, path, 1, None, 0, None, None, t, 1, 4, None) == B.TU_ERR_ARG
    assert b"too many channels" in B.lib().tu_last_error() and c.len == 10


def test_a_stack_holds_one_context():
    pair = tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[z(20, 2, 64)] * 2, v_cache=[z(20, 2, 64)] * 2)
    with pytest.raises(ValueError):
        tu.DraftStack([pair], ATTN)
    with pytest.raises(ValueError):
        tu.DraftStack([tu.LayerIO(tu.TU_LAYER_DELTA, None, z(3, 2, 64), z(3, 4, 64), None, beta=z(3, 4, dtype=f32),
                                  g=z(3, 4, dtype=f32))], None, DELTA)


def _splits(p, rows, n):
    """Splits of the key range, read off the workspace's size."""
    size = B.lib().draft_attention_workspace_size(ctypes.byref(p), n, rows)
    if size == 256:
        return 1
    waves = -(-n * (p.n_q_heads // p.n_kv_heads) // 32) * p.n_kv_heads
    s = round((size - 256) / (waves * 32 * (p.head_dim * 2 + 8)))
    up = lambda x: -(-x // 256) * 256
    assert size == 256 + up(s * waves * 32 * p.head_dim * 2) + up(s * waves * 32 * 8)
    return s


def test_splits_of_the_attention():
    big, mid = tu.attn_params(16, 2, 256), tu.attn_params(32, 8, 128)
    for p in (big, mid):                                  # a few stages of 16 KB of keys are not split
        assert [_splits(p, r, 24) for r in (0, 1, 40)] == [1, 1, 1]
        assert _splits(p, 600, 1) > 4
    assert _splits(big, 32767, 1) == 128 and _splits(big, 65536, 64) == 64     # a workgroup on every CU
    assert _splits(big, 2976, 1) == 94 and _splits(big, 2976, 24) == 32        # partial outputs cost more with more rows
    for n in (1, 7, 24, 64, 128):
        for rows in (0, 1, 31, 500, 5000, 200000):
            for p in (big, mid, tu.attn_params(40, 1, 64)):
                assert 1 <= _splits(p, rows, n) <= 128
    for s in (1, 2, 7, 64):                               # as asked for, as far as there are stages
        assert _splits(tu.attn_params(16, 2, 256, kv_splits=s), 4096, 24) == s
    assert _splits(tu.attn_params(16, 2, 256, kv_splits=64), 60, 4) == 2

"""What a program may keep from one call to the next: workspaces, prepared stacks (host only)."""
import ctypes
import gc
import random
import weakref

import pytest
import torch

import paper_2609_18935_amd as tu
from paper_2609_18935_amd import binding as B


def _size(p, n, rows):
    return B.lib().draft_attention_workspace_size(ctypes.byref(p), n, rows)


def _drawn(seed):
    rng = random.Random(seed)
    hkv = rng.choice([1, 2, 3, 8])
    return tu.attn_params(hkv * rng.choice([1, 4, 5, 8]), hkv, rng.choice([64, 128, 256]), kv_splits=rng.choice([0, 0, 0, 1, 7, 64]))


@pytest.mark.parametrize("p", [tu.attn_params(16, 2, 256), tu.attn_params(32, 8, 128), tu.attn_params(16, 4, 64), tu.attn_params(40, 1, 256),
                               tu.attn_params(16, 2, 256, kv_splits=5), *[_drawn(s) for s in range(12)]])
@pytest.mark.parametrize("nodes,rows", [(1, 0), (1, 32768), (24, 2150), (24, 12000), (40, 12000), (128, 70000), (128, 300)])
def test_one_attention_workspace_serves_every_shorter_context_and_smaller_draft(p, nodes, rows):
    bound = tu.draft_attention_workspace_bound(p, nodes, rows)
    lengths = sorted({*range(0, min(rows, 600) + 1, 7), *range(0, rows + 1, max(1, rows // 97)), rows})
    for n in range(1, nodes + 1):
        assert max(_size(p, n, r) for r in lengths) <= bound


def test_a_context_beyond_32_bit_offsets():
    p = tu.attn_params(32, 32, 256)        # 16 KB a row: a split takes 131,000 rows
    bound = tu.draft_attention_workspace_bound(p, 8, 3_000_000)
    assert all(_size(p, n, r) <= bound for n in range(1, 9) for r in range(0, 3_000_001, 50_000))


def test_an_exact_size_is_no_bound():
    p = tu.attn_params(16, 2, 256)
    assert _size(p, 24, 2100) > _size(p, 24, 2150)          # the reason for the bound


def test_bounds_refused():
    p, b = tu.attn_params(16, 2, 256), tu.draft_attention_workspace_bound
    assert b(p, 129, 10) == b(p, -1, 10) == b(p, 4, -1) == b(p, 4, 2 ** 30) == 0
    assert b(tu.attn_params(16, 3, 256), 4, 10) == 0
    assert b(p, 0, 10) >= 256


@pytest.mark.skipif(torch.cuda.is_available(), reason="host tensors stand in for device tensors")
def test_a_draft_stack_holds_its_tensors():
    """A layer that gets a new tensor, or a list that gets a new element, leaves the prepared stack its own."""
    bf = torch.bfloat16
    delta = tu.LayerIO(tu.TU_LAYER_DELTA, None, torch.zeros(3, 2, 64, dtype=bf), torch.zeros(3, 4, 64, dtype=bf), None,
                       state=[torch.zeros(4, 64, 64)], beta=torch.zeros(3, 4), g=torch.zeros(3, 4))
    attn = tu.LayerIO(tu.TU_LAYER_ATTN, None, None, None, None, k_cache=[torch.zeros(20, 2, 64, dtype=bf)],
                      v_cache=[torch.zeros(20, 2, 64, dtype=bf)])
    convs = [(torch.zeros(3, 8, dtype=bf), torch.zeros(3, 8, dtype=bf))]
    stack = tu.DraftStack([delta, attn], tu.attn_params(4, 2, 64), tu.delta_params(2, 4, 64, 64, 16), convs)
    given = [delta.k, delta.v, delta.beta, delta.g, delta.state[0], attn.k_cache[0], attn.v_cache[0], *convs[0]]
    refs, addresses = [weakref.ref(t) for t in given], [t.data_ptr() for t in given]
    del given
    delta.k = delta.v = delta.beta = delta.g = None
    delta.state[0], attn.k_cache[0], attn.v_cache[0], convs[0] = None, None, None, None
    gc.collect()
    assert all(r() is not None for r in refs)
    d, a, c = stack._layers[0], stack._layers[1], stack._convs[0]
    assert [d.k, d.v, d.beta, d.g, d.state[0], a.k_cache[0], a.v_cache[0], c.state, c.x] == addresses
    del stack, d, a, c
    gc.collect()
    assert all(r() is None for r in refs)


@pytest.mark.skipif(torch.cuda.is_available(), reason="host tensors stand in for device tensors")
def test_a_stack_update_holds_its_tensors():
    bf = torch.bfloat16
    ctx = tu.Context(20, device="cpu")
    ctx.set_metadata([(0, 10)], 50)
    delta = tu.LayerIO(tu.TU_LAYER_DELTA, torch.zeros(3, 2, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf),
                       torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 4, 64), state=[torch.zeros(4, 64, 64)],
                       beta=torch.zeros(3, 4), g=torch.zeros(3, 4))
    attn = tu.LayerIO(tu.TU_LAYER_ATTN, torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf),
                      torch.zeros(3, 2, 64, dtype=bf), torch.zeros(3, 4, 64), k_cache=[torch.zeros(20, 2, 64, dtype=bf)],
                      v_cache=[torch.zeros(20, 2, 64, dtype=bf)])
    index = [torch.zeros(20, dtype=torch.int32)]
    up = tu.StackUpdate([ctx], [[[2, 4]]], [3], [delta, attn], tu.attn_params(4, 2, 64), tu.delta_params(2, 4, 64, 64, 16),
                        src_index=index)
    given = [delta.q, delta.k, delta.v, delta.out, delta.beta, delta.g, delta.state[0], attn.q, attn.k, attn.v, attn.out,
             attn.k_cache[0], attn.v_cache[0], index[0]]
    refs = [weakref.ref(t) for t in given]
    del given
    for L in (delta, attn):
        L.q = L.k = L.v = L.out = L.beta = L.g = None
    delta.state[0], attn.k_cache[0], attn.v_cache[0], index[0] = None, None, None, None
    gc.collect()
    assert all(r() is not None for r in refs)
    del up
    gc.collect()
    assert all(r() is None for r in refs)

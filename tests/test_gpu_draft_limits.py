"""Speculative decoding on the GPU at the limits of its inputs, against the float64 definitions: rows
behind a short split."""
import numpy as np
import pytest
import torch

from draft_cases import bf16, tree, worst
from test_gpu_draft import _attn

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

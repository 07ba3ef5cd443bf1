"""Attention over selected blocks whose blocks are shared by several workgroups: the last of them combines
few states in one or two rounds of loads, a second kernel more; lists with fewer blocks than parts,
repeats and none at all. Against the fp64 oracle, with the tolerance of long_helpers.py."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal, poison  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

# (B, Hq, Hkv, Sq, Skv, D, block, topk): rows of a kv head x parts in the comments.
SHAPES = [
    (1, 32, 8, 1, 3000, 128, 64, 8),    # 4 x 8
    (1, 32, 8, 1, 3000, 128, 64, 16),   # 4 x 16
    (1, 32, 8, 1, 3000, 128, 64, 17),   # 4 x 17: a second kernel
    (2, 12, 4, 1, 2000, 128, 64, 13),   # 3 x 13
    (1, 10, 2, 1, 1000, 128, 64, 7),    # 5 x 7
    (1, 64, 8, 1, 2000, 128, 64, 8),    # 8 x 8
    (1, 36, 4, 1, 2000, 128, 64, 8),    # 9 x 8: a second kernel
    (1, 16, 4, 2, 1500, 128, 128, 5),   # 8 x 5
    (1, 8, 8, 5, 1500, 64, 64, 8),      # 5 x 8
    (1, 32, 8, 4, 2500, 64, 64, 4),     # 16 x 4
    (1, 34, 2, 1, 2500, 64, 64, 4),     # 17 x 4: a second kernel
    (3, 4, 1, 2, 2500, 64, 128, 16),    # 8 x 16
    (16, 32, 8, 1, 4100, 128, 64, 20),  # 4 x 4, parts of five blocks
    (16, 64, 8, 1, 4100, 64, 64, 10),   # 8 x 4, parts of three
    (64, 4, 4, 1, 700, 128, 64, 9),     # 1 x 2, as many heads as share their rows
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_parts(shape):
    announce(f"parts {shape}")
    B, Hq, H, Sq, S, D, bs, K = shape
    q, k, v = normal(420, B, Hq, Sq, D), normal(421, B, H, S, D), normal(422, B, H, S, D)
    n = [S - 61 * b if b % 4 != 3 else b % 3 for b in range(B)]
    n = [max(x, 1 + b % 5) if b % 4 != 3 else x for b, x in enumerate(n)]
    nb = -(-S // bs)
    g = torch.Generator("cpu").manual_seed(423)
    lists = torch.rand(B, H, Sq, max(nb, K), generator=g).argsort(-1)[..., :K].to(torch.int32)
    lists = torch.where(lists < nb, lists, -1)
    lists[:, 0, 0, 1:] = -1                # one block for all parts
    lists[:, H - 1, Sq - 1] = -1           # none
    lists[:, 1 % H, Sq - 1, K // 2:] = lists[:, 1 % H, Sq - 1, :1]
    a = [f64(t) for t in (q, k, v)]
    ref = oracle.attention_blocks_ref(*a, lists.numpy(), bs, D ** -0.5, n)
    mag = oracle.attention_blocks_ref(*a[:2], np.abs(a[2]), lists.numpy(), bs, D ** -0.5, n)
    args = (q.cuda(), poison(k, n), poison(v, n), lists.cuda(), bs)
    ws = ef.make_blocks_workspace(args[0], args[1], K, bs)
    ws[ef.COUNTER_REGION_BYTES:] = 255  # states that are not written are NaN
    for _ in range(2):
        got = ef.attention_blocks(*args, lengths=lengths_of(n), workspace=ws)
        torch.cuda.synchronize()
        close(got, ref, mag, shape)
    assert not ef.workspace_counters(ws).any()

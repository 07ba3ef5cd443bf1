"""Block selection of batches with hundreds of kv heads, whose few queries fill a row tile in part, as a
whole, or a little more than one. Against the fp64 oracle, for equality."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, f64, lengths_of, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Sq", [1, 3, 4, 5, 8, 9, 17])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_select_of_many_heads(G, Sq):
    announce(f"select of many heads: {Sq} queries, groups of {G}")
    B, H, NB, D, K = 129, 4, 64 * 8 // G, 64, 9
    S = 64 * NB
    n = [S - 64 * b - b % 7 if b % 5 else S for b in range(B)]
    n = [max(x, b % 3) for b, x in enumerate(n)]
    q, m = normal(330, B, G * H, Sq, D), normal(331, B, H, NB, D)
    got = ef.block_select(q.cuda(), m.cuda(), S, K, 64, 1, 2, lengths=lengths_of(n))
    torch.cuda.synchronize()
    ref = oracle.block_select_ref(f64(q), f64(m), S, K, 64, 1, 2, n)
    bad = np.argwhere((got.cpu().numpy() != ref).any(-1))
    assert len(bad) == 0, (len(bad), bad[0])

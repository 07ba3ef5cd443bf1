"""Calls of more threads than a launch holds, which are made in several: the last sequences and rows are
what they are in a call of their own, and as the fp64 oracle has them."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu


def test_select_in_several_launches():
    """More than 2^23 workgroups of one query each. Few of the queries have a place."""
    announce("selection in several launches")
    B, H, Sq, D, S, K = 130, 4, 17000, 64, 64 * 16000, 9
    n = torch.full((B,), 700)
    n[::13], n[-1] = 0, 64 * 15
    q = torch.randn(B, H, Sq, D, device="cuda", dtype=torch.bfloat16)
    m = torch.randn(B, H, S // 64, D, device="cuda", dtype=torch.bfloat16)
    n = n.int().cuda()
    got = ef.block_select(q, m, S, K, 64, 1, 2, lengths=n)
    torch.cuda.synchronize()
    # The positions before the first key have no block.
    place = torch.arange(Sq, device="cuda") + n[:, None] - Sq
    assert (got.transpose(1, 2)[place < 0] == -1).all()
    tail = slice(Sq - 1000, Sq)
    for b in (0, 1, 64, 123, 124, 128, 129):
        ref = oracle.block_select_ref(f64(q[b:b + 1, :, tail]), f64(m[b:b + 1]), S, K, 64, 1, 2,
                                      [int(n[b])])
        assert np.array_equal(got[b:b + 1, :, tail].cpu().numpy(), ref), b


def test_combine_in_several_launches():
    """More than 2^25 rows whose states a second kernel combines."""
    announce("combine in several launches")
    B, Sq, D, Lp, S = 65535, 513, 64, 8400, 1
    size = ef.ef_attention_shared_prefix_workspace_size(B, 1, 1, Sq, Lp, S, D)
    assert size > ef.COUNTER_REGION_BYTES + B * Sq * 2 * D * 4  # two states to a row
    q = torch.empty(B, 1, Sq, D, device="cuda", dtype=torch.bfloat16)
    for i in range(0, B, 4096):
        q[i:i + 4096].normal_()
    k, v = (torch.randn(B, 1, S, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    kp, vp = (torch.randn(1, Lp, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    got = ef.attention_shared_prefix(q, kp, vp, k, v)
    torch.cuda.synchronize()
    for b in (0, 32703, 32767, 65408, 65534):  # about the ends of 2^24 and 2^25 rows too
        a = [f64(t) for t in (q[b:b + 1], kp, vp, k[b:b + 1], v[b:b + 1])]
        ref = oracle.shared_prefix_ref(*a, D ** -0.5)
        mag = oracle.shared_prefix_ref(a[0], a[1], np.abs(a[2]), a[3], np.abs(a[4]), D ** -0.5)
        close(got[b:b + 1], ref, mag, b)

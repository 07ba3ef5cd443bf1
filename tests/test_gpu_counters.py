"""Arrival counters that were not zero when a call began: from the number of workgroups that share a row
on, its rows are NaN; below that they are undefined; clearing the region makes the workspace good."""

import pytest
import torch

from long_helpers import _gpu, announce, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

P = 8  # blocks of a list, each with a workgroup of its own


@pytest.mark.parametrize("value", [1, P - 1, P, P + 1, 64, 2 ** 30])
def test_blocks_with_a_counter_that_was_not_zero(value):
    announce(f"counter {value}")
    B, Hq, H, D, S = 1, 8, 2, 64, 2000
    q, k = normal(410, B, Hq, 1, D).cuda(), normal(411, B, H, S, D).cuda()
    lists = ef.block_select(q, ef.block_summary(k), S, P)
    ws = ef.make_blocks_workspace(q, k, P)
    # The workspace's size says how many share a row: counters, two sums of 256 bytes, values.
    assert ws.numel() == ef.COUNTER_REGION_BYTES + 512 + Hq * P * D * 4
    want = ef.attention_blocks(q, k, k, lists, workspace=ws)
    counters = ef.workspace_counters(ws)
    counters[1, 0] = value  # of the second kv head
    got = ef.attention_blocks(q, k, k, lists, workspace=ws)
    torch.cuda.synchronize()
    half = Hq // H
    assert torch.equal(got[:, :half], want[:, :half])
    if value >= P:
        assert torch.isnan(got[:, half:]).all()
    counters.zero_()
    for _ in range(2):
        assert torch.equal(ef.attention_blocks(q, k, k, lists, workspace=ws), want)
    assert not counters.any()

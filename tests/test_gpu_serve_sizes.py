"""Attention over pages where one sequence has a chunk of its prompt and many others a single token:
launches without a second one, with one, and with several. Tolerance of long_helpers.py."""

import pytest
import torch

from long_helpers import _gpu, announce, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, starts_of
from test_gpu_serve_attention import run_packed, run_paged

pytestmark = pytest.mark.gpu


def beside(chunk, keys, at, B):
    """new tokens and lengths of B sequences, the one at `at` with a chunk."""
    new, lengths = [1] * B, [1 + 37 * i % 400 for i in range(B)]
    new[at], lengths[at] = chunk, keys
    return new, lengths


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,page,chunk,keys,at,B", [
    # 2048 heads and row tiles: a workgroup each, nothing is cut.
    (64, 8, 64, 16, 1024, 1100, 0, 34),
    # 1024: two each, which cut the chunk's keys.
    (64, 8, 128, 64, 512, 3000, 33, 66),
    # The parts of 1024 sequences are joined by a launch, those behind them by another.
    (64, 8, 64, 32, 512, 1500, 1050, 1100),
])
def test_chunk_beside_many_sequences(Hq, H, D, page, chunk, keys, at, B, e4m3):
    announce(f"chunk of {chunk} over {keys} at {at} of {B} e4m3 {e4m3}")
    new, lengths = beside(chunk, keys, at, B)
    run_paged((Hq, H, D, page, new, lengths), e4m3)


@pytest.mark.parametrize("H", [1030, 2100])
def test_many_heads(H):
    """A workgroup to each head: counters where there are enough of them, none where not, and nothing to
    join."""
    announce(f"{H} kv heads")
    run_paged((2 * H, H, 64, 16, [1, 2], [40, 7]), False)


def test_paged_workspace_of_the_largest_call():
    """One made for a chunk of 520 tokens serves all shorter ones, with the same results as their own."""
    announce("a paged workspace for smaller calls")
    B, lengths = 16, [530 + 60 * i for i in range(16)]
    p = Pages(120, 8, 64, 64, lengths, False)
    q = normal(121, 520 + B - 1, 64, 64).cuda()
    ws = ef.make_paged_workspace(q, p.cache, B, 520)
    for n in (520, 500, 257, 40, 4, 1):
        new = [n] + [1] * (B - 1)
        qn, starts = q[:sum(new)].contiguous(), ints(starts_of(new))
        got = ef.attention_paged(qn, p.cache, p.dev_table, ints(lengths), starts=starts, max_queries=n,
                                 workspace=ws)
        own = ef.attention_paged(qn, p.cache, p.dev_table, ints(lengths), starts=starts, max_queries=n)
        assert torch.isfinite(got).all() and torch.equal(got, own), n
    few = ints(lengths[:3])
    got = ef.attention_paged(q[:3], p.cache, p.dev_table[:3].contiguous(), few, workspace=ws)
    assert torch.equal(got, ef.attention_paged(q[:3], p.cache, p.dev_table[:3].contiguous(), few))


@pytest.mark.parametrize("Tk,B", [(900, 1), (5000, 1), (1000, 8)])
def test_packed_workspace_of_the_largest_call(Tk, B):
    """One made for the longest chunks serves shorter ones, whose keys are cut into more parts."""
    announce(f"a packed workspace for smaller calls, {Tk} keys of {B}")
    most = 200
    ws = ef.make_packed_workspace(torch.empty(most, 32, 128, device="cuda"),
                                  torch.empty(Tk, 8, 128, device="cuda"), B)
    ws[ef.COUNTER_REGION_BYTES:] = 0xff  # (NaN, if anything were read before it was written)
    keys = [Tk // B + (-1) ** i * 20 * (B > 1) for i in range(B)]
    for T in (most, 128, 127, 20, 16, 15, 9, 8):
        new = [T // B] * B
        got = run_packed((32, 8, 128, new, keys, True), workspace=ws)
        assert torch.equal(got, run_packed((32, 8, 128, new, keys, True))), T
        assert not ef.workspace_counters(ws).any()

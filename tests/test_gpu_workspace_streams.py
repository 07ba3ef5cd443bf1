"""Workspaces and the streams they belong to: one made for a stream is cleared there, and one that a
call makes for itself is that call's stream's, whatever the current stream is busy with."""

import pytest
import torch

from long_helpers import _gpu, announce, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

B, HQ, H, D, S = 1, 8, 2, 128, 3000


def tensors():
    return normal(400, B, HQ, 1, D).cuda(), normal(401, B, H, S, D).cuda()


def dirty(n):
    """What memory of n bytes held before, as the current stream's allocator gives it again."""
    torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def occupy(busy):
    for _ in range(20):
        busy = (busy @ busy).clamp(-1, 1)
    return busy


MAKE = {
    "blocks": (lambda q, k, x, **s: ef.make_blocks_workspace(q, k, 12, **s),
               lambda q, k, x, **s: ef.attention_blocks(q, k, k, x, **s)),
    "shared_prefix": (lambda q, k, x, **s: ef.make_shared_prefix_workspace(q, k[0], k, **s),
                      lambda q, k, x, **s: ef.attention_shared_prefix(q, k[0], k[0], k, k, **s)),
    "splitkv": (lambda q, k, x, **s: ef.make_workspace(q, k, **s),
                lambda q, k, x, **s: ef.attention_splitkv(q, k, k, **s)),
}


@pytest.mark.parametrize("name", MAKE)
def test_workspace_made_for_a_stream(name):
    """Its first call, on that stream, waits for nothing of the current one."""
    announce(f"workspace for a stream: {name}")
    make, call = MAKE[name]
    q, k = tensors()
    x = ef.block_select(q, ef.block_summary(k), S, 12)
    want = call(q, k, x)
    busy = torch.randn(4096, 4096, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    n = make(q, k, x).numel()
    for i in range(3):
        dirty(n)
        with torch.cuda.stream(stream):
            dirty(n)
        busy = occupy(busy)
        ws = make(q, k, x, stream=stream)
        got = call(q, k, x, workspace=ws, stream=stream)
        stream.synchronize()
        assert torch.equal(got, want), i
        torch.cuda.synchronize()
        assert not ef.workspace_counters(ws).any()


def diff_args(q, k):
    vec = [normal(402 + i, D).cuda().float() / 8 for i in range(5)]
    return (q, q.flip(1).contiguous(), k, k.flip(2).contiguous(), k, *vec, 0.5)


OWN = {
    "fwd": lambda q, k, x, **s: ef.attention_fwd(q, k, k, **s),
    "splitkv": lambda q, k, x, **s: ef.attention_splitkv(q, k, k, **s),
    "splitkv_window": lambda q, k, x, **s: ef.attention_splitkv(q, k, k, causal=True, window=2000,
                                                                sinks=4, **s),
    "dsplit": lambda q, k, x, **s: ef.attention_decode_dsplit(q, k, k, **s),
    "diff": lambda q, k, x, **s: ef.diff_attention(*x, **s),
    "partials": lambda q, k, x, **s: ef.workspace_views(
        ef.attention_splitkv_partials(q, k, k, partition_size=256, **s), B, HQ, 1, S, D, 256)[1],
}


@pytest.mark.parametrize("name", OWN)
def test_workspace_of_the_call(name):
    """A call on another stream that is given no workspace makes it there."""
    announce(f"own workspace on a stream: {name}")
    call = OWN[name]
    q, k = tensors()
    x = diff_args(q, k)
    want = call(q, k, x).clone()
    n = max(ef.splitkv_workspace_size(B, HQ, H, 1, S, D, p) for p in (0, 256))
    busy = torch.randn(4096, 4096, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(3):
        dirty(n)
        busy = occupy(busy)
        got = call(q, k, x, stream=stream)
        busy = occupy(busy)
        dirty(n)  # would take the memory of a workspace freed here
        stream.synchronize()
        with torch.cuda.stream(stream):
            same = torch.equal(got, want)
        assert same, i
        torch.cuda.synchronize()

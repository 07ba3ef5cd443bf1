"""Which sizes the serving entry points take, and how their workspaces grow. No call here reaches a GPU."""

import os
import random

import pytest

from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.skipif(not os.path.exists(ef.LIB_PATH), reason="libef_attention.so not built")

A = 0x10000  # a fake device address, never dereferenced
SHAPE, MISALIGNED, WS = 2, 5, 7

paged_size = ef.ef_attention_paged_workspace_size
packed_size = ef.ef_attention_packed_workspace_size


def paged_without_workspace(T, B, Hq, Hkv, D, max_queries, width=64, page=16):
    """Status of a call that has all but a workspace, which is the last thing looked at."""
    return ef.ef_attention_paged(A, A, A, None, None, A, A, A, A, T, B, Hq, Hkv, D, max_queries, 99,
                                 page, width, 0, 0.1, None, 0, None)


@pytest.mark.parametrize("T,B,Hq,Hkv,D,max_queries", [
    (8192, 33, 32, 8, 128, 2048),    # a chunk of a prompt beside single tokens
    (8192, 128, 32, 8, 128, 2048),
    (8192, 512, 64, 8, 64, 4096),
    (4096, 66, 64, 8, 128, 512),     # two workgroups a head and row tile
    (3000, 2000, 32, 8, 128, 600),
    (100000, 100000, 32, 8, 128, 5),
])
def test_chunks_beside_many_sequences(T, B, Hq, Hkv, D, max_queries):
    assert paged_size(T, B, Hq, Hkv, D, max_queries) > ef.COUNTER_REGION_BYTES
    assert paged_without_workspace(T, B, Hq, Hkv, D, max_queries) == WS


def test_most_row_tiles():
    """max_queries Hq / 32 workgroups of a launch, up to 2^23."""
    assert paged_without_workspace(2 ** 23, 1, 32, 8, 128, 2 ** 23) == WS
    assert paged_without_workspace(2 ** 23 + 8, 1, 32, 8, 128, 2 ** 23 + 8) == SHAPE


def spread(rng, most):
    """A number up to `most`, over its logarithm."""
    return max(1, round(most ** rng.random()))


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (64, 8, 64), (12, 12, 64), (6, 3, 128), (16, 1, 128),
                                      (2100, 700, 64), (3000, 3000, 64)])
def test_paged_workspace_serves_smaller_calls(Hq, Hkv, D):
    rng = random.Random(Hq)
    for _ in range(4000):
        T, B, n = spread(rng, 100000), spread(rng, 5000), spread(rng, 10000)
        large = paged_size(T, B, Hq, Hkv, D, n)
        assert large > 0
        for smaller in ((spread(rng, T), spread(rng, B), spread(rng, n)), (T, B, spread(rng, n)),
                        (T, B, max(n - 1, 1)), (max(T - 1, 1), B, n), (T, max(B - 1, 1), n)):
            assert paged_size(*smaller[:2], Hq, Hkv, D, smaller[2]) <= large, (T, B, n, smaller)


def test_paged_workspace_of_one_chunk():
    """Each step of a growing chunk, where a head's workgroups go from two to one."""
    sizes = [paged_size(8192, 16, 32, 8, 128, n) for n in range(1, 3000)]
    assert sizes == sorted(sizes) and sizes[-1] < 2 ** 27


HEADS = [(32, 8, 128), (64, 8, 64), (12, 12, 64), (6, 3, 128), (16, 1, 128), (3000, 1000, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_packed_workspace_serves_smaller_calls(Hq, Hkv, D):
    rng = random.Random(Hq)
    for _ in range(4000):
        T, Tk, B = spread(rng, 50000), spread(rng, 200000), spread(rng, 3000)
        large = packed_size(T, Tk, B, Hq, Hkv, D)
        for smaller in ((spread(rng, T), spread(rng, Tk), spread(rng, B)), (spread(rng, T), Tk, B),
                        (max(T - 1, 1), Tk, B), (T, max(Tk - 1, 1), B), (T, Tk, max(B - 1, 1))):
            assert packed_size(*smaller, Hq, Hkv, D) <= large, (T, Tk, B, smaller)


@pytest.mark.parametrize("B,Tk", [(1, 900), (1, 5000), (8, 1000)])
def test_packed_workspace_of_one_chunk(B, Tk):
    """Each step of growing chunks, across the border where parts become longer."""
    sizes = [packed_size(T, Tk, B, 32, 8, 128) for T in range(1, 300)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert packed_size(300, 512, B, 32, 8, 128) == 0  # (nothing is cut)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_packed_calls_take_the_workspace_of_larger_ones(Hq, Hkv, D):
    """Of that size it is enough, or where the call cuts nothing not looked at. (The address is not
    aligned, which is found behind the size; calls that cut nothing are left out.)"""
    rng = random.Random(Hkv)
    for _ in range(2000):
        T, Tk, B = spread(rng, 50000), spread(rng, 200000), spread(rng, 3000)
        t, tk, b = spread(rng, T), spread(rng, Tk), spread(rng, B)
        if tk <= 1024:
            continue
        size = packed_size(T, Tk, B, Hq, Hkv, D)
        call = (A, A, A, A, A, A, t, tk, b, Hq, Hkv, D, 0.1, 1, A + 8)
        assert ef.ef_attention_packed(*call, size, None) == MISALIGNED, (T, Tk, B, t, tk, b)
        assert ef.ef_attention_packed(*call, 1000, None) == WS


def test_most_packed_sequences():
    """T Hq / 128 + B Hkv workgroups of a launch, up to 2^23 (fewer for sequences of one token)."""
    call = (A, A, A, A, A, A)
    assert ef.ef_attention_packed(*call, 2 ** 20, 2 ** 21, 2 ** 19, 32, 8, 128, 0.1, 1, None, 0,
                                  None) == WS
    for T, B in ((2 ** 22, 2 ** 22), (2 ** 25, 2 ** 19)):
        assert ef.ef_attention_packed(*call, T, 2 ** 21, B, 32, 8, 128, 0.1, 1, None, 0, None) == SHAPE

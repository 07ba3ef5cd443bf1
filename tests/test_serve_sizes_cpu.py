"""Which sizes the serving entry points take, and how their workspaces grow. No call here reaches a GPU."""

import os

import pytest

from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.skipif(not os.path.exists(ef.LIB_PATH), reason="libef_attention.so not built")

A = 0x10000  # a fake device address, never dereferenced
SHAPE, WS = 2, 7

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

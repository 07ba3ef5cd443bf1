"""Selections of more queries than a launch takes are refused on the host."""

import os

import pytest

from paper_2609_12330_amd import ef_attention as ef

A = 0x10000  # a fake device address, never dereferenced: the call is refused


@pytest.mark.skipif(not os.path.exists(ef.LIB_PATH), reason="libef_attention.so not built")
@pytest.mark.parametrize("Sq", [2 ** 24, 2 ** 25 - 1])
def test_select_of_too_many_queries(Sq):
    # 15625 blocks: the scores of one query fill a workgroup's LDS, so each has one.
    assert ef.ef_block_select(A, A, None, A, 1, 1, 1, Sq, 10 ** 6, 64, 64, 8, 1, 2, None) == 2
    assert ef.ef_block_select(A, A, A, A, 3, 32, 2, Sq, 10 ** 6, 64, 64, 8, 1, 2, None) == 2

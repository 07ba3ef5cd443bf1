"""Attention over pages and of packed sequences written over its queries: a row's queries are read by all
workgroups that have keys of it before the row is written. The result is that of a separate output."""

import pytest
import torch

from long_helpers import _gpu, announce, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,new,lengths", [
    (8, 2, 128, [1, 1, 1], [3000, 40, 900]),      # parts joined in the launch
    (64, 8, 64, [4, 1, 3], [2000, 50, 3]),        # by a second one
    (64, 8, 128, [30, 7, 1], [1000, 50, 9000]),   # several row tiles
])
def test_paged_in_place(Hq, H, D, new, lengths, e4m3):
    announce(f"paged in place {Hq} {H} {D} {new} {e4m3}")
    p = Pages(150, H, 16, D, lengths, e4m3)
    q = normal(151, sum(new), Hq, D).cuda()
    args = (p.cache, p.dev_table, ints(lengths), ints(starts_of(new)), max(new))
    want = ef.attention_paged(q.clone(), *args)
    assert ef.attention_paged(q, *args, out=q) is q
    assert torch.equal(q, want)


@pytest.mark.parametrize("Hq,H,D,new,keys,causal", [
    (32, 8, 128, [17, 1, 130], [17, 1, 130], True),    # whole
    (8, 1, 128, [3, 40], [9000, 2000], True),          # keys in parts
    (8, 2, 64, [300, 5], [5000, 5], False),            # both
])
def test_packed_in_place(Hq, H, D, new, keys, causal):
    announce(f"packed in place {Hq} {H} {D} {new} {keys}")
    q = normal(152, sum(new), Hq, D).cuda()
    k, v = (normal(153 + i, sum(keys), H, D).cuda() for i in range(2))
    args = (k, v, ints(starts_of(new)), ints(starts_of(keys)))
    want = ef.attention_packed(q.clone(), *args, causal=causal)
    assert ef.attention_packed(q, *args, causal=causal, out=q) is q
    assert torch.equal(q, want)

"""Attention over a paged cache and of packed sequences on the GPU, against the fp64 oracle. The
tolerance is the one derived in long_helpers.py (8-bit caches: their codes and scales are exact in
the kernel, so nothing is added)."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, starts_of

pytestmark = pytest.mark.gpu

# (Hq, Hkv, D, page, new tokens, lengths)
PAGED = [
    (1, 1, 64, 16, [1], [1]),
    (4, 2, 128, 16, [1], [777]),
    (32, 8, 128, 16, [1, 1, 1], [1, 300, 64]),
    (8, 8, 64, 32, [1] * 5, [5, 1000, 33, 0, 129]),       # a sequence without keys
    (16, 4, 128, 64, [3, 1, 4, 2], [3, 500, 2, 1300]),    # rows in front of position 0
    (64, 8, 128, 16, [4] * 3, [1000, 17, 2300]),          # 32 rows a head
    (64, 8, 64, 128, [5, 0, 1, 16], [700, 90, 1, 16]),    # several row tiles, an empty one
    (12, 4, 128, 256, [2, 2], [513, 256]),                # groups of 3
    (8, 2, 64, 16, [1] * 70, [1 + 37 * i % 200 for i in range(70)]),  # over 64 sequences
    (32, 8, 128, 32, [1] * 130, [1 + 91 * i % 400 for i in range(130)]),
    (4, 1, 128, 16, [7], [20000]),                        # one sequence in many parts
    (40, 2, 128, 16, [1, 2], [3000, 40]),                 # 20 rows of one token
]


def run_paged(case, e4m3, seed=70, scale=None, queries=None, even=False, **kw):
    Hq, H, D, page, new, lengths = case
    starts = starts_of(new)
    T = starts[-1]
    q = normal(seed, T, Hq, D) if queries is None else queries
    p = Pages(seed + 1, H, page, D, lengths, e4m3)
    scale = D ** -0.5 if scale is None else scale
    got = ef.attention_paged(q.cuda(), p.cache, p.dev_table, ints(lengths),
                             starts=None if even else ints(starts),
                             max_queries=None if even else max(new), scale=scale, **kw)
    torch.cuda.synchronize()
    args = (f64(q), p.values[0])
    ref = oracle.paged_attention_ref(*args, p.values[1], p.table, lengths, starts, scale)
    mag = oracle.paged_attention_ref(*args, np.abs(p.values[1]), p.table, lengths, starts, scale)
    close(got, ref, mag, case)
    return got


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", PAGED, ids=lambda c: str(c)[:60])
def test_paged(case, e4m3):
    announce(f"paged {case} e4m3 {e4m3}")
    run_paged(case, e4m3)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [0.0, -0.1])
def test_paged_scale(scale, e4m3):
    announce(f"paged scale {scale} {e4m3}")
    run_paged((8, 2, 128, 16, [2, 2], [300, 40]), e4m3, scale=scale)


def test_paged_even():
    announce("paged without starts")
    case = (8, 2, 128, 16, [3] * 4, [300, 40, 3, 1200])
    a, b = run_paged(case, False, even=True), run_paged(case, False)
    assert torch.equal(a, b)


# (Hq, Hkv, D, rows, keys or None for prompts, causal)
PACKED = [
    (1, 1, 64, [1], None, True),
    (4, 2, 128, [17, 1, 130], None, True),
    (4, 2, 128, [17, 1, 130], None, False),
    (32, 8, 128, [5, 0, 64, 33], [700, 9, 64, 20], True),     # fewer keys than rows
    (32, 8, 64, [5, 0, 64, 33], [700, 9, 0, 20], False),      # no keys
    (12, 4, 128, [100, 43], [1000, 43], True),
    (8, 2, 64, [300, 2, 77], None, True),
    (16, 16, 128, [260], [1500], True),                       # split keys
    (8, 1, 128, [3, 40], [9000, 2000], True),                 # few rows, many parts
    (8, 2, 128, [1] * 70, [1 + 37 * i % 300 for i in range(70)], True),   # over 64 sequences
    (4, 2, 64, [1 + 7 * i % 60 for i in range(100)], None, True),
    (64, 8, 64, [10, 900], [5000, 1200], True),
]


def run_packed(case, seed=80, scale=None, queries=None, **kw):
    Hq, H, D, new, keys, causal = case
    starts = starts_of(new)
    ks = starts if keys is None else starts_of(keys)
    q = normal(seed, starts[-1], Hq, D) if queries is None else queries
    k, v = normal(seed + 1, ks[-1], H, D), normal(seed + 2, ks[-1], H, D)
    scale = D ** -0.5 if scale is None else scale
    got = ef.attention_packed(q.cuda(), k.cuda(), v.cuda(), ints(starts),
                              None if keys is None else ints(ks), causal=causal, scale=scale, **kw)
    torch.cuda.synchronize()
    a = (f64(q), f64(k))
    ref = oracle.packed_attention_ref(*a, f64(v), starts, ks, scale, causal)
    mag = oracle.packed_attention_ref(*a, np.abs(f64(v)), starts, ks, scale, causal)
    close(got, ref, mag, case)
    return got


@pytest.mark.parametrize("case", PACKED, ids=lambda c: str(c)[:60])
def test_packed(case):
    announce(f"packed {case}")
    run_packed(case)


@pytest.mark.parametrize("scale", [0.0, -0.1])
def test_packed_scale(scale):
    announce(f"packed scale {scale}")
    run_packed((8, 2, 128, [40, 3], [300, 1000], True), scale=scale)

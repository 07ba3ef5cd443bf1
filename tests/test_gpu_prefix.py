"""Attention of a batch over a shared prefix on the GPU, against the fp64 oracle. The tolerance
is the one derived in long_helpers.py."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal, poison  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

# (B, Hq, Hkv, Sq, Lp, Skv, D, causal, lengths)
SHAPES = [
    (1, 1, 1, 1, 1, 1, 64, True, None),
    (1, 4, 2, 1, 100, 0, 128, True, None),           # no own keys
    (2, 4, 2, 3, 0, 50, 128, True, [50, 7]),         # no prefix
    (2, 4, 2, 3, 0, 0, 128, False, None),            # no keys at all
    (3, 8, 2, 1, 500, 300, 128, True, [300, 1, 64]),
    (5, 8, 2, 1, 64, 64, 64, False, [64, 0, 3, 63, 1]),
    (4, 12, 4, 2, 1000, 129, 128, True, [129, 2, 70, 128]),  # groups of 3
    (3, 12, 12, 5, 333, 40, 64, True, [40, 5, 3]),   # fewer own keys than queries
    (3, 4, 4, 6, 2, 9, 64, True, [0, 1, 9]),         # queries before the first key
    (40, 32, 8, 1, 3000, 200, 128, True, list(range(1, 201, 5))),
    (37, 8, 8, 3, 2000, 100, 64, True, None),        # packed rows of more than one tile
    (2, 64, 8, 16, 4000, 900, 128, True, [900, 100]),
    (3, 16, 2, 100, 700, 100, 128, True, None),
    (26, 32, 8, 30, 650, 30, 64, True, None),        # whole walks: rows fill the chip
    (24, 16, 8, 70, 333, 90, 128, True, [90 - i for i in range(24)]),
    (24, 16, 8, 64, 130, 64, 128, False, [64 - i for i in range(24)]),
    (2, 40, 10, 500, 77, 500, 64, True, [500, 20]),
    (1, 4, 2, 1, 70000, 70, 64, True, None),         # many partitions
]


def attend_prefix(shape, seed=50, scale=None, **kw):
    B, Hq, H, Sq, Lp, S, D, causal, n = shape
    q, k, v = (normal(seed + i, B, h, m, D) for i, (h, m) in
               enumerate(((Hq, Sq), (H, S), (H, S))))
    kp, vp = normal(seed + 3, H, Lp, D), normal(seed + 4, H, Lp, D)
    scale = D ** -0.5 if scale is None else scale
    got = ef.attention_shared_prefix(q.cuda(), kp.cuda(), vp.cuda(), poison(k, n), poison(v, n),
                                     scale=scale, causal=causal, lengths=lengths_of(n), **kw)
    torch.cuda.synchronize()
    a = [f64(t) for t in (q, kp, vp, k, v)]
    ref = oracle.shared_prefix_ref(*a, scale, causal, n)
    mag = oracle.shared_prefix_ref(a[0], a[1], np.abs(a[2]), a[3], np.abs(a[4]), scale, causal, n)
    close(got, ref, mag, shape)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: str(s)[:60])
def test_shared_prefix(shape):
    announce(f"shared_prefix {shape}")
    attend_prefix(shape)


@pytest.mark.parametrize("scale", [0.0, -0.1])
def test_scale(scale):
    announce(f"shared_prefix scale {scale}")
    attend_prefix((3, 8, 2, 2, 500, 300, 128, True, [300, 1, 64]), scale=scale)

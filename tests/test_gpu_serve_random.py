"""Attention over pages and of packed sequences on seeded random shapes: head layouts, pages, lengths,
new tokens, rows in front of and behind the sequences. Tolerance of long_helpers.py."""

import random

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, starts_of

pytestmark = pytest.mark.gpu


def shape(rng, most_new):
    H = rng.choice((1, 2, 3, 8))
    G = rng.choice((1, 2, 3, 4, 8, 16))
    D = rng.choice((64, 128))
    B = rng.choice((1, 2, 5, 17, 66))
    room = 6_000_000 // (H * G * B)  # pairs of a row and a key, for the oracle's sake
    new = [rng.choice((0, 1, 1, 2, rng.randint(1, most_new))) for _ in range(B)]
    lengths = []
    for n in new:
        most = max(2, min(6000, room // max(n, 1)))
        lengths.append(rng.choice((n, rng.randint(0, most), rng.randint(most // 2, most))))
    return H, G, D, new, lengths


@pytest.mark.parametrize("seed", range(14))
def test_paged(seed):
    rng = random.Random(900 + seed)
    H, G, D, new, lengths = shape(rng, 20)
    page, e4m3 = rng.choice((16, 32, 64, 128, 256)), rng.random() < 0.5
    starts = starts_of(new, rng.randrange(3))
    T = starts[-1] + rng.randrange(3)
    announce(f"paged random {seed}: {H} {G} {D} page {page} e4m3 {e4m3} {new} {lengths}")
    q = normal(seed, T, H * G, D)
    p = Pages(seed + 50, H, page, D, lengths, e4m3)
    out = torch.zeros_like(q.cuda())
    got = ef.attention_paged(q.cuda(), p.cache, p.dev_table, ints(lengths), starts=ints(starts),
                             max_queries=max(new), out=out)
    a = (f64(q), p.values[0])
    b = (p.table, lengths, starts, D ** -0.5)
    close(got, oracle.paged_attention_ref(*a, p.values[1], *b),
          oracle.paged_attention_ref(*a, np.abs(p.values[1]), *b), seed)


@pytest.mark.parametrize("seed", range(14))
def test_packed(seed):
    rng = random.Random(950 + seed)
    H, G, D, new, lengths = shape(rng, 300)
    causal = rng.random() < 0.7
    starts, ks = starts_of(new, rng.randrange(3)), starts_of(lengths, rng.randrange(3))
    announce(f"packed random {seed}: {H} {G} {D} causal {causal} {new} {lengths}")
    q = normal(seed, starts[-1] + rng.randrange(3), H * G, D)
    k, v = (normal(seed + 20 + i, ks[-1] + 1, H, D) for i in range(2))
    out = torch.zeros_like(q.cuda())
    got = ef.attention_packed(q.cuda(), k.cuda(), v.cuda(), ints(starts), ints(ks), causal=causal,
                              out=out)
    a = (f64(q), f64(k))
    b = (starts, ks, D ** -0.5, causal)
    close(got, oracle.packed_attention_ref(*a, f64(v), *b),
          oracle.packed_attention_ref(*a, np.abs(f64(v)), *b), seed)

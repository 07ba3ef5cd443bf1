"""A query that is not finite makes its rows NaN, whatever its scores are, where they see a key; a row
that sees none is 0; the rows of other queries are what they are without it. (An infinite element
against keys of one sign there gives scores that are all -inf.) Against the fp64 oracle, with the
tolerance of long_helpers.py."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
BAD = [INF, -INF, NAN]


def inputs(seed, B, Hq, H, Sq, S, D, one_sign):
    q, k, v = normal(seed, B, Hq, Sq, D), normal(seed + 1, B, H, S, D), normal(seed + 2, B, H, S, D)
    if one_sign:  # channel 5 of every key is above 0
        k[..., 5] = k[..., 5].abs() + 0.25
    return q, k, v


def spoil(q, rows, bad):
    q = q.clone()
    for b, h, i in rows:
        q[b, h, i, 5] = bad
    return q


def check(got, ref, mag, rows, sees, what):
    """rows: the spoilt ones; sees(b, h, i): whether the row sees a key."""
    good = np.ones(ref.shape[:3], bool)
    for b, h, i in rows:
        row = got[b, h, i]
        if sees(b, h, i):
            assert torch.isnan(row).all(), (what, b, h, i)
        else:
            assert (row == 0).all(), (what, b, h, i)
        good[b, h, i] = False
    close(got[torch.from_numpy(good).cuda()], ref[good], mag[good], what)


# (B, Hq, Hkv, Sq, Skv, D, block, topk, lengths, one_sign)
BLOCKS = [
    (1, 4, 4, 70, 70, 128, 64, 1, None, False),          # first queries see one key, two ...
    (2, 8, 2, 40, 900, 64, 64, 5, [900, 23], True),      # several parts; queries before the first key
    (1, 8, 2, 1, 3000, 128, 64, 20, None, True),         # parts, joined by the last of them
    (2, 8, 2, 5, 4000, 64, 128, 20, [4000, 130], True),  # parts, joined by a second kernel
    (1, 32, 32, 2050, 2050, 64, 64, 3, None, True),      # row tiles of 128, one part
    (1, 4, 2, 64, 64 * 700, 64, 64, 16, None, True),     # a union of more than one window
]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("shape", BLOCKS, ids=str)
def test_attention_blocks(shape, bad):
    announce(f"blocks, query {bad} {shape}")
    B, Hq, H, Sq, S, D, bs, K, n, one_sign = shape
    q, k, v = inputs(310, B, Hq, H, Sq, S, D, one_sign)
    nb = -(-S // bs)
    g = torch.Generator("cpu").manual_seed(313)
    lists = torch.rand(B, H, Sq, max(nb, K), generator=g).argsort(-1)[..., :K].to(torch.int32)
    lists = torch.where(lists < nb, lists, -1)
    lists[:, :, :, 0] = 0  # so that a query with a key sees one
    lists[:, 0, Sq // 3] = -1  # but for this one
    rows = {(0, 0, 0), (B - 1, Hq - 1, 0), (0, 1, Sq // 3), (B - 1, 0, Sq // 3), (0, 2, Sq - 1),
            (B - 1, 3, Sq // 2)}
    args = (f64(k), f64(v))
    scale = D ** -0.5
    ref = oracle.attention_blocks_ref(f64(q), *args, lists.numpy(), bs, scale, n)
    mag = oracle.attention_blocks_ref(f64(q), args[0], np.abs(args[1]), lists.numpy(), bs, scale, n)
    got = ef.attention_blocks(spoil(q, rows, bad).cuda(), k.cuda(), v.cuda(), lists.cuda(), bs,
                              lengths=lengths_of(n))
    torch.cuda.synchronize()
    length = [S] * B if n is None else n

    def sees(b, h, i):
        d = i + length[b] - Sq
        return d >= 0 and any(0 <= x <= d // bs for x in lists[b, h // (Hq // H), i].tolist())

    assert any(not sees(*r) for r in rows) and any(sees(*r) for r in rows)
    check(got, ref, mag, rows, sees, shape)


# (B, Hq, Hkv, Sq, Lp, Skv, D, causal, lengths, one_sign)
PREFIX = [
    (2, 4, 2, 40, 0, 40, 128, True, [40, 17], False),    # no prefix: first queries see one key
    (3, 4, 4, 6, 2, 9, 64, True, [0, 1, 9], False),      # queries before the first key
    (1, 4, 2, 1, 1, 0, 64, False, None, False),          # the prefix's one key
    (2, 4, 2, 3, 0, 50, 128, False, [0, 7], True),       # a sequence without keys
    (5, 8, 2, 1, 500, 300, 64, True, [300, 1, 64, 0, 7], True),  # parts of both
    (26, 32, 8, 30, 650, 30, 64, True, None, True),      # whole walks
]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("shape", PREFIX, ids=lambda s: str(s)[:60])
def test_shared_prefix(shape, bad):
    announce(f"prefix, query {bad} {shape}")
    B, Hq, H, Sq, Lp, S, D, causal, n, one_sign = shape
    q, k, v = inputs(320, B, Hq, H, Sq, S, D, one_sign)
    kp, vp = normal(323, H, Lp, D), normal(324, H, Lp, D)
    if one_sign:
        kp[..., 5] = kp[..., 5].abs() + 0.25
    rows = {(b, h, i) for b in range(min(B, 5)) for h, i in ((b % Hq, 0), ((b + 1) % Hq, Sq - 1),
                                                           ((b + 2) % Hq, Sq // 2))}
    a = [f64(t) for t in (q, kp, vp, k, v)]
    scale = D ** -0.5
    ref = oracle.shared_prefix_ref(*a, scale, causal, n)
    mag = oracle.shared_prefix_ref(a[0], a[1], np.abs(a[2]), a[3], np.abs(a[4]), scale, causal, n)
    got = ef.attention_shared_prefix(spoil(q, rows, bad).cuda(), kp.cuda(), vp.cuda(), k.cuda(),
                                     v.cuda(), causal=causal, lengths=lengths_of(n))
    torch.cuda.synchronize()
    length = [S] * B if n is None else n

    def sees(b, h, i):
        return Lp + i + length[b] - Sq >= 0 if causal else Lp + length[b] > 0

    check(got, ref, mag, rows, sees, shape)

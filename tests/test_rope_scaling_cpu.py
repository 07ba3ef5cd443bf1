"""Rotary frequencies scaled by the pair's number, where a border lies among the pairs or outside them.
No GPU is needed."""

import math

import pytest
import torch

from paper_2609_12330_amd import ef_attention as ef


def by_index(rot, base, factor, length, low, high):
    """The definition, pair by pair."""
    def number(turns):  # base^(-2 i / rot) length / 2 pi = turns
        return rot / 2 * math.log(length / (2 * math.pi * turns), base)

    first = min(max(math.floor(number(high)), 0), rot - 1)
    last = min(max(math.ceil(number(low)), 0), rot - 1)
    out = []
    for i in range(rot // 2):
        t = base ** (-2 * i / rot) / (2 * math.pi)
        if i <= first:
            out.append(t)
        elif i >= last:
            out.append(t / factor)
        else:
            part = (i - first) / (last - first)
            out.append(t * (1 - part) + t / factor * part)
    return out


CASES = [  # (rot, base, length, low, high)
    (128, 10000.0, 8192, 1.0, 32.0),     # both borders among the pairs
    (16, 10000.0, 32768, 1.0, 32.0),     # the lower one behind the last pair
    (32, 10000.0, 65536, 1.0, 32.0),
    (128, 10000.0, 65536, 1.0, 4.0),
    (128, 10000.0, 131072, 1.0, 4.0),
    (64, 10000.0, 10 ** 6, 1.0, 32.0),   # both behind it
    (64, 10000.0, 10 ** 9, 1.0, 32.0),   # the lower one at rot - 1
    (64, 500000.0, 100, 1.0, 32.0),      # the upper one in front of the first pair
]


@pytest.mark.parametrize("rot,base,length,low,high", CASES)
def test_index_scaling(rot, base, length, low, high):
    factor = 8.0
    got = ef.rope_turns(rot, base, scaling="index", factor=factor, length=length, low=low, high=high)
    want = torch.tensor(by_index(rot, base, factor, length, low, high), dtype=torch.float64)
    # (each entry is a power, a division and a sum or two in 64 bits)
    assert torch.allclose(got, want, rtol=1e-13, atol=0)
    plain = ef.rope_turns(rot, base)
    # Pairs that turn more than `low` times are not divided as a whole, ones that turn `high` times
    # or more not at all.
    assert (got > plain / factor * (1 + 1e-9))[length * plain > low].all()
    assert torch.equal(got[length * plain >= high], plain[length * plain >= high])


def test_index_scaling_of_the_last_pair():
    """rot 16, base 10000, length 32768: the last pair (7) turns 1.65 times; the borders are 4 (32
    turns) and 8 (one), so it keeps a quarter: 1/4 + 3/4 / 8."""
    t, s = ef.rope_turns(16), ef.rope_turns(16, scaling="index", factor=8.0, length=32768, low=1.0,
                                            high=32.0)
    assert 1.6 < 32768 * t[-1] < 1.7
    assert math.isclose(s[-1] / t[-1], 0.25 + 0.75 / 8, rel_tol=1e-12)


@pytest.mark.parametrize("base", [0.5, 0.999, 1.0])
def test_index_scaling_needs_falling_turns(base):
    """With a base below 1 later pairs turn more often and the borders change places."""
    with pytest.raises(ValueError, match="base > 1"):
        ef.rope_turns(16, base, scaling="index", factor=8.0, length=64, low=1.0, high=32.0)
    assert ef.rope_turns(16, base, scaling="turns", factor=8.0, length=64, low=1.0,
                         high=32.0).shape == (8,)

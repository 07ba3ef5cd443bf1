"""Block selection where few of the competing scores are numbers: a NaN score counts as -inf, so the
lists hold every block with a score and the lowest of the others. Against the fp64 oracle, for
equality."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu


def select_both(q, m, K, sinks, local):
    S, bs = 64 * m.shape[2], 64
    got = ef.block_select(q.cuda(), m.cuda(), S, K, bs, sinks, local)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref = oracle.block_select_ref(f64(q), f64(m), S, K, bs, sinks, local)
    got = got.cpu().numpy()
    bad = np.argwhere((got != ref).any(-1))
    if len(bad):
        at = tuple(bad[0])
        raise AssertionError(f"{len(bad)} lists differ, first {at}: {got[at]} want {ref[at]}")


# Competing blocks (of the last query; one fewer or as many for those before it): few to a lane
# and many, with and without lanes left over; wanted blocks: one to a lane, and more.
@pytest.mark.parametrize("rest", [40, 64, 65, 87, 100, 128, 256, 257, 300, 511, 700, 1024, 1025,
                                  1500, 2048])
@pytest.mark.parametrize("need", [1, 8, 64, 65, 200])
def test_few_scores_that_are_numbers(rest, need):
    if need >= rest:
        pytest.skip("all of them are taken")
    announce(f"select nan: {need} of {rest}")
    for numbers in sorted({0, 1, 3, need - 1, need, need + 1}):
        if not 0 <= numbers <= rest:
            continue
        q, m = normal(300, 1, 4, 2, 64), normal(301, 1, 2, rest + 3, 64)
        # Sink block 0, competing blocks 1 .. rest, the last two local. Numbers stand late.
        late = torch.linspace(rest * 0.8, rest, numbers).long() if numbers else []
        keep = torch.zeros(rest + 3, dtype=torch.bool)
        keep[late] = True
        m[:, :, ~keep, 7] = float("nan")
        select_both(q, m, need + 3, 1, 2)


def test_few_numbers_in_a_prompt():
    """Many queries, whose competing blocks grow from none on; both heads of a group and one head
    of it are NaN somewhere."""
    announce("select nan: prompt")
    q, m = normal(302, 2, 8, 1300, 64), normal(303, 2, 2, 400, 64)
    m[:, :, :390, 3] = float("nan")
    m[:, 0, [70, 75, 280]] = normal(304, 2, 3, 64)
    m[1, :, [9, 333], 5] = float("-inf")
    q[0, 5, 100:200, 1] = float("nan")
    q[1, :4, 1290:] = float("nan")
    select_both(q, m, 12, 1, 1)


@pytest.mark.parametrize("value", [0.0, -0.0, 3.0])
def test_equal_scores_and_nan(value):
    """Fewer numbers than wanted, all equal, of either sign of zero."""
    announce(f"select nan: equal {value}")
    q, m = normal(305, 1, 2, 3, 64).abs(), torch.full((1, 1, 150, 64), float("nan"))
    m = m.to(torch.bfloat16)
    m[:, :, [40, 41, 99, 130]] = value
    select_both(q, m, 10, 0, 1)

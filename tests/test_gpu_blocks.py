"""Block summaries, block selection and attention over selected blocks on the GPU, against the
fp64 oracle.

Tolerances. A summary is an fp32 sum rounded to bf16 once: half a step of the value (2^-8) plus
one rounding (2^-24) of a partial sum per key, each at most the sum of the keys' magnitudes. A
selection is compared for equality. The tolerance of the attention is derived at its test.
"""

import os
import sys

import numpy as np
import pytest
import torch

import oracle
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu


def announce(msg):
    print(f"[gpu case] {msg}", file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if not os.path.exists(ef.LIB_PATH):
        raise RuntimeError("libef_attention.so is not built; the HIP path must be present")
    ef.library()
    yield


def f64(t):
    return t.double().cpu().numpy()


def normal(seed, *shape):
    g = torch.Generator("cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16)


def lengths_of(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def same_lists(got, ref):
    """Raises with the first list that differs (and no more: they are long)."""
    got = got.cpu().numpy()
    assert got.shape == ref.shape
    bad = np.argwhere((got != ref).any(-1))
    if len(bad):
        at = tuple(bad[0])
        raise AssertionError(f"{len(bad)} lists differ, first {at}: {got[at]} want {ref[at]}")


# (B, Hkv, Skv, D, block, lengths)
SUMMARIES = [
    (1, 1, 1, 64, 64, None),
    (1, 2, 64, 128, 64, None),
    (2, 3, 65, 128, 64, None),
    (2, 2, 200, 64, 128, None),
    (3, 2, 1000, 128, 128, [1000, 0, 129]),
    (4, 1, 517, 64, 64, [1, 64, 517, 448]),
    (2, 2, 300, 128, 64, [-5, 4000]),  # clamped to [0, 300]
]


@pytest.mark.parametrize("shape", SUMMARIES, ids=str)
def test_summary(shape):
    B, H, S, D, bs, n = shape
    announce(f"summary {shape}")
    k = normal(3, B, H, S, D)
    kd = k.cuda()
    valid = [S] * B if n is None else [min(max(x, 0), S) for x in n]
    for b, m in enumerate(valid):  # what lies behind a length is not read
        kd[b, :, m:] = float("nan")
    got = ef.block_summary(kd, bs, lengths=lengths_of(n))
    torch.cuda.synchronize()
    ref = oracle.block_summary_ref(f64(k), bs, n)
    mag = oracle.block_summary_ref(np.abs(f64(k)), bs, n)
    assert got.shape == ref.shape
    tol = 2.0 ** -8 * np.abs(ref) + (bs + 2) * 2.0 ** -24 * mag
    assert (np.abs(f64(got) - ref) <= tol).all()


@pytest.mark.parametrize("new", [1, 2, 63, 64, 65, 130, 1000])
@pytest.mark.parametrize("bs", [64, 128])
def test_summary_of_the_last_keys(new, bs):
    """Only the blocks of the last `new` keys are written, the others keep what they hold."""
    announce(f"summary step new {new} block {bs}")
    B, H, S, D = 6, 2, 700, 128
    n = [700, 0, 1, 128, 129, 640]
    k = normal(4, B, H, S, D).cuda()
    full = ef.block_summary(k, bs, lengths=lengths_of(n))
    out = torch.full_like(full, 7.0)
    got = ef.block_summary(k, bs, lengths=lengths_of(n), new_keys=new, out=out)
    torch.cuda.synchronize()
    assert got is out
    want = torch.full_like(full, 7.0)
    for b, m in enumerate(n):
        for j in range(full.shape[2]):
            if j * bs < m and (j + 1) * bs > m - new:
                want[b, :, j] = full[b, :, j]
    assert torch.equal(got, want)


# (B, Hq, Hkv, Sq, Skv, D, block, topk, sinks, local, lengths)
SELECTS = [
    (1, 1, 1, 1, 1, 64, 64, 1, 0, 1, None),
    (1, 4, 4, 1, 640, 128, 64, 8, 1, 1, None),      # more blocks than topk
    (2, 8, 2, 1, 4096, 128, 64, 8, 1, 2, [4096, 1000]),
    (2, 8, 2, 5, 1500, 64, 128, 4, 0, 1, [1500, 3]),  # queries before the first key
    (1, 12, 4, 70, 3000, 128, 64, 16, 2, 3, None),  # groups of 3
    (1, 12, 2, 33, 2500, 64, 64, 13, 0, 1, None),   # groups of 6
    (1, 20, 1, 9, 2100, 128, 64, 9, 1, 1, None),    # groups of 20, two column tiles
    (1, 32, 1, 3, 5000, 64, 64, 32, 1, 2, None),    # groups of 32
    (1, 3, 3, 130, 2000, 128, 64, 5, 4, 1, None),   # every choice forced
    (2, 4, 2, 2000, 2000, 64, 64, 7, 1, 1, None),   # four column tiles
    (1, 16, 16, 300, 2000, 128, 128, 6, 1, 1, None),
    (1, 4, 2, 40, 33000, 128, 64, 256, 1, 1, None),  # the longest list
    (1, 2, 1, 2, 1023999, 64, 64, 40, 1, 2, None),  # as many blocks as there may be
]


@pytest.mark.parametrize("shape", SELECTS, ids=str)
def test_select(shape):
    B, Hq, H, Sq, S, D, bs, K, sinks, local, n = shape
    announce(f"select {shape}")
    q = normal(5, B, Hq, Sq, D)
    m = normal(6, B, H, -(-S // bs), D)
    got = ef.block_select(q.cuda(), m.cuda(), S, K, bs, sinks, local, lengths=lengths_of(n))
    torch.cuda.synchronize()
    assert got.dtype == torch.int32
    ref = oracle.block_select_ref(f64(q), f64(m), S, K, bs, sinks, local, n)
    same_lists(got, ref)


def test_select_where_fp32_cannot_tell():
    """Summaries that differ by less than fp32 holds of the score: only their exact products
    tell the blocks apart, and equal ones go by index."""
    announce("select near ties")
    B, Hq, H, Sq, S, D, bs, K = 2, 8, 2, 6, 64 * 200, 128, 64, 20
    q = normal(7, B, Hq, Sq, D)
    m = normal(8, B, H, 1, D).repeat(1, 1, 200, 1)
    g = torch.Generator("cpu").manual_seed(9)
    # One element of each block is its own and tiny: the scores agree to about 2^-24.
    m[..., :32] = 0
    at = torch.randint(0, 32, (B, H, 200), generator=g)
    tiny = (torch.randn(B, H, 200, generator=g) * 2.0 ** -22).to(torch.bfloat16)
    m.scatter_(3, at[..., None], tiny[..., None])
    m[:, :, 50:60] = m[:, :, 40:50]
    m[:, :, 100:] = m[:, :, :100].flip(2)
    ref = oracle.block_select_ref(f64(q), f64(m), S, K, bs, 1, 2)
    got = ef.block_select(q.cuda(), m.cuda(), S, K, bs, 1, 2)
    torch.cuda.synchronize()
    same_lists(got, ref)


@pytest.mark.parametrize("what", ["zero_q", "zero_summary", "equal", "nan_q", "nan_summary",
                                  "inf_summary", "negative", "tiny", "huge"])
def test_select_degenerate(what):
    announce(f"select {what}")
    B, Hq, H, Sq, S, D, bs, K = 1, 4, 2, 37, 64 * 90, 64, 64, 10
    q, m = normal(10, B, Hq, Sq, D), normal(11, B, H, 90, D)
    if what == "zero_q":
        q[:, :, ::2] = 0
    elif what == "zero_summary":
        m[:] = 0
    elif what == "equal":
        m[:] = m[:, :, :1].clone()
    elif what == "nan_q":
        q[:, 1, 3] = float("nan")
        q[:, :, 5] = float("nan")
    elif what == "nan_summary":
        m[:, :, ::3, 5] = float("nan")
    elif what == "inf_summary":
        m[:, 0, 4, 3] = float("inf")
        m[:, 1, 7, 3] = float("-inf")
    elif what == "negative":
        q, m = q.abs(), -m.abs()
    elif what == "tiny":
        q, m = q * 2.0 ** -60, m * 2.0 ** -60
    else:
        q, m = q * 2.0 ** 55, m * 2.0 ** 55
    got = ef.block_select(q.cuda(), m.cuda(), S, K, bs, 1, 1)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref = oracle.block_select_ref(f64(q), f64(m), S, K, bs, 1, 1)
    same_lists(got, ref)

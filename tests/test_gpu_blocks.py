"""Block summaries, block selection and attention over selected blocks on the GPU, against the
fp64 oracle.

Tolerances. A summary is an fp32 sum rounded to bf16 once: half a step of the value (2^-8) plus
one rounding (2^-24) of a partial sum per key, each at most the sum of the keys' magnitudes. A
selection is compared for equality. The tolerance of the
attention is derived in long_helpers.py.
"""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal, poison  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu


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
    (2, 4, 2, 2000, 2000, 64, 64, 7, 1, 1, None),
    (2, 16, 2, 2000, 9000, 64, 64, 7, 1, 1, None),  # four column tiles
    (3, 8, 2, 1403, 9000, 128, 64, 9, 0, 1, [9000, 1403, 5000]),
    (1, 4, 2, 9, 100000, 128, 64, 16, 1, 2, None),  # scores that stay in LDS
    (1, 4, 2, 5, 80000, 64, 64, 200, 2, 1, None),   # ... with a long list
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


@pytest.mark.parametrize("junk", [float("inf"), float("nan"), 1e30])
def test_select_does_not_read_the_last_summaries(junk):
    """What stands in the summaries of the local blocks and behind the sequence does not matter."""
    announce(f"select junk {junk}")
    B, Hq, H, Sq, S, D, bs, K, local = 2, 8, 2, 1, 64 * 100, 128, 64, 12, 2
    n = [64 * 70 + 5, 64 * 100]
    q, m = normal(14, B, Hq, Sq, D), normal(15, B, H, 100, D)
    ref = oracle.block_select_ref(f64(q), f64(m), S, K, bs, 1, local, n)
    for b, x in enumerate(n):
        m[b, :, (x - 1) // bs + 1 - local:] = junk
    got = ef.block_select(q.cuda(), m.cuda(), S, K, bs, 1, local, lengths=lengths_of(n))
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


# ------------------------------------------------------------------------------- attention


def random_lists(seed, B, H, Sq, K, nb, junk=False):
    """Distinct blocks of [0, nb) in random order; with junk also repeats, -1 and blocks that do
    not exist."""
    g = torch.Generator("cpu").manual_seed(seed)
    x = torch.rand(B, H, Sq, max(nb, K), generator=g).argsort(-1)[..., :K].to(torch.int32)
    x = torch.where(x < nb, x, -1)
    if junk and K > 3:
        x[..., 1] = x[..., 0]
        x[..., 2] = nb + 5
        x[..., 3] = -7
    return x.contiguous()


# (B, Hq, Hkv, Sq, Skv, D, block, topk, lengths, junk)
ATTENTION = [
    (1, 1, 1, 1, 1, 64, 64, 1, None, False),
    (1, 4, 1, 1, 63, 128, 64, 3, None, False),
    (2, 8, 2, 1, 1000, 128, 64, 5, [1000, 65], False),
    (3, 8, 2, 1, 2000, 64, 128, 7, [2000, 0, 129], True),
    (2, 4, 4, 7, 900, 128, 64, 4, [900, 3], True),     # queries before the first key
    (1, 12, 4, 50, 1200, 128, 64, 6, None, False),     # groups of 3: tiles cut positions
    (1, 12, 2, 40, 777, 64, 128, 3, None, True),       # groups of 6
    (2, 6, 6, 130, 1500, 64, 64, 8, [1500, 200], False),  # 64 positions to a tile
    (1, 8, 2, 200, 200, 128, 64, 2, None, False),
    (1, 64, 1, 3, 1111, 128, 64, 9, None, False),      # groups of 64
    (1, 2, 2, 64, 64 * 700, 64, 64, 16, None, False),  # a union of more than one window
    (1, 2, 2, 3, 64 * 1500, 64, 64, 250, None, False),  # ... and split over workgroups
    (1, 4, 4, 150, 128 * 300, 128, 128, 12, None, True),
    (1, 32, 32, 2048, 2100, 64, 64, 4, None, True),    # 128 positions to a tile
    (2, 16, 16, 2049, 2100, 128, 128, 3, [2100, 2060], False),
    (1, 64, 32, 1030, 4000, 64, 64, 9, None, False),   # 64 positions to a tile of 128 rows
]


def attend_blocks(shape, seed=20, scale=None, lists=None):
    B, Hq, H, Sq, S, D, bs, K, n, junk = shape
    q, k, v = normal(seed, B, Hq, Sq, D), normal(seed + 1, B, H, S, D), normal(seed + 2, B, H, S, D)
    if lists is None:
        lists = random_lists(seed + 3, B, H, Sq, K, -(-S // bs), junk)
    scale = D ** -0.5 if scale is None else scale
    got = ef.attention_blocks(q.cuda(), poison(k, n), poison(v, n), lists.cuda(), bs, scale=scale,
                              lengths=lengths_of(n))
    torch.cuda.synchronize()
    args = (f64(q), f64(k), f64(v))
    ref = oracle.attention_blocks_ref(*args, lists.numpy(), bs, scale, n)
    mag = oracle.attention_blocks_ref(*args[:2], np.abs(args[2]), lists.numpy(), bs, scale, n)
    close(got, ref, mag, shape)
    return got, ref


@pytest.mark.parametrize("shape", ATTENTION, ids=str)
def test_attention_blocks(shape):
    announce(f"attention_blocks {shape}")
    attend_blocks(shape)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_attention_blocks_scale(scale):
    announce(f"attention_blocks scale {scale}")
    # A scale of 1 makes scores of up to 11 sqrt(128) = 128: their error grows with it, and the
    # weights' with them by e^(1.5e-5 * 1.6 * 128) - 1 = 3e-3: the tolerance's 1e-3 is too small
    # for D = 128, so D = 64 and short keys (|q| |k| of about 64 / 4).
    B, Hq, H, Sq, S, D = 1, 8, 2, 20, 700, 64
    q, k, v = normal(30, B, Hq, Sq, D), normal(31, B, H, S, D) / 4, normal(32, B, H, S, D)
    lists = random_lists(33, B, H, Sq, 6, 11)
    got = ef.attention_blocks(q.cuda(), k.cuda(), v.cuda(), lists.cuda(), 64, scale=scale)
    torch.cuda.synchronize()
    args = (f64(q), f64(k))
    ref = oracle.attention_blocks_ref(*args, f64(v), lists.numpy(), 64, scale)
    mag = oracle.attention_blocks_ref(*args, np.abs(f64(v)), lists.numpy(), 64, scale)
    close(got, ref, mag, scale)


def test_attention_blocks_without_blocks():
    """Empty lists, and lists of blocks behind the query only, give zero rows."""
    announce("attention_blocks empty lists")
    B, Hq, H, Sq, S, D, K = 2, 4, 2, 9, 640, 128, 4
    q, k = normal(34, B, Hq, Sq, D).cuda(), normal(35, B, H, S, D).cuda()
    lists = torch.full((B, H, Sq, K), -1, dtype=torch.int32, device="cuda")
    lists[0] = 9  # keys 576 .. 639: of sequence 0 only the last query sees one, key 576
    n = torch.tensor([577, 640], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    ef.attention_blocks(q, k, k, lists, lengths=n, out=out)
    torch.cuda.synchronize()
    assert (out[0, :, :-1] == 0).all() and (out[1] == 0).all()
    assert torch.equal(out[0, :, -1], k[0, :, 576].repeat_interleave(Hq // H, 0))


def test_all_blocks_is_plain_causal_attention():
    announce("attention_blocks against attention_fwd")
    B, Hq, H, Sq, S, D = 1, 8, 2, 300, 1500, 128
    q, k, v = (normal(40 + i, B, h, n, D).cuda() for i, (h, n) in
               enumerate(((Hq, Sq), (H, S), (H, S))))
    every = torch.arange(24, dtype=torch.int32, device="cuda").expand(B, H, Sq, 24).contiguous()
    got = ef.attention_blocks(q, k, v, every)
    ref = ef.attention_fwd(q, k, v, causal=True)
    mag = ef.attention_fwd(q, k, v.abs(), causal=True)
    torch.cuda.synchronize()
    # Both round the weights: twice the tolerance of one.
    close(got, f64(ref), 2 * f64(mag), "plain")


def test_refused_tensors():
    """Shapes, types and strides that do not fit are refused before anything is enqueued."""
    announce("refused tensors")
    bf = torch.bfloat16
    q, k = (torch.zeros(1, h, n, 64, dtype=bf, device="cuda") for h, n in ((4, 2), (2, 100)))
    lists = torch.zeros(1, 2, 2, 3, dtype=torch.int32, device="cuda")
    m = torch.zeros(1, 2, 2, 64, dtype=bf, device="cuda")
    kp = torch.zeros(2, 30, 64, dtype=bf, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    for exc, call in (
            (ValueError, lambda: ef.block_summary(k.transpose(1, 2))),
            (ValueError, lambda: ef.block_summary(k, 32)),
            (ValueError, lambda: ef.block_summary(k, new_keys=1)),
            (ValueError, lambda: ef.block_summary(k, out=m[:, :1].contiguous())),
            (TypeError, lambda: ef.block_summary(k, lengths=n.long())),
            (ValueError, lambda: ef.block_summary(k, lengths=n.repeat(2))),
            (TypeError, lambda: ef.block_summary(k, lengths=n.cpu())),
            (ef.EfError, lambda: ef.block_summary(k, new_keys=-1, out=m)),
            (ValueError, lambda: ef.block_select(q, m, 200, 3)),
            (ef.EfError, lambda: ef.block_select(q, m, 100, 1, sink_blocks=1)),
            (ef.EfError, lambda: ef.block_select(q, m, 100, 257)),
            (TypeError, lambda: ef.block_select(q, m, 100, 3, out=lists.long())),
            (TypeError, lambda: ef.attention_blocks(q, k, k, lists.long())),
            (ValueError, lambda: ef.attention_blocks(q, k, k, lists[:, :, :1].contiguous())),
            (ValueError, lambda: ef.attention_blocks(q, k, k[:, :, :50].contiguous(), lists)),
            (TypeError, lambda: ef.attention_blocks(q, k, k, lists, out=q.float())),
            (ef.EfError, lambda: ef.attention_blocks(q, k, k, lists, block_size=96)),
            (ef.EfError, lambda: ef.attention_blocks(q, k, k, lists, scale=float("nan"))),
            (ef.EfError, lambda: ef.attention_blocks(q, k, k, lists, workspace=n.byte())),
            (ValueError, lambda: ef.attention_shared_prefix(q, kp[:1].contiguous(), kp, k, k)),
            (ValueError, lambda: ef.attention_shared_prefix(q, kp, kp[:, :9].contiguous(), k, k)),
            (ef.EfError, lambda: ef.attention_shared_prefix(q, kp, kp, k, k, workspace=n))):
        with pytest.raises(exc):
            call()
    torch.cuda.synchronize()

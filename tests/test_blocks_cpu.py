"""The long-context entry points on the CPU: every refusal is made on the host before any HIP
call, and their oracle is pinned by closed forms and by the plain attention oracle."""

import os

import numpy as np
import pytest

import oracle
from paper_2609_12330_amd import ef_attention as ef

needs_lib = pytest.mark.skipif(not os.path.exists(ef.LIB_PATH),
                               reason="libef_attention.so not built")

# Fake device addresses: non-null, 16-byte aligned; never dereferenced on these paths.
A = 0x10000
MIS = 0x10008


def summary(**kw):
    a = dict(k=A, n=None, s=A, B=1, Hkv=2, Skv=100, D=128, bs=64, new=0)
    a.update(kw)
    return ef.ef_block_summary(a["k"], a["n"], a["s"], a["B"], a["Hkv"], a["Skv"], a["D"],
                               a["bs"], a["new"], None)


def select(**kw):
    a = dict(q=A, s=A, n=None, o=A, B=1, Hq=4, Hkv=2, Sq=3, Skv=1000, D=128, bs=64, K=8, sinks=1,
             local=2)
    a.update(kw)
    return ef.ef_block_select(a["q"], a["s"], a["n"], a["o"], a["B"], a["Hq"], a["Hkv"], a["Sq"],
                              a["Skv"], a["D"], a["bs"], a["K"], a["sinks"], a["local"], None)


def blocks(**kw):
    a = dict(q=A, k=A, v=A, x=A, n=None, o=A, B=1, Hq=4, Hkv=2, Sq=3, Skv=1000, D=128, scale=0.1,
             bs=64, K=8, ws=A, wsb=1 << 40)
    a.update(kw)
    return ef.ef_attention_blocks(a["q"], a["k"], a["v"], a["x"], a["n"], a["o"], a["B"], a["Hq"],
                                  a["Hkv"], a["Sq"], a["Skv"], a["D"], a["scale"], a["bs"],
                                  a["K"], a["ws"], a["wsb"], None)


def prefix(**kw):
    a = dict(q=A, kp=A, vp=A, k=A, v=A, n=None, o=A, B=2, Hq=4, Hkv=2, Sq=3, Lp=500, Skv=1000,
             D=128, scale=0.1, causal=1, ws=A, wsb=1 << 40)
    a.update(kw)
    return ef.ef_attention_shared_prefix(a["q"], a["kp"], a["vp"], a["k"], a["v"], a["n"], a["o"],
                                         a["B"], a["Hq"], a["Hkv"], a["Sq"], a["Lp"], a["Skv"],
                                         a["D"], a["scale"], a["causal"], a["ws"], a["wsb"], None)


@needs_lib
@pytest.mark.parametrize("call", [summary, select, blocks, prefix],
                         ids=["summary", "select", "blocks", "prefix"])
def test_refusals(call):
    assert call(D=96) == 4
    assert call(B=-1) == 2
    assert call(Hkv=0) == 2
    assert call(Skv=-1) == 2
    assert call(B=70000) == 2
    assert call(Skv=2**24, D=128) == 2


@needs_lib
@pytest.mark.parametrize("call", [summary, select, blocks], ids=["summary", "select", "blocks"])
def test_refused_blocks(call):
    assert call(bs=32) == 14
    assert call(bs=0) == 14
    assert call(bs=-64) == 14
    assert call(Skv=64 * 16000 + 1) == 14
    assert call(Skv=128 * 16000 + 1, bs=128) == 14


@needs_lib
def test_refusals_of_their_own():
    assert summary(k=None) == 1
    assert summary(s=None) == 1
    assert summary(k=MIS) == 5
    assert summary(s=MIS) == 5
    assert summary(new=-1) == 14
    assert summary(B=0, k=None, s=None) == 0
    assert summary(Skv=0, k=None, s=None) == 0
    assert select(Hq=5) == 3
    assert select(Sq=-1) == 2
    assert select(q=None) == 1
    assert select(s=None) == 1
    assert select(o=None) == 1
    assert select(q=MIS) == 5
    assert select(s=MIS) == 5
    assert select(o=MIS) == 5
    assert select(K=0) == 14
    assert select(K=257) == 14
    assert select(K=2) == 14
    assert select(sinks=-1) == 14
    assert select(local=0) == 14
    assert select(sinks=2**31 - 1, local=2**31 - 1) == 14
    assert select(Sq=0, q=None, o=None) == 0
    assert ef.library().ef_status_string(14) != b"unknown status"


@needs_lib
@pytest.mark.parametrize("call", [blocks, prefix], ids=["blocks", "prefix"])
def test_refused_attention(call):
    assert call(Hq=5) == 3
    assert call(Hq=0) == 2
    assert call(Sq=-1) == 2
    assert call(Sq=2**24) == 2
    # Rows of the whole batch are counted in 32 bits.
    assert call(B=512, Hq=64, Hkv=64, Sq=2**16) == 2
    for name in ("q", "k", "v", "o"):
        assert call(**{name: None}) == 1
        assert call(**{name: MIS}) == 5
    assert call(scale=float("nan")) == 8
    assert call(scale=float("inf")) == 8
    assert call(ws=None) == 7
    assert call(wsb=100) == 7
    assert call(ws=MIS) == 5
    assert call(B=0, q=None, k=None, v=None, o=None, ws=None) == 0
    assert call(Sq=0, q=None, k=None, v=None, o=None, ws=None) == 0


@needs_lib
def test_refused_lists_and_prefixes():
    assert blocks(x=None) == 1
    assert blocks(x=MIS) == 5
    assert blocks(K=0) == 14
    assert blocks(K=257) == 14
    assert prefix(Lp=-1) == 2
    assert prefix(Lp=2**24) == 2
    assert prefix(kp=None) == 1
    assert prefix(vp=None) == 1
    assert prefix(kp=MIS) == 5
    assert prefix(vp=MIS) == 5


@needs_lib
def test_workspace_sizes():
    size = ef.ef_attention_blocks_workspace_size
    assert size(1, 4, 2, 3, 1000, 96, 64, 8) == 0
    assert size(1, 4, 2, 3, 1000, 128, 65, 8) == 0
    assert size(1, 4, 2, 3, 1000, 128, 64, 0) == 0
    assert size(0, 4, 2, 3, 1000, 128, 64, 8) == 0
    assert size(1, 4, 2, 1, 1000, 128, 64, 1) == 0     # one block: nothing to share
    assert size(1, 32, 8, 4096, 8192, 128, 64, 16) == 0  # row tiles fill the chip
    n = size(1, 32, 8, 1, 16384, 128, 64, 16)
    assert n > 0
    assert blocks(B=1, Hq=32, Hkv=8, Sq=1, Skv=16384, K=16, wsb=n - 1) == 7
    size = ef.ef_attention_shared_prefix_workspace_size
    assert size(2, 4, 2, 3, 500, 1000, 96) == 0
    assert size(2, 4, 2, 3, -1, 1000, 128) == 0
    assert size(2, 4, 2, 3, 0, 0, 128) == 0
    n = size(2, 4, 2, 3, 500, 1000, 128)
    assert n > 0
    assert prefix(wsb=n - 1) == 7


def test_oracle_summary_and_selection():
    k = np.arange(10.0).reshape(1, 1, 10, 1) * np.ones((1, 1, 10, 3))
    m = oracle.block_summary_ref(k, 4, [9])
    assert np.array_equal(m[0, 0, :, 0], [1.5, 5.5, 8.0])
    assert np.array_equal(oracle.block_summary_ref(k, 4, [0]), np.zeros((1, 1, 3, 3)))
    # Six blocks of four keys, one head pair; the score of a block is its larger product.
    q = np.array([[1.0, 0.0], [0.0, 1.0]]).reshape(1, 2, 1, 2)
    s = np.array([[0, 0], [3, -9], [1, 3], [2, 2], [5, 5], [0, 0]], float).reshape(1, 1, 6, 2)
    assert oracle.block_select_ref(q, s, 24, 3, 4, 1, 1).tolist() == [[[[0, 4, 5]]]]
    assert oracle.block_select_ref(q, s, 24, 4, 4, 1, 1).tolist() == [[[[0, 1, 4, 5]]]]  # tie: 1
    assert oracle.block_select_ref(q, s, 24, 3, 4, 0, 1, [9]).tolist() == [[[[0, 1, 2]]]]
    assert oracle.block_select_ref(q, s, 24, 3, 4, 1, 2, [20]).tolist() == [[[[0, 3, 4]]]]
    assert oracle.block_select_ref(q, s, 24, 3, 4, 1, 2, [0]).tolist() == [[[[-1, -1, -1]]]]


def test_oracle_attention_agrees_with_the_plain_one():
    rng = np.random.default_rng(0)
    B, Hq, H, Sq, S, Lp, D = 2, 4, 2, 5, 37, 19, 64
    q, k, v = (rng.standard_normal((B, h, n, D)) for h, n in ((Hq, Sq), (H, S), (H, S)))
    every = np.broadcast_to(np.arange(3), (B, H, Sq, 3))
    full = oracle.attention_ref(q, k, v, 0.2, True)
    assert np.allclose(oracle.attention_blocks_ref(q, k, v, every, 16, 0.2), full, atol=1e-12)
    assert np.array_equal(
        oracle.attention_blocks_ref(q, k, v, np.full((B, H, Sq, 2), -1), 16, 0.2), 0 * q)
    kp, vp = (rng.standard_normal((H, Lp, D)) for _ in range(2))
    kk = np.concatenate([np.broadcast_to(kp, (B, H, Lp, D)), k], 2)
    vv = np.concatenate([np.broadcast_to(vp, (B, H, Lp, D)), v], 2)
    for causal in (False, True):
        assert np.allclose(oracle.shared_prefix_ref(q, kp, vp, k, v, 0.2, causal),
                           oracle.attention_ref(q, kk, vv, 0.2, causal), atol=1e-12)
    short = oracle.shared_prefix_ref(q, kp, vp, k, v, 0.2, True, [30, 2])
    assert np.allclose(short[0], oracle.attention_ref(q[:1], kk[:1, :, :49], vv[:1, :, :49], 0.2,
                                                      True)[0], atol=1e-12)


def test_tensors_that_are_refused():
    """The torch-level calls check their tensors before the library sees them."""
    import torch
    bf = torch.bfloat16
    q, k = torch.zeros(1, 4, 2, 64, dtype=bf), torch.zeros(1, 2, 100, 64, dtype=bf)
    lists = torch.zeros(1, 2, 2, 3, dtype=torch.int32)
    m = torch.zeros(1, 2, 2, 64, dtype=bf)
    kp = torch.zeros(2, 30, 64, dtype=bf)
    for call in (lambda: ef.block_summary(k), lambda: ef.block_select(q, m, 100, 3),
                 lambda: ef.attention_blocks(q, k, k, lists),
                 lambda: ef.attention_shared_prefix(q, kp, kp, k, k)):
        with pytest.raises(TypeError, match="GPU"):
            call()
    for call in (lambda: ef.block_summary(k.float()), lambda: ef.block_select(q.half(), m, 100, 3),
                 lambda: ef.attention_blocks(q.float(), k, k, lists),
                 lambda: ef.attention_shared_prefix(q.float(), kp, kp, k, k)):
        with pytest.raises(TypeError, match="bfloat16"):
            call()

"""The serving operators on the CPU: what the entry points refuse, workspace sizes, frequencies of
rotary positions, and the oracle against other formulations. No call here reaches a GPU."""

import math
import os

import numpy as np
import pytest
import torch

import oracle
from paper_2609_12330_amd import ef_attention as ef

needs_lib = pytest.mark.skipif(not os.path.exists(ef.LIB_PATH),
                               reason="libef_attention.so not built")
A, MIS, MIS4 = 0x10000, 0x10008, 0x10002  # fake device addresses, never dereferenced


def rope(**kw):
    a = dict(x=A, positions=A, turns=A, out=A, T=4, H=8, D=128, rot=128, interleaved=0,
             amplitude=1.0, transpose=0, stream=None)
    a.update(kw)
    return ef.ef_rope(*a.values())


def write(**kw):
    a = dict(k=A, v=A, q=A, turns=A, k_cache=A, v_cache=A, k_scale=None, v_scale=None, table=A,
             lengths=A, starts=A, q_out=A, T=6, B=3, Hq=8, Hkv=2, D=128, pages=9, page=16, width=4,
             format=0, rot=64, interleaved=0, amplitude=1.0, stream=None)
    a.update(kw)
    return ef.ef_cache_write(*a.values())


def read(**kw):
    a = dict(k_cache=A, v_cache=A, k_scale=None, v_scale=None, table=A, starts=A, k_out=A, v_out=A,
             T=6, B=3, Hkv=2, D=128, pages=9, page=16, width=4, format=0, stream=None)
    a.update(kw)
    return ef.ef_cache_read(*a.values())


def paged(**kw):
    a = dict(q=A, k_cache=A, v_cache=A, k_scale=None, v_scale=None, table=A, lengths=A, starts=A,
             o=A, T=6, B=3, Hq=8, Hkv=2, D=128, max_queries=2, pages=9, page=16, width=4, format=0,
             scale=0.1, ws=A, wsb=1 << 30, stream=None)
    a.update(kw)
    return ef.ef_attention_paged(*a.values())


def packed(**kw):
    a = dict(q=A, k=A, v=A, starts=A, k_starts=A, o=A, T=6, Tk=5000, B=3, Hq=8, Hkv=2, D=128,
             scale=0.1, causal=1, ws=A, wsb=1 << 30, stream=None)
    a.update(kw)
    return ef.ef_attention_packed(*a.values())


NULL, SHAPE, GQA, DIM, MISAL, WS, SCALE, PAGES, ROPE = 1, 2, 3, 4, 5, 7, 8, 15, 16

REFUSED = [
    (rope, dict(x=None), NULL), (rope, dict(positions=None), NULL), (rope, dict(turns=None), NULL),
    (rope, dict(out=None), NULL), (rope, dict(T=-1), SHAPE), (rope, dict(H=0), SHAPE),
    (rope, dict(D=96), DIM), (rope, dict(D=64), ROPE), (rope, dict(rot=0), ROPE),
    (rope, dict(rot=24), ROPE), (rope, dict(amplitude=math.inf), ROPE),
    (rope, dict(amplitude=math.nan), ROPE), (rope, dict(x=MIS), MISAL), (rope, dict(out=MIS), MISAL),
    (rope, dict(turns=MIS), MISAL), (rope, dict(positions=MIS4), MISAL),
    (rope, dict(T=2 ** 30, H=4), SHAPE),
    (write, dict(k=None), NULL), (write, dict(v=None), NULL), (write, dict(q=None), NULL),
    (write, dict(q_out=None), NULL), (write, dict(k_cache=None), NULL),
    (write, dict(v_cache=None), NULL), (write, dict(table=None), NULL),
    (write, dict(lengths=None), NULL), (write, dict(format=1), NULL),
    (write, dict(format=1, k_scale=A), NULL), (write, dict(format=1, k_scale=A, v_scale=MIS), MISAL),
    (write, dict(format=2), PAGES), (write, dict(page=8), PAGES), (write, dict(page=48), PAGES),
    (write, dict(page=512), PAGES), (write, dict(pages=0), PAGES), (write, dict(width=-1), PAGES),
    (write, dict(width=2 ** 27), PAGES), (write, dict(rot=40), ROPE), (write, dict(rot=144), ROPE),
    (write, dict(amplitude=math.nan), ROPE), (write, dict(Hq=7), GQA), (write, dict(Hq=-8), SHAPE),
    (write, dict(Hkv=0), SHAPE), (write, dict(D=32), DIM), (write, dict(T=-6), SHAPE),
    (write, dict(B=-1), SHAPE), (write, dict(starts=None, T=7), SHAPE), (write, dict(k=MIS), MISAL),
    (write, dict(q=MIS), MISAL), (write, dict(k_cache=MIS), MISAL), (write, dict(table=MIS4), MISAL),
    (write, dict(lengths=MIS4), MISAL), (write, dict(starts=MIS4), MISAL),
    (write, dict(T=3, Hq=65535 * 32767, Hkv=65535), SHAPE),  # more rows of a token than are counted
    (read, dict(k_cache=None), NULL), (read, dict(starts=None), NULL), (read, dict(k_out=None), NULL),
    (read, dict(v_out=None), NULL), (read, dict(table=None), NULL), (read, dict(format=1), NULL),
    (read, dict(page=20), PAGES), (read, dict(pages=-1), PAGES), (read, dict(D=100), DIM),
    (read, dict(T=-1), SHAPE), (read, dict(v_out=MIS), MISAL), (read, dict(starts=MIS4), MISAL),
    (paged, dict(q=None), NULL), (paged, dict(o=None), NULL), (paged, dict(lengths=None), NULL),
    (paged, dict(k_cache=None), NULL), (paged, dict(table=None), NULL), (paged, dict(format=1), NULL),
    (paged, dict(max_queries=-1), SHAPE), (paged, dict(starts=None, T=7), SHAPE),
    (paged, dict(starts=None, max_queries=1), SHAPE), (paged, dict(Hq=9), GQA),
    (paged, dict(D=256), DIM), (paged, dict(page=1), PAGES), (paged, dict(format=-1), PAGES),
    (paged, dict(scale=math.inf), SCALE), (paged, dict(scale=math.nan), SCALE),
    (paged, dict(ws=None), WS), (paged, dict(wsb=1000), WS), (paged, dict(ws=MIS), MISAL),
    (paged, dict(o=MIS), MISAL), (paged, dict(lengths=MIS4), MISAL),
    (paged, dict(B=2 ** 20, T=2 ** 20, width=2 ** 20), SHAPE),  # more units of work than are counted
    (packed, dict(q=None), NULL), (packed, dict(k=None), NULL), (packed, dict(v=None), NULL),
    (packed, dict(o=None), NULL), (packed, dict(starts=None), NULL),
    (packed, dict(k_starts=None), NULL), (packed, dict(Tk=-1), SHAPE), (packed, dict(T=-1), SHAPE),
    (packed, dict(Hq=3), GQA), (packed, dict(D=80), DIM), (packed, dict(scale=math.nan), SCALE),
    (packed, dict(ws=None), WS), (packed, dict(wsb=10), WS), (packed, dict(ws=MIS), MISAL),
    (packed, dict(k=MIS), MISAL), (packed, dict(starts=MIS4), MISAL),
    (packed, dict(k_starts=MIS4), MISAL), (packed, dict(Hkv=70000, Hq=70000), SHAPE),
]


@needs_lib
@pytest.mark.parametrize("call,kw,status", REFUSED,
                         ids=lambda x: getattr(x, "__name__", str(x))[:40])
def test_refused(call, kw, status):
    assert call(**kw) == status
    assert ef.library().ef_status_string(status) not in (b"unknown status", b"ok")


@needs_lib
def test_nothing_to_do():
    """Calls without rows or sequences need no buffers."""
    assert rope(T=0, x=None, out=None, positions=None, turns=None) == 0
    assert write(T=0, k=None, v=None, k_cache=None) == 0 and write(B=0, k=None, starts=None) == 0
    assert read(T=0, k_out=None) == 0 and read(B=0, starts=None) == 0
    assert paged(T=0, q=None, o=None, ws=None) == 0 and paged(B=0, ws=None) == 0
    assert paged(max_queries=0, q=None, ws=None) == 0
    assert packed(T=0, q=None, ws=None) == 0 and packed(B=0, ws=None) == 0


@needs_lib
def test_workspace_sizes():
    size = ef.ef_attention_paged_workspace_size
    assert size(8, 8, 32, 8, 128, 1) > ef.COUNTER_REGION_BYTES
    assert size(8, 8, 33, 8, 128, 1) == size(8, 8, 32, 8, 128, -1) == size(8, 0, 32, 8, 128, 1) == 0
    # It does not grow without end with the sequences, and shrinks with none of them.
    assert size(4000, 4000, 32, 8, 128, 1) < 2 ** 28
    for n in range(1, 20):
        assert size(n * 8, n, 64, 8, 128, 8) >= size(n, n, 64, 8, 128, 1)
    size = ef.ef_attention_packed_workspace_size
    assert size(100, 500, 3, 32, 8, 128) == 0           # too few keys to cut
    assert size(100, 50000, 3, 32, 8, 128) > ef.COUNTER_REGION_BYTES
    assert size(0, 50000, 3, 32, 8, 128) == size(100, 50000, 3, 31, 8, 128) == 0


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_refuses_cpu_tensors_and_shapes():
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError, match="k must be a GPU tensor"):
        ef.PagedCache(bf16(3, 2, 16, 64), bf16(3, 2, 16, 64))
    with pytest.raises(TypeError, match="turns must be a GPU tensor"):
        ef.make_rope(32, device="cpu")
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        ef.attention_packed(bf16(4, 2, 64), bf16(4, 2, 64), bf16(4, 2, 64), i32)
    with pytest.raises(ValueError, match="multiple of 16"):
        ef.make_rope(40)


def test_rope_turns():
    t = ef.rope_turns(64, 10000.0)
    assert t.dtype == torch.float64 and t.shape == (32,)
    assert torch.allclose(t * 2 * math.pi, torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)],
                                                        dtype=torch.float64), rtol=1e-14)
    assert torch.equal(ef.rope_turns(64, scaling="linear", factor=4.0), t / 4)
    b = ef.rope_turns(64, scaling="base", factor=4.0)
    assert b[0] == t[0] and math.isclose(b[-1], t[-1] / 4, rel_tol=1e-12)
    for kind in ("turns", "index"):
        s = ef.rope_turns(64, scaling=kind, factor=4.0, length=2048, low=1.0, high=8.0)
        fast, slow = 2048 * t >= 8 * 1.4, 2048 * t <= 1 / 1.4
        assert torch.equal(s[fast], t[fast]) and torch.allclose(s[slow], t[slow] / 4, rtol=1e-14)
        assert ((s <= t) & (s >= t / 4)).all()
    for bad in (dict(rot=0), dict(rot=7), dict(rot=16, base=0.0), dict(rot=16, factor=0.0),
                dict(rot=16, scaling="other"), dict(rot=16, scaling="turns"),
                dict(rot=16, scaling="index", length=10, low=4.0, high=4.0),
                dict(rot=2, scaling="base", factor=2.0),
                dict(rot=16, base=1.0, scaling="index", length=10)):
        with pytest.raises(ValueError):
            ef.rope_turns(**bad)


def test_oracle_rope():
    """Against matrices, norms and the transposed map."""
    rng = np.random.default_rng(0)
    x, y = rng.normal(size=(2, 5, 3, 16))
    pos, turns = np.array([0, 1, 5, 100, 7]), np.array([0.3, 0.01, 0.002, 1e-4])
    for inter in (False, True):
        r = oracle.rope_ref(x, pos, turns, inter, 1.5)
        assert np.array_equal(r[..., 8:], x[..., 8:])
        assert np.allclose(r[0, :, :8], 1.5 * x[0, :, :8])
        for t, p in enumerate(pos):
            for i, f in enumerate(turns):
                a, b = (2 * i, 2 * i + 1) if inter else (i, i + 4)
                c, s = math.cos(2 * math.pi * p * f), math.sin(2 * math.pi * p * f)
                assert np.allclose(r[t, :, a], 1.5 * (x[t, :, a] * c - x[t, :, b] * s))
                assert np.allclose(r[t, :, b], 1.5 * (x[t, :, b] * c + x[t, :, a] * s))
        back = oracle.rope_ref(y, pos, turns, inter, 1.5, True)
        assert np.allclose((r * y).sum(), (x * back).sum())  # <R x, y> = <x, R^T y>


def test_oracle_sequences():
    """Packed and paged attention against the dense oracle, rows and pages against loops."""
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(4, 6, 64)), rng.normal(size=(9, 2, 64)), rng.normal(size=(9, 2, 64))
    dense = oracle.attention_ref(q.transpose(1, 0, 2)[None], k.transpose(1, 0, 2)[None],
                                 v.transpose(1, 0, 2)[None], 0.1, True)[0].transpose(1, 0, 2)
    assert np.allclose(oracle.sequence_attention_ref(q, k, v, 0.1, True), dense)
    table = np.array([[2, 0, 7], [1, 7, 7]])
    kc, vc = rng.normal(size=(2, 3, 2, 4, 64))
    rows = oracle.cached_rows(kc, table, 0, 9)
    assert np.array_equal(rows[5], kc[0, :, 1]) and np.isnan(rows[8]).all()
    out = oracle.paged_attention_ref(q, kc, vc, table, [7, 3], [0, 3, 4], 0.1)
    assert np.allclose(out[:3], oracle.sequence_attention_ref(
        q[:3], rows[:7], oracle.cached_rows(vc, table, 0, 7), 0.1, True))
    assert oracle.token_places([0, 3, 4], [7, 3]) == [(0, 0, 4), (1, 0, 5), (2, 0, 6), (3, 1, 2)]
    both = oracle.packed_attention_ref(q, k, v, [0, 3, 4], [0, 9, 9], 0.1)
    assert np.array_equal(both[3], np.zeros((6, 64)))

"""Rotary positions, cache writes and cache reads on the GPU, against the fp64 oracle.

Tolerances. A turned element is A (a cos - b sin): cos and sin (times A) rounded to fp32, two
products and a sum rounded to fp32, at most 3.1 2^-24 of A (|a| + |b|); then one rounding to bf16,
at most 2^-8 of the value. Copied elements are equal. 8-bit rows: the scale is that of the exact
row unless its largest magnitude lies within that fp32 error of the border (checked as bounds), a
code is off by half a step, 2^-4 of the value, or half of 2^-9 s among the smallest codes."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, make_table, quantised, starts_of

pytestmark = pytest.mark.gpu

FP32 = 3.1 * 2.0 ** -24


def pair_size(x, rot, interleaved):
    """|a| + |b| of each element's pair, 0 where it is copied."""
    m = np.zeros(x.shape)
    if rot == 0:
        return m
    a, b = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved else
            (slice(0, rot // 2), slice(rot // 2, rot)))
    m[..., a] = m[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return m


def check_rows(got, x, ref, rot, interleaved, amplitude, what):
    err = FP32 * amplitude * pair_size(f64(x), rot, interleaved)
    tol = err + 2.0 ** -8 * (np.abs(ref) + err)
    worst = np.max(np.abs(f64(got) - ref) - tol, initial=-1.0)
    assert worst <= 0, f"{what}: {worst:.3e} over the tolerance"
    assert np.array_equal(f64(got)[..., rot:], f64(x)[..., rot:]), what


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 16), (3, 5, 64, 64), (7, 32, 128, 128),
                                       (257, 3, 128, 48), (2500, 2, 64, 32), (9000, 4, 128, 96)])
def test_rope(T, H, D, rot, interleaved, transpose):
    announce(f"rope {T} {H} {D} {rot} {interleaved} {transpose}")
    x = normal(T, T, H, D)
    g = torch.Generator().manual_seed(T)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    pos[-1] = -3
    pos[0] = 2 ** 31 - 1
    r = ef.make_rope(rot, interleaved=interleaved, amplitude=1.3)
    xd = x.cuda()
    got = ef.rope(xd, pos.cuda(), r, transpose=transpose)
    ref = oracle.rope_ref(f64(x), pos.numpy(), f64(r.turns), interleaved, 1.3, transpose)
    check_rows(got, x, ref, rot, interleaved, 1.3, "rope")
    assert torch.equal(xd.cpu(), x)
    assert ef.rope(xd, pos.cuda(), r, transpose=transpose, out=xd) is xd
    assert torch.equal(xd, got)  # in place


def test_rope_gradient():
    """The transposed map against differences of the map: it is linear, so one step tells."""
    announce("rope gradient")
    T, H, D = 5, 3, 64
    r = ef.make_rope(32, amplitude=1.0)
    pos = torch.tensor([0, 1, 77, 5000, 123456], dtype=torch.int32)
    w = normal(1, T, H, D)  # gradient of the result
    got = f64(ef.rope(w.cuda(), pos.cuda(), r, transpose=True))
    e = np.zeros((T, H, D))
    for d in range(D):
        e[:] = 0
        e[..., d] = 1
        y = oracle.rope_ref(e, pos.numpy(), f64(r.turns))
        want = (y * f64(w)).sum(-1)
        size = np.abs(y * f64(w)).sum(-1)
        assert (np.abs(got[..., d] - want) <= 2.0 ** -8 * np.abs(want) + 2 * FP32 * size).all(), d


def write_case(new, lengths, page, e4m3, rot, interleaved=False, even=False, Hq=4, H=2, D=128,
               seed=30, first=0, behind=0):
    starts = starts_of(new, first)
    T = starts[-1] + behind
    q, k, v = normal(seed, T, Hq, D), normal(seed + 1, T, H, D), normal(seed + 2, T, H, D)
    pages, table = make_table(seed + 3, page, [max(n, 0) for n in lengths])
    cache = ef.make_cache(pages, H, page, D, e4m3)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(0x55)
    if e4m3:
        cache.k_scale.fill_(-7.0)
        cache.v_scale.fill_(-7.0)
    r = ef.make_rope(rot, interleaved=interleaved, amplitude=1.1) if rot else None
    q_out = torch.full_like(q.cuda(), 9.0)
    got = ef.cache_write(cache, k.cuda(), v.cuda(), torch.from_numpy(table).cuda(), ints(lengths),
                         starts=None if even else ints(starts), q=q.cuda(), rope=r, q_out=q_out)
    torch.cuda.synchronize()
    places = oracle.token_places(starts, lengths)
    rows = [t for t, b, p in places]
    pos = [p for t, b, p in places]

    def turned(x):
        x = f64(x[rows])
        return oracle.rope_ref(x, pos, f64(r.turns), interleaved, 1.1) if rot else x

    qr, kr = turned(q), turned(k)
    check_rows(got[rows], q[rows], qr, rot, interleaved, 1.1, "q")
    outside = [t for t in range(T) if t not in set(rows)]
    assert (got[outside] == 9.0).all()

    kept = {}  # (page, row) -> packed row
    for i, (t, b, p) in enumerate(places):
        if p >= 0 and 0 <= table[b, p // page] < pages:
            kept[(int(table[b, p // page]), p % page)] = i
    at = list(kept)
    ids = [kept[a] for a in at]
    pi, ri = [a[0] for a in at], [a[1] for a in at]
    blank = torch.ones(pages, page, dtype=torch.bool)
    blank[pi, ri] = False
    tr = torch.tensor(rows)[ids] if ids else torch.zeros(0, dtype=torch.long)
    err = FP32 * 1.1 * pair_size(f64(k[tr]), rot, interleaved)
    if e4m3:
        codes, scales = quantised(v[tr])
        assert torch.equal(cache.v.cpu()[pi, :, ri].view(torch.uint8), codes.view(torch.uint8))
        assert torch.equal(cache.v_scale.cpu()[pi, :, ri], scales)
        s = f64(cache.k_scale)[pi, :, ri]
        top = np.abs(kr[ids]).max(-1)
        slack = err.max(-1)
        assert (np.log2(s) % 1 == 0).all()
        assert (top - slack <= 448 * s).all() and (top + slack > 224 * s).all()
        val = f64(cache.k.cpu().float())[pi, :, ri] * s[..., None]
        tol = err + np.maximum(2.0 ** -4 * (np.abs(kr[ids]) + err), 2.0 ** -10 * s[..., None])
        assert (np.abs(val - kr[ids]) <= tol).all()
    else:
        assert torch.equal(cache.v.cpu()[pi, :, ri], v[tr])
        check_rows(cache.k.cpu()[pi, :, ri], k[tr], kr[ids], rot, interleaved, 1.1, "k")
    for t in (cache.k, cache.v):
        assert (t.cpu().view(torch.uint8).transpose(1, 2)[blank] == 0x55).all()
    if e4m3:
        for t in (cache.k_scale, cache.v_scale):
            assert (t.cpu().transpose(1, 2)[blank] == -7.0).all()
    return cache


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("kw", [
    dict(new=[1], lengths=[1], page=16, rot=128),
    dict(new=[1, 1, 1], lengths=[1, 300, 64], page=16, rot=64, even=True),
    dict(new=[5, 0, 70, 1], lengths=[5, 9, 200, 33], page=32, rot=0),
    dict(new=[40, 3], lengths=[40, 1000], page=64, rot=32, interleaved=True, first=2, behind=3),
    dict(new=[4, 6], lengths=[2, 100], page=128, rot=128),         # tokens in front of position 0
    dict(new=[3000, 900, 1, 6000], lengths=[3000, 1000, 1, 6000], page=256, rot=16, Hq=2, H=1, D=64),
    dict(new=[1] * 150, lengths=[1 + i for i in range(150)], page=16, rot=48, Hq=3, H=3, D=64),
    dict(new=[7, 9], lengths=[7, 9], page=16, rot=64, Hq=32, H=8, D=64, interleaved=True),
], ids=lambda kw: str(kw["new"])[:30])
def test_cache_write(kw, e4m3):
    announce(f"cache_write {kw} {e4m3}")
    write_case(e4m3=e4m3, **kw)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("H,D,page,counts,lengths,first,behind", [
    (1, 64, 16, [1], [1], 0, 0),
    (8, 128, 16, [300, 0, 17, 1], [300, 5, 17, 1], 0, 0),
    (3, 64, 128, [40, 129, 500], [60, 129, 700], 5, 7),
    (2, 128, 64, [3] * 150, [3] * 150, 0, 1),
])
def test_cache_read(H, D, page, counts, lengths, first, behind, e4m3):
    announce(f"cache_read {H} {D} {page} {e4m3}")
    p = Pages(40, H, page, D, lengths, e4m3)
    starts = starts_of(counts, first)
    T = starts[-1] + behind
    outs = [torch.full((T, H, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = ef.cache_read(p.cache, p.dev_table, ints(starts), k_out=outs[0], v_out=outs[1])
    for got, values in ((k, p.values[0]), (v, p.values[1])):
        want = np.full((T, H, D), 3.0)
        for b, n in enumerate(counts):
            want[starts[b]:starts[b + 1]] = oracle.cached_rows(values, p.table, b, n)
        assert np.array_equal(f64(got), want)

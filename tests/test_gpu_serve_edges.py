"""Where the serving operators could go wrong: rows that belong to no sequence, pages that do not
exist, queries and rows that are not finite, large scores, offsets past 32 bits, streams, workspaces
and their counters."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import Pages, ints, quantised, starts_of
from test_gpu_serve_attention import run_packed, run_paged

pytestmark = pytest.mark.gpu

FMT = pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])


def paged(p, q, lengths, starts, most, **kw):
    return ef.attention_paged(q.cuda(), p.cache, p.dev_table, ints(lengths), starts=ints(starts),
                              max_queries=most, **kw)


def paged_ref(p, q, lengths, starts):
    D = q.shape[-1]
    a = (f64(q), p.values[0])
    b = (p.table, lengths, starts, D ** -0.5)
    return (oracle.paged_attention_ref(*a, p.values[1], *b),
            oracle.paged_attention_ref(*a, np.abs(p.values[1]), *b))


# ------------------------------------------------------------------ rows of no sequence


def test_rows_outside_stay():
    announce("rows of no sequence")
    lengths, new = [100, 7, 50], [3, 0, 2]
    starts = starts_of(new, 4)
    q = normal(1, starts[-1] + 6, 8, 128)
    p = Pages(2, 2, 16, 128, lengths, False)
    out = torch.full_like(q.cuda(), 5.0)
    paged(p, q, lengths, starts, 3, out=out)
    keep = [t for t in range(q.shape[0]) if not 4 <= t < starts[-1]]
    assert (out[keep] == 5.0).all() and not (out[4:starts[-1]] == 5.0).all(-1).any()
    ref, mag = paged_ref(p, q, lengths, starts)
    close(out[4:starts[-1]], ref[4:starts[-1]], mag[4:starts[-1]], "paged")
    ks = starts_of(lengths, 3)
    k, v = normal(3, ks[-1] + 2, 2, 128), normal(4, ks[-1] + 2, 2, 128)
    out.fill_(5.0)
    ef.attention_packed(q.cuda(), k.cuda(), v.cuda(), ints(starts), ints(ks), out=out)
    assert (out[keep] == 5.0).all()
    ref = oracle.packed_attention_ref(f64(q), f64(k), f64(v), starts, ks, 128 ** -0.5)
    mag = oracle.packed_attention_ref(f64(q), f64(k), np.abs(f64(v)), starts, ks, 128 ** -0.5)
    close(out[4:starts[-1]], ref[4:starts[-1]], mag[4:starts[-1]], "packed")


def test_max_queries_writes_the_first_rows():
    announce("more rows than max_queries")
    lengths, new = [90, 40], [6, 2]
    starts = starts_of(new)
    q = normal(5, 8, 8, 64)
    p = Pages(6, 2, 32, 64, lengths, False)
    out = torch.full_like(q.cuda(), 5.0)
    paged(p, q, lengths, starts, 3, out=out)
    ref, mag = paged_ref(p, q, lengths, starts)
    rows = [0, 1, 2, 6, 7]
    close(out[rows], ref[rows], mag[rows], "first rows")
    assert (out[3:6] == 5.0).all()


def test_lengths_and_starts_out_of_range():
    """Lengths beyond the table count as the table, negative ones as 0; starts as their next
    number in range."""
    announce("lengths and starts out of range")
    p = Pages(7, 2, 16, 64, [64, 64, 64], False)
    q = normal(8, 3, 4, 64)
    got = ef.attention_paged(q.cuda(), p.cache, p.dev_table, ints([10 ** 9, -5, 64]))
    ref, mag = paged_ref(p, q, [64, 0, 64], [0, 1, 2, 3])
    close(got, ref, mag, "lengths")
    k, v = normal(9, 30, 2, 64), normal(10, 30, 2, 64)
    out = torch.full_like(q.cuda(), 5.0)
    ef.attention_packed(q.cuda(), k.cuda(), v.cuda(), ints([-7, 2, 10 ** 6]), ints([-1, 10, 99]),
                        out=out)
    args = ([0, 2, 3], [0, 10, 30], 64 ** -0.5)
    close(out, oracle.packed_attention_ref(f64(q), f64(k), f64(v), *args),
          oracle.packed_attention_ref(f64(q), f64(k), np.abs(f64(v)), *args), "starts")


@pytest.mark.parametrize("Hq,H", [(4, 2), (64, 8)])
def test_empty_calls(Hq, H):
    announce("calls without rows, keys or sequences")
    p = Pages(11, H, 16, 64, [5], False)
    q = normal(12, 2, Hq, 64).cuda()
    none, empty = ints([]), torch.empty(0, Hq, 64, dtype=torch.bfloat16, device="cuda")
    no_table = p.dev_table[:0].contiguous()
    assert ef.attention_paged(empty, p.cache, no_table, none).shape == empty.shape
    assert ef.attention_packed(empty, empty, empty, ints([0])).shape == empty.shape
    wide = torch.empty(2, 0, dtype=torch.int32, device="cuda")  # tables without pages
    assert (ef.attention_paged(q, p.cache, wide, ints([9, 0])) == 0).all()
    nokeys = torch.empty(0, H, 64, dtype=torch.bfloat16, device="cuda")
    assert (ef.attention_packed(q, nokeys, nokeys, ints([0, 1, 2]), ints([0, 0, 0])) == 0).all()
    k, v = ef.cache_read(p.cache, p.dev_table, ints([0, 0]), total=0)
    assert k.shape == v.shape == (0, H, 64)
    kv = normal(13, 2, H, 64).cuda()
    before = p.cache.k.clone()
    ef.cache_write(p.cache, kv, kv, wide, ints([9, 1]))  # no page to write to
    assert torch.equal(p.cache.k.view(torch.int16), before.view(torch.int16))


# ------------------------------------------------------------------ pages


@FMT
def test_pages_that_do_not_exist(e4m3):
    """Rows that see a key of such a page are NaN, others are as if it were there."""
    announce(f"missing pages {e4m3}")
    lengths, new = [4000, 300, 2000], [4, 1, 8]
    starts = starts_of(new)
    q = normal(14, starts[-1], 8, 128)
    p = Pages(15, 2, 16, 128, lengths, e4m3)
    for page in (10 ** 6, -1, p.pages):
        t = p.dev_table.clone()
        t[0, 100] = page                  # all rows of sequence 0 see it
        t[2, (2000 - 3) // 16] = page     # positions 1984 .. : all rows of sequence 2, too
        t[2, 0] = t[2, 1]                 # (the same page twice is no fault)
        got = ef.attention_paged(q.cuda(), p.cache, t, ints(lengths), starts=ints(starts),
                                 max_queries=8)
        assert torch.isnan(got[:4]).all() and torch.isnan(got[5:]).all()
        ref, mag = paged_ref(p, q, lengths, starts)
        close(got[4:5], ref[4:5], mag[4:5], "whole sequence")
    # Rows in front of the page see all they should.
    lengths, new = [68], [8]
    q = normal(16, 8, 8, 128)
    p = Pages(17, 2, 16, 128, lengths, e4m3)
    t = p.dev_table.clone()
    t[0, 4] = -1  # positions 64 .. 67, rows 4 .. 7
    got = ef.attention_paged(q.cuda(), p.cache, t, ints(lengths))
    ref, mag = paged_ref(p, q, lengths, [0, 8])
    close(got[:4], ref[:4], mag[:4], "rows in front")
    assert torch.isnan(got[4:]).all()
    # Reads give NaN, writes leave the cache alone.
    k, v = ef.cache_read(p.cache, t, ints([0, 68]), total=68)
    assert torch.isnan(k[64:]).all() and torch.isnan(v[64:]).all()
    assert np.array_equal(f64(k[:64]), oracle.cached_rows(p.values[0], p.table, 0, 64))
    before = [x.view(torch.uint8).clone() for x in (p.cache.k, p.cache.v)]
    kv = normal(18, 4, 2, 128).cuda()
    ef.cache_write(p.cache, kv, kv, t, ints([68]))
    for x, y in zip((p.cache.k, p.cache.v), before):
        assert torch.equal(x.view(torch.uint8), y)


@FMT
def test_pages_of_several_sequences(e4m3):
    """Sequences may share pages to read."""
    announce(f"shared pages {e4m3}")
    p = Pages(19, 2, 16, 64, [200, 200], e4m3)
    t = p.dev_table.clone()
    t[1, :8] = t[0, :8]
    q = normal(20, 2, 8, 64)
    q[1] = q[0]
    got = ef.attention_paged(q.cuda(), p.cache, t, ints([128, 128]))
    assert torch.equal(got[0], got[1])


# ------------------------------------------------------------------ values


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_query_not_finite(bad):
    announce(f"query {bad}")
    for D, at in ((64, 3), (128, 127)):
        case = (8, 2, D, 16, [3, 2, 1], [2000, 2, 0])
        q = normal(21, 6, 8, D)
        clean = run_paged(case, False, queries=q)
        q[1, 5, at] = q[3, 0, at] = q[5, 2, at] = bad
        p = Pages(71, 2, 16, D, case[5], False)  # run_paged's
        got = paged(p, q, case[5], starts_of(case[4]), 3)
        hit = torch.zeros(6, 8, dtype=torch.bool, device="cuda")
        hit[1, 5] = hit[3, 0] = True  # row 5 sees no key
        assert torch.isnan(got[hit]).all()
        assert torch.equal(got[~hit], clean[~hit])
        case = (8, 2, D, [3, 200, 1], [9000, 200, 0], True)
        q = normal(22, 204, 8, D)
        clean = run_packed(case, queries=q)
        q[1, 5, at] = q[150, 0, at] = q[203, 2, at] = bad
        starts, ks = starts_of(case[3]), starts_of(case[4])
        k, v = normal(81, ks[-1], 2, D), normal(82, ks[-1], 2, D)
        got = ef.attention_packed(q.cuda(), k.cuda(), v.cuda(), ints(starts), ints(ks))
        hit = torch.zeros(204, 8, dtype=torch.bool, device="cuda")
        hit[1, 5] = hit[150, 0] = True
        assert torch.isnan(got[hit]).all()
        assert torch.equal(got[~hit], clean[~hit])


@FMT
@pytest.mark.parametrize("rising", [False, True])
def test_large_scores(rising, e4m3):
    """Scores of up to hundreds, rising or falling along the keys, so that references move (or a few
    keys have all the weight). A score is off by at most 2 D 2^-24 scale |q| |k|, e here, which
    moves a weight by a factor of up to e^e, in the sum of the weights too."""
    announce(f"large scores {rising} {e4m3}")
    D, lengths = 128, [3000, 500]
    size = torch.linspace(0.1, 3.0, 4096)
    p = Pages(23, 2, 16, D, lengths, False)
    for b, n in enumerate(lengths):
        order = torch.arange(n) if rising else torch.arange(n).flip(0)
        for pos in range(n):
            p.cache.k[p.table[b, pos // 16], :, pos % 16] *= size[order[pos]].item()
    q = normal(24, 2, 8, D) * 8
    if e4m3:
        codes, scales = zip(*(quantised(torch.nan_to_num(x.cpu())) for x in (p.cache.k, p.cache.v)))
        p.cache = ef.PagedCache(*(c.cuda() for c in codes), *(s.cuda() for s in scales))
        p.values = [f64(c.float()) * f64(s)[..., None] for c, s in zip(codes, scales)]
    else:
        p.values = [f64(p.cache.k), f64(p.cache.v)]
    ref, mag = paged_ref(p, q, lengths, [0, 1, 2])
    got = f64(paged(p, q, lengths, [0, 1, 2], 1))
    k = np.nan_to_num(p.values[0])
    e = 2 * D * 2.0 ** -24 * D ** -0.5 * (np.sqrt((f64(q) ** 2).sum(-1).max()) *
                                          np.sqrt((k ** 2).sum(-1).max()))
    tol = (2.0 ** -8 + 2.5 * np.expm1(e) + 1e-4) * mag + 2.0 ** -8 * 1.01 * np.abs(ref)
    assert (np.abs(got - ref) <= tol).all(), np.max(np.abs(got - ref) - tol)
    # Packed rows of the same.
    ks = starts_of(lengths)
    rows = [np.concatenate([oracle.cached_rows(x, p.table, b, n) for b, n in enumerate(lengths)])
            for x in p.values]
    kv = [torch.from_numpy(x).bfloat16() for x in rows]
    assert np.array_equal(f64(kv[0]), rows[0])  # 8-bit rows are exact in bf16
    got = f64(ef.attention_packed(q.cuda(), kv[0].cuda(), kv[1].cuda(), ints([0, 1, 2]), ints(ks)))
    assert (np.abs(got - ref) <= tol).all(), np.max(np.abs(got - ref) - tol)


def test_extreme_rows_of_8_bits():
    """Zeros, the smallest and the largest magnitudes, and elements that are not finite."""
    announce("extreme 8-bit rows")
    D, page = 64, 16
    rows = torch.zeros(12, 1, D)
    g = torch.Generator().manual_seed(0)
    for i, top in enumerate((0.0, 1e-40, 1e-38, 2.0 ** -100, 448 * 2.0 ** -100, 448.0, 449.0, 1.75,
                             1.76, 3e38)):
        rows[i] = torch.randn(1, D, generator=g).clamp(-1, 1) * top
        rows[i, 0, 5] = top
    rows[10] = rows[5]
    rows[10, 0, 3:6] = torch.tensor([float("inf"), float("nan"), float("-inf")])
    rows[11] = float("nan")
    rows = rows.bfloat16()
    cache = ef.make_cache(1, 1, page, D, True)
    ef.cache_write(cache, rows.cuda(), rows.cuda(), ints([0]).view(1, 1), ints([12]))
    finite = torch.isfinite(rows)
    codes, scales = quantised(torch.where(finite, rows, 0.0))
    for got, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert torch.equal(s.cpu()[0, 0, :12], scales[:, 0])
        got = got.cpu()[0, 0, :12].float()
        assert torch.isnan(got[~finite[:, 0]]).all()
        assert torch.equal(got[finite[:, 0]], codes.float()[:, 0][finite[:, 0]])
    k, _ = ef.cache_read(cache, ints([0]).view(1, 1), ints([0, 12]), total=12)
    want = codes.float() * scales[..., None]
    assert torch.equal(k.cpu()[finite], want[finite].bfloat16())


# ------------------------------------------------------------------ sizes


def test_offsets_past_32_bits():
    """A cache of 5 GiB each for k and v: its last pages."""
    announce("large cache")
    H, page, D, pages = 8, 16, 128, 163840
    cache = ef.make_cache(pages, H, page, D)
    n = 200
    last = [pages - 1 - 3 * i for i in range(13)]
    table = ints(last).view(1, 13)
    k, v, q = (normal(30 + i, n, h, D) for i, h in enumerate((H, H, 16)))
    ef.cache_write(cache, k.cuda(), v.cuda(), table, ints([n]))
    a, b = ef.cache_read(cache, table, ints([0, n]), total=n)
    assert torch.equal(a.cpu(), k) and torch.equal(b.cpu(), v)
    got = ef.attention_paged(q[:1].cuda(), cache, table, ints([n]))
    args = (f64(q[:1]), f64(k))
    close(got, oracle.sequence_attention_ref(*args, f64(v), D ** -0.5, True),
          oracle.sequence_attention_ref(*args, np.abs(f64(v)), D ** -0.5, True), "paged")
    del cache


def test_packed_rows_past_32_bits():
    """Rows of 64 heads of 128 behind 300000 others (4.9 GB), the last sequence's."""
    announce("packed rows past 32 bits")
    H, D, Tk, n = 64, 128, 300000, 150
    k = torch.zeros(Tk, H, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(Tk, H, D, dtype=torch.bfloat16, device="cuda")
    kk, vv, q = (normal(40 + i, n, H, D) for i in range(3))
    k[-n:], v[-n:] = kk.cuda(), vv.cuda()
    got = ef.attention_packed(q.cuda(), k, v, ints([0, 0, n]), ints([0, Tk - n, Tk]))
    args = (f64(q), f64(kk))
    close(got, oracle.sequence_attention_ref(*args, f64(vv), D ** -0.5, True),
          oracle.sequence_attention_ref(*args, np.abs(f64(vv)), D ** -0.5, True), "packed")


# ------------------------------------------------------------------ streams and workspaces


def test_streams_and_workspaces():
    """Calls on another stream, with a workspace made for it or by the call; one workspace for calls
    of other shapes; the counters are left zero; two runs give the same bits."""
    announce("streams and workspaces")
    lengths = [3000, 40, 900]
    p = Pages(50, 2, 16, 128, lengths, False)
    n = ints(lengths)
    q = normal(51, 3, 8, 128).cuda()
    ws = ef.make_paged_workspace(q, p.cache, 3, 1)
    want = ef.attention_paged(q, p.cache, p.dev_table, n, workspace=ws)
    big = normal(52, 48, 8, 128).cuda()
    ws = ef.make_paged_workspace(big, p.cache, 3, 16)
    first = ef.attention_paged(big, p.cache, p.dev_table, n, workspace=ws)
    assert torch.equal(ef.attention_paged(q, p.cache, p.dev_table, n, workspace=ws), want)
    assert torch.equal(ef.attention_paged(big, p.cache, p.dev_table, n, workspace=ws), first)
    kv = normal(53, 3940, 2, 128).cuda()
    ks = ints([0, 3000, 3040, 3940])
    packed = ef.attention_packed(q, kv, kv, ints([0, 1, 2, 3]), ks)
    assert not ef.workspace_counters(ws).any()
    busy = torch.randn(4096, 4096, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(3):
        for _ in range(10):
            busy = (busy @ busy).clamp(-1, 1)
        mine = ef.make_paged_workspace(q, p.cache, 3, 1, stream=stream)
        got = [ef.attention_paged(q, p.cache, p.dev_table, n, workspace=mine, stream=stream),
               ef.attention_paged(q, p.cache, p.dev_table, n, stream=stream),
               ef.attention_packed(q, kv, kv, ints([0, 1, 2, 3]), ks, stream=stream)]
        stream.synchronize()
        with torch.cuda.stream(stream):
            same = [torch.equal(a, b) for a, b in zip(got, (want, want, packed))]
        assert all(same), i
        torch.cuda.synchronize()


def test_workspace_of_several_operators():
    """Attention of packed sequences leaves the counters of a shared workspace alone."""
    announce("a workspace for both")
    p = Pages(49, 2, 16, 128, [1500, 700], False)
    q = normal(50, 2, 8, 128).cuda()
    starts, ks = [0, 5, 9], [0, 4000, 9000]
    qp = normal(51, 9, 8, 128).cuda()
    k, v = normal(52, 9000, 2, 128).cuda(), normal(53, 9000, 2, 128).cuda()
    alone = (ef.attention_paged(q, p.cache, p.dev_table, ints([1500, 700])),
             ef.attention_packed(qp, k, v, ints(starts), ints(ks)))
    n = max(ef.ef_attention_paged_workspace_size(2, 2, 8, 2, 128, 1),
            ef.ef_attention_packed_workspace_size(9, 9000, 2, 8, 2, 128))
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = ef.attention_packed(qp, k, v, ints(starts), ints(ks), workspace=ws)
        assert torch.equal(got, alone[1])
        assert not ws[:ef.COUNTER_REGION_BYTES].any()
        got = ef.attention_paged(q, p.cache, p.dev_table, ints([1500, 700]), workspace=ws)
        assert torch.equal(got, alone[0])


@pytest.mark.parametrize("Hq,H,counts", [(8, 2, True), (16, 8, True), (32, 2, False)])
def test_counter_that_was_not_zero(Hq, H, counts):
    """From the number of parts on: NaN rows, and the region cleared makes it good again. (The parts
    of 16 rows of a kv head are joined by a second launch, without counters.)"""
    announce(f"paged counters {H}")
    p = Pages(54, H, 16, 128, [3000], False)
    q = normal(55, 1, Hq, 128).cuda()
    ws = ef.make_paged_workspace(q, p.cache, 1, 1)
    want = ef.attention_paged(q, p.cache, p.dev_table, ints([3000]), workspace=ws)
    ef.workspace_counters(ws)[:] = 1000
    got = ef.attention_paged(q, p.cache, p.dev_table, ints([3000]), workspace=ws)
    assert torch.isnan(got).all() if counts else torch.equal(got, want)
    ef.workspace_counters(ws)[:] = 0
    got = ef.attention_paged(q, p.cache, p.dev_table, ints([3000]), workspace=ws)
    assert torch.equal(got, want)


def test_refusals_of_the_binding():
    announce("binding refusals")
    p = Pages(56, 2, 16, 128, [100, 5], False)
    q, kv = normal(57, 2, 8, 128).cuda(), normal(58, 2, 2, 128).cuda()
    n, t = ints([100, 5]), p.dev_table
    r = ef.make_rope(64)
    bad = [
        (TypeError, lambda: ef.attention_paged(q.float(), p.cache, t, n)),
        (TypeError, lambda: ef.attention_paged(q, p.cache, t, n.long())),
        (TypeError, lambda: ef.attention_paged(q, p.cache, t.cpu(), n)),
        (ValueError, lambda: ef.attention_paged(q, p.cache, t, n[:1])),
        (ValueError, lambda: ef.attention_paged(q[:1], p.cache, t, n)),
        (ValueError, lambda: ef.attention_paged(q, p.cache, t, n, starts=ints([0, 1, 2]))),
        (ValueError, lambda: ef.attention_paged(q[..., :64].contiguous(), p.cache, t, n)),
        (ValueError, lambda: ef.attention_paged(q.transpose(0, 1), p.cache, t, n)),
        (ValueError, lambda: ef.attention_paged(q, p.cache, t, n, out=q[:1])),
        (ef.EfError, lambda: ef.attention_paged(q[:, :7].contiguous(), p.cache, t, n)),
        (ef.EfError, lambda: ef.attention_paged(q, p.cache, t, n, scale=float("nan"))),
        (ef.EfError, lambda: ef.attention_paged(q, p.cache, t, n, workspace=ints([0] * 64))),
        (ValueError, lambda: ef.cache_write(p.cache, kv, kv[:1], t, n)),
        (ValueError, lambda: ef.cache_write(p.cache, kv, kv, t, n, q_out=q)),
        (ValueError, lambda: ef.cache_write(p.cache, kv[:, :1].contiguous(), kv[:, :1].contiguous(),
                                            t, n)),
        (ValueError, lambda: ef.cache_write(p.cache, kv, kv, t, n, q=q[:1])),
        (ValueError, lambda: ef.cache_write(p.cache, kv, kv, t, n, starts=ints([0, 2]))),
        (ValueError, lambda: ef.cache_read(p.cache, t, ints([0, 1, 2]))),
        (ValueError, lambda: ef.cache_read(p.cache, t, ints([0, 2]), total=2)),
        (ValueError, lambda: ef.cache_read(p.cache, t, ints([0, 1, 2]), total=3, k_out=kv)),
        (ValueError, lambda: ef.cache_read(p.cache, t, ints([0, 1, 2]), total=-1)),
        (ValueError, lambda: ef.attention_packed(q, kv, kv, ints([0, 1, 2]), ints([0, 2]))),
        (ValueError, lambda: ef.attention_packed(q, kv, kv[:1], ints([0, 1, 2]))),
        (ValueError, lambda: ef.attention_packed(q, kv, kv, ints([]))),
        (AttributeError, lambda: ef.attention_packed(q, kv, kv, [0, 1, 2])),
        (ValueError, lambda: ef.rope(q, ints([1]), r)),
        (TypeError, lambda: ef.rope(q, ints([1, 2]).long(), r)),
        (ValueError, lambda: ef.rope(q[:, :, :64], ints([1, 2]), r)),
        (ef.EfError, lambda: ef.rope(q[..., :64].contiguous(), ints([1, 2]), ef.make_rope(128))),
        (ValueError, lambda: ef.PagedCache(p.cache.k, p.cache.v, p.cache.k, p.cache.v)),
        (ValueError, lambda: ef.PagedCache(p.cache.k, p.cache.v[:1])),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()

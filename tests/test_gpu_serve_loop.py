"""The serving operators together, as a serving loop runs them: prompts are written to the cache and
attended, a chunk of each follows behind what came before, then single steps, eager and as a
replayed graph. Every stage is compared with the fp64 oracle over the rows the cache holds.

Tolerances: attention that of long_helpers.py (its inputs are the rotated rows as they were
rounded, and the cached values); the rows themselves are tested in test_gpu_serve_rows.py."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef
from serve_helpers import ints, make_table, starts_of

pytestmark = pytest.mark.gpu


class Loop:
    def __init__(self, Hq, H, D, page, e4m3, room, seed=90):
        self.Hq, self.H, self.D, self.seed = Hq, H, D, seed
        pages, table = make_table(seed, page, room)
        self.table = table
        self.dev_table = torch.from_numpy(table).cuda()
        self.cache = ef.make_cache(pages, H, page, D, e4m3)
        self.rope = ef.make_rope(D // 2, scaling="linear", factor=2.0)
        self.scale = D ** -0.5

    def tokens(self, T):
        self.seed += 3
        return [normal(self.seed + i, T, h, self.D).cuda() for i, h in
                enumerate((self.Hq, self.H, self.H))]

    def held(self, lengths):
        """Cached values of every sequence in 64 bits."""
        out = []
        for x, s in ((self.cache.k, self.cache.k_scale), (self.cache.v, self.cache.v_scale)):
            x = f64(x.float()) if s is None else f64(x.float()) * f64(s)[..., None]
            out.append([oracle.cached_rows(x, self.table, b, n) for b, n in enumerate(lengths)])
        return out

    def check(self, got, q, starts, lengths, what):
        k, v = self.held(lengths)
        ref, mag = np.zeros(q.shape), np.zeros(q.shape)
        for b in range(len(lengths)):
            rows = slice(starts[b], starts[b + 1])
            ref[rows] = oracle.sequence_attention_ref(f64(q)[rows], k[b], v[b], self.scale, True)
            mag[rows] = oracle.sequence_attention_ref(f64(q)[rows], k[b], np.abs(v[b]), self.scale,
                                                      True)
        close(got, ref, mag, what)


@pytest.mark.parametrize("Hq,H,D,page,e4m3", [(32, 8, 128, 16, False), (8, 2, 64, 64, True),
                                              (12, 4, 128, 32, True), (16, 1, 64, 16, False)])
def test_serving_loop(Hq, H, D, page, e4m3):
    announce(f"serving loop {Hq} {H} {D} {page} {e4m3}")
    lengths = [130, 1, 700, 65]
    chunk = [40, 17, 1, 300]
    steps = 6
    room = [a + b + steps + 2 for a, b in zip(lengths, chunk)]
    s = Loop(Hq, H, D, page, e4m3, room)

    # Prompts: with an 8-bit cache they attend to what it holds, like everything behind them.
    starts = starts_of(lengths)
    q, k, v = s.tokens(starts[-1])
    q = ef.cache_write(s.cache, k, v, s.dev_table, ints(lengths), starts=ints(starts), q=q,
                       rope=s.rope)
    kr, vr = ef.cache_read(s.cache, s.dev_table, ints(starts), total=starts[-1])
    s.check(ef.attention_packed(q, kr, vr, ints(starts)), q, starts, lengths, "prompts")

    # A chunk of each sequence.
    lengths = [a + b for a, b in zip(lengths, chunk)]
    starts, ks = starts_of(chunk), starts_of(lengths)
    q, k, v = s.tokens(starts[-1])
    ef.cache_write(s.cache, k, v, s.dev_table, ints(lengths), starts=ints(starts), q=q, rope=s.rope,
                   q_out=q)
    kr, vr = ef.cache_read(s.cache, s.dev_table, ints(ks), total=ks[-1])
    packed = ef.attention_packed(q, kr, vr, ints(starts), ints(ks))
    s.check(packed, q, starts, lengths, "chunks")
    # The same rows straight from the pages.
    paged = ef.attention_paged(q, s.cache, s.dev_table, ints(lengths), starts=ints(starts),
                               max_queries=max(chunk))
    s.check(paged, q, starts, lengths, "chunks over pages")

    # Steps of one token, all on tensors that are kept.
    B = len(lengths)
    dev_lengths = ints(lengths)
    q, k, v = s.tokens(B)
    out = torch.empty_like(q)
    ws = ef.make_paged_workspace(q, s.cache, B, 1)

    def step():
        dev_lengths.add_(1)
        ef.cache_write(s.cache, k, v, s.dev_table, dev_lengths, q=q, rope=s.rope, q_out=out)
        ef.attention_paged(out, s.cache, s.dev_table, dev_lengths, workspace=ws, out=out)

    turned = torch.empty_like(q)
    for i in range(2):
        for x, y in zip((q, k, v), s.tokens(B)):
            x.copy_(y)
        step()
        lengths = [n + 1 for n in lengths]
        pos = ints([n - 1 for n in lengths])
        ef.rope(q, pos, s.rope, out=turned)
        s.check(out, turned, list(range(B + 1)), lengths, f"step {i}")
    # The step as a graph, replayed with other tokens and lengths, eager work between.
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for i in range(4):
        for x, y in zip((q, k, v), s.tokens(B)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        lengths = [n + 1 for n in lengths]
        assert dev_lengths.tolist() == lengths
        ef.rope(q, ints([n - 1 for n in lengths]), s.rope, out=turned)
        s.check(out, turned, list(range(B + 1)), lengths, f"replay {i}")
        again = ef.attention_paged(turned, s.cache, s.dev_table, dev_lengths, workspace=ws)
        assert torch.equal(again, out), i
    assert not ef.workspace_counters(ws).any()


@pytest.mark.parametrize("Hq,H,D,e4m3", [(8, 1, 128, False), (8, 2, 64, True)])
def test_chunk_as_a_graph(Hq, H, D, e4m3):
    """A chunk of every sequence, written, read back and attended (with keys cut into parts), captured
    once and replayed with other tokens, lengths and starts, eager work between."""
    announce(f"chunk graph {Hq} {H} {D} {e4m3}")
    room = [5000, 3000, 300]
    s = Loop(Hq, H, D, 32, e4m3, room, seed=140)
    T, Tk = 96, sum(room)
    q, k, v = s.tokens(T)
    lengths, starts, ks = ints([0] * 3), ints([0] * 4), ints([0] * 4)
    kr, vr = (torch.zeros(Tk, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    turned, out = torch.empty_like(q), torch.empty_like(q)
    ws = ef.make_packed_workspace(q, kr, 3)
    assert ws is not None

    def chunk():
        ef.cache_write(s.cache, k, v, s.dev_table, lengths, starts=starts, q=q, rope=s.rope,
                       q_out=turned)
        ef.cache_read(s.cache, s.dev_table, ks, k_out=kr, v_out=vr)
        ef.attention_packed(turned, kr, vr, starts, ks, workspace=ws, out=out)

    def at(new, keys):
        for t, values in ((lengths, keys), (starts, starts_of(new)), (ks, starts_of(keys))):
            t.copy_(torch.tensor(values, dtype=torch.int32))
        for x, y in zip((q, k, v), s.tokens(T)):
            x.copy_(y)

    at([0, 0, 0], [0, 0, 0])
    chunk()  # (no row at all)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            chunk()
    torch.cuda.synchronize()
    # Caches of zeros: what a chunk attends to before all of it was written is well defined.
    for t in (s.cache.k, s.cache.v):
        t.view(torch.uint8).zero_()
    if e4m3:
        s.cache.k_scale.fill_(1.0)
        s.cache.v_scale.fill_(1.0)
    for i, (new, keys) in enumerate((([64, 32, 0], [4000, 32, 0]), ([1, 90, 5], [4001, 3000, 5]),
                                     ([90, 0, 6], [5000, 3000, 11]), ([3, 3, 3], [7, 2000, 300]))):
        at(new, keys)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        n = sum(new)
        s.check(got[:n], turned[:n], starts_of(new), keys, f"replay {i}")
        chunk()
        torch.cuda.synchronize()
        assert torch.equal(out[:n], got[:n]), i

"""The long-context operators as a program uses them: together, step after step, captured in a
graph and replayed, on another stream, with one workspace for several entry points, on caches of
more than 2^31 elements."""

import numpy as np
import pytest
import torch

import oracle
from long_helpers import _gpu, announce, close, f64, lengths_of, normal  # noqa: F401
from paper_2609_12330_amd import ef_attention as ef

pytestmark = pytest.mark.gpu

BS, K, SINKS, LOCAL = 64, 6, 1, 2


def check_blocks(got, q, k, v, lists, lengths, what):
    n = [int(x) for x in lengths]
    args = [f64(t) for t in (q, k, v)]
    scale = q.shape[-1] ** -0.5
    lists = lists.cpu().numpy()
    ref = oracle.attention_blocks_ref(*args, lists, BS, scale, n)
    mag = oracle.attention_blocks_ref(*args[:2], np.abs(args[2]), lists, BS, scale, n)
    close(got, ref, mag, what)


def test_prompt_then_steps():
    """A prompt attends to selected blocks; then every sequence goes on alone, its summaries kept
    up to date key by key; a dense layer reads the prompt as the prefix of all of them."""
    announce("prompt, then steps")
    B, Hq, H, D, Lp, cap = 3, 8, 2, 128, 900, 1100
    kp, vp = normal(60, 1, H, Lp, D).cuda(), normal(61, 1, H, Lp, D).cuda()

    # Prompt: all its queries choose their blocks and attend to them.
    q = normal(62, 1, Hq, Lp, D).cuda()
    m = ef.block_summary(kp, BS)
    lists = ef.block_select(q, m, Lp, K, BS, SINKS, LOCAL)
    out = ef.attention_blocks(q, kp, vp, lists, BS)
    torch.cuda.synchronize()
    want = oracle.block_select_ref(f64(q), f64(m), Lp, K, BS, SINKS, LOCAL)
    assert np.array_equal(lists.cpu().numpy(), want)
    check_blocks(out, q, kp, vp, lists, [Lp], "prompt")

    # Steps: the sparse layer's caches hold the prompt and what follows it.
    k, v = (torch.full((B, H, cap, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    k[:, :, :Lp], v[:, :, :Lp] = kp, vp
    ks, vs = (torch.full((B, H, cap - Lp, D), float("nan"), dtype=torch.bfloat16, device="cuda")
              for _ in range(2))
    nb = -(-cap // BS)
    m = torch.cat([m.expand(B, H, -1, D), torch.zeros(B, H, nb - m.shape[2], D, device="cuda")],
                  2).to(torch.bfloat16).contiguous()
    n = torch.full((B,), Lp, dtype=torch.int32, device="cuda")
    own = torch.zeros_like(n)
    ws = None
    for step in range(5):
        grow = torch.tensor([1, 0 if step == 2 else 1, 1], dtype=torch.int32, device="cuda")
        new_k, new_v = normal(70 + step, B, H, D).cuda(), normal(80 + step, B, H, D).cuda()
        for b in range(B):
            if int(grow[b]):
                i = int(n[b])
                k[b, :, i], v[b, :, i] = new_k[b], new_v[b]
                ks[b, :, i - Lp], vs[b, :, i - Lp] = new_k[b], new_v[b]
        n += grow
        own += grow
        q = normal(90 + step, B, Hq, 1, D).cuda()
        ef.block_summary(k, BS, lengths=n, new_keys=1, out=m)
        lists = ef.block_select(q, m, cap, K, BS, SINKS, LOCAL, lengths=n)
        if ws is None:
            ws = ef.make_blocks_workspace(q, k, K, BS)
        sparse = ef.attention_blocks(q, k, v, lists, BS, lengths=n, workspace=ws)
        dense = ef.attention_shared_prefix(q, kp[0], vp[0], ks, vs, lengths=own)
        torch.cuda.synchronize()
        lens = n.tolist()
        want = oracle.block_select_ref(f64(q), oracle.block_summary_ref(
            f64(k.nan_to_num()), BS, lens), cap, K, BS, SINKS, LOCAL, lens)
        # (Summaries are rounded to bf16; the choice is that of the rounded ones.)
        exact = oracle.block_select_ref(f64(q), f64(m), cap, K, BS, SINKS, LOCAL, lens)
        assert np.array_equal(lists.cpu().numpy(), exact)
        assert (np.sort(want[..., -LOCAL:]) == exact[..., -LOCAL:]).all()
        check_blocks(sparse, q, k.nan_to_num(), v.nan_to_num(), lists, lens, f"step {step}")
        a = [f64(t) for t in (q, kp[0], vp[0], ks.nan_to_num(), vs.nan_to_num())]
        ref = oracle.shared_prefix_ref(*a, D ** -0.5, True, own.tolist())
        mag = oracle.shared_prefix_ref(a[0], a[1], np.abs(a[2]), a[3], np.abs(a[4]), D ** -0.5,
                                       True, own.tolist())
        close(dense, ref, mag, f"dense step {step}")


def test_captured_step():
    """A whole step in a graph, replayed on changing inputs with eager work between."""
    announce("captured step")
    B, Hq, H, D, cap, Lp = 4, 16, 4, 64, 2000, 700
    k, v = normal(100, B, H, cap, D).cuda(), normal(101, B, H, cap, D).cuda()
    kp, vp = normal(102, H, Lp, D).cuda(), normal(103, H, Lp, D).cuda()
    q = normal(104, B, Hq, 1, D).cuda()
    n = lengths_of([2000, 1999, 640, 5])
    m = ef.block_summary(k, BS, lengths=n)
    lists = torch.empty(B, H, 1, K, dtype=torch.int32, device="cuda")
    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    w1 = ef.make_blocks_workspace(q, k, K, BS)
    w2 = ef.make_shared_prefix_workspace(q, kp, k)
    assert w1 is not None and w2 is not None

    def step():
        ef.block_summary(k, BS, lengths=n, new_keys=2, out=m)
        ef.block_select(q, m, cap, K, BS, SINKS, LOCAL, lengths=n, out=lists)
        ef.attention_blocks(q, k, v, lists, BS, lengths=n, workspace=w1, out=o1)
        ef.attention_shared_prefix(q, kp, vp, k, v, lengths=n, workspace=w2, out=o2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(normal(110 + i, B, Hq, 1, D))
        k[:, :, -70:] = normal(120 + i, B, H, 70, D).cuda()
        n.copy_(torch.tensor([2000 - i, 1999, 640 + 64 * i, 5 + i], dtype=torch.int32))
        before = m.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (m, lists, o1, o2)]
        m.copy_(before)
        for t in (lists, o1, o2):
            t.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (m, lists, o1, o2)):
            assert torch.equal(a, b)


def test_other_stream_and_shared_workspace():
    """Calls on a stream of their own, and one workspace for these and the split-KV entry points,
    in stream order."""
    announce("other stream, shared workspace")
    B, Hq, H, D, S = 2, 8, 2, 128, 3000
    q, k, v = (normal(130 + i, B, h, n, D).cuda() for i, (h, n) in
               enumerate(((Hq, 1), (H, S), (H, S))))
    lists = ef.block_select(q, ef.block_summary(k), S, 12)
    want = (ef.attention_blocks(q, k, v, lists), ef.attention_splitkv(q, k, v),
            ef.attention_shared_prefix(q, k[0], v[0], k, v))
    ws = ef.make_workspace(q, k, 64)
    big = max((ef.make_blocks_workspace(q, k, 12), ef.make_shared_prefix_workspace(q, k[0], k), ws),
              key=lambda t: t.numel())
    ws = torch.zeros_like(big)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = (ef.attention_blocks(q, k, v, lists, workspace=ws, stream=stream),
               ef.attention_splitkv(q, k, v, workspace=ws, stream=stream),
               ef.attention_shared_prefix(q, k[0], v[0], k, v, workspace=ws, stream=stream))
        with torch.cuda.stream(stream):
            again = ef.block_select(q, ef.block_summary(k, stream=stream), S, 12, stream=stream)
        stream.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert torch.equal(again, lists)
        assert not ef.workspace_counters(ws).any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("Sq", [1, 40, 900])
def test_query_that_is_not_finite(Sq, bad):
    """Its rows are NaN, in one part and in many, and nobody else's."""
    announce(f"query {bad} {Sq}")
    B, Hq, H, D, S = 2, 8, 2, 128, 3000
    q, k, v = (normal(170 + i, B, h, n, D).cuda() for i, (h, n) in
               enumerate(((Hq, Sq), (H, S), (H, S))))
    lists = ef.block_select(q, ef.block_summary(k), S, 12)
    calls = (lambda v: ef.attention_blocks(q, k, v, lists),
             lambda v: ef.attention_blocks(q, k, v, lists[..., -1:].contiguous()),
             lambda v: ef.attention_shared_prefix(q, k[0], v[0], k, v),
             lambda v: ef.attention_shared_prefix(q, k[0, :, :64].contiguous(),
                                                  v[0, :, :64].contiguous(), k[:, :, :0],
                                                  v[:, :, :0], causal=False))
    want = [(f(v), f(v.abs())) for f in calls]
    q[0, 3, Sq // 2, 5] = bad
    q[1, 6, 0] = bad
    rows = torch.zeros(B, Hq, Sq, dtype=torch.bool, device="cuda")
    rows[0, 3, Sq // 2] = rows[1, 6, 0] = True
    for f, (w, mag) in zip(calls, want):
        got = f(v)
        torch.cuda.synchronize()
        assert torch.isnan(got[rows]).all()
        # The 32 rows of a wave renew their references together, so a row's roundings may change:
        # both results are within the tolerance of the exact one, twice that of each other.
        w, mag = f64(w[~rows]), f64(mag[~rows])
        close(got[~rows], w, 2 * mag + np.abs(w), "other rows")


def test_other_stream_without_a_workspace():
    """A call on another stream makes what it needs there: nothing of it waits for, or is
    overtaken by, the work of the current stream."""
    announce("other stream, own workspace")
    B, Hq, H, D, S = 1, 8, 2, 128, 3000
    q, k = normal(160, B, Hq, 1, D).cuda(), normal(161, B, H, S, D).cuda()
    lists = ef.block_select(q, ef.block_summary(k), S, 12)
    want = (ef.attention_blocks(q, k, k, lists), ef.attention_shared_prefix(q, k[0], k[0], k, k))
    stream = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for i in range(3):
        n = ef.make_blocks_workspace(q, k, 12).numel()
        torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # what its memory holds
        for _ in range(20):
            busy = (busy @ busy).clamp(-1, 1)
        got = (ef.attention_blocks(q, k, k, lists, stream=stream),
               ef.attention_shared_prefix(q, k[0], k[0], k, k, stream=stream))
        for _ in range(20):  # would take the memory of a workspace freed here
            busy = (busy @ busy).clamp(-1, 1)
            torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        stream.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i
        torch.cuda.synchronize()


def test_counters_that_were_not_zero():
    announce("counters not zero")
    B, Hq, H, D, S = 1, 4, 1, 64, 2000
    q, k = normal(140, B, Hq, 1, D).cuda(), normal(141, B, H, S, D).cuda()
    lists = ef.block_select(q, ef.block_summary(k), S, 8)
    ws = ef.make_blocks_workspace(q, k, 8)
    ws.fill_(1)
    out = ef.attention_blocks(q, k, k, lists, workspace=ws)
    torch.cuda.synchronize()
    assert torch.isnan(out).all()


def test_same_inputs_same_bits():
    announce("determinism")
    B, Hq, H, D, S = 2, 16, 4, 128, 5000
    q, k, v = (normal(150 + i, B, h, n, D).cuda() for i, (h, n) in
               enumerate(((Hq, 40), (H, S), (H, S))))
    n = lengths_of([5000, 777])
    m = ef.block_summary(k, lengths=n)
    lists = ef.block_select(q, m, S, 9, lengths=n)
    outs = [(ef.block_summary(k, lengths=n), ef.block_select(q, m, S, 9, lengths=n),
             ef.attention_blocks(q, k, v, lists, lengths=n),
             ef.attention_shared_prefix(q, k[0], v[0], k, v, lengths=n)) for _ in range(3)]
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("shape", [(2, 4, 2, 3, 0, 64), (1, 2, 2, 70, 0, 128)], ids=str)
def test_no_keys(shape):
    announce(f"no keys {shape}")
    B, Hq, H, Sq, S, D = shape
    q = normal(160, B, Hq, Sq, D).cuda()
    k = torch.empty(B, H, S, D, dtype=torch.bfloat16, device="cuda")
    lists = ef.block_select(q, ef.block_summary(k), S, 5)
    assert (lists == -1).all()
    assert (ef.attention_blocks(q, k, k, lists) == 0).all()
    assert (ef.attention_shared_prefix(q, k[0], k[0], k, k) == 0).all()


def test_nothing_to_do():
    announce("nothing to do")
    q = torch.empty(0, 4, 3, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(0, 2, 100, 64, dtype=torch.bfloat16, device="cuda")
    kp = torch.empty(2, 30, 64, dtype=torch.bfloat16, device="cuda")
    lists = ef.block_select(q, ef.block_summary(k), 100, 5)
    assert lists.shape == (0, 2, 3, 5)
    assert ef.attention_blocks(q, k, k, lists).shape == q.shape
    assert ef.attention_shared_prefix(q, kp, kp, k, k).shape == q.shape


def test_lengths_outside_the_capacity():
    """Clamped to [0, Skv] on the device."""
    announce("lengths clamped")
    B, Hq, H, D, S = 3, 4, 2, 64, 300
    q, k, v = (normal(170 + i, B, h, n, D).cuda() for i, (h, n) in
               enumerate(((Hq, 2), (H, S), (H, S))))
    wild, tame = lengths_of([-7, 10 ** 9, 299]), lengths_of([0, 300, 299])
    m = ef.block_summary(k)
    lists = ef.block_select(q, m, S, 3, lengths=wild)
    assert torch.equal(lists, ef.block_select(q, m, S, 3, lengths=tame))
    assert torch.equal(ef.attention_blocks(q, k, v, lists, lengths=wild),
                       ef.attention_blocks(q, k, v, lists, lengths=tame))
    assert torch.equal(ef.attention_shared_prefix(q, k[0], v[0], k, v, lengths=wild),
                       ef.attention_shared_prefix(q, k[0], v[0], k, v, lengths=tame))


def test_caches_past_32_bits():
    """K and V of 2^31 + 2^30 elements: the last sequence's last head lies past 2^32 bytes, and
    its last block past 2^31 elements."""
    announce("large caches")
    B, Hq, H, D, S = 3, 16, 8, 128, 1 << 20
    k, v = (torch.zeros(B, H, S, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bs, nb = 128, S // 128
    blocks = [0, 17, nb // 2, nb - 2, nb - 1]
    b, h = B - 1, H - 1
    for j, n in enumerate(blocks):
        k[b, h, n * bs:(n + 1) * bs] = normal(180 + j, bs, D).cuda()
        v[b, h, n * bs:(n + 1) * bs] = normal(190 + j, bs, D).cuda()
    m = ef.block_summary(k, bs)
    q = normal(200, B, Hq, 2, D).cuda()
    lists = ef.block_select(q, m, S, 5, bs, 1, 2)
    want = torch.tensor(blocks, dtype=torch.int32, device="cuda").expand(B, H, 2, 5).contiguous()
    out = ef.attention_blocks(q, k, v, want, bs)
    dense = ef.attention_shared_prefix(q, k[0, :, :64].contiguous(), v[0, :, :64].contiguous(), k,
                                       v)
    torch.cuda.synchronize()
    ref_m = oracle.block_summary_ref(f64(k[b:, h:, -2 * bs:]), bs)
    got_m = f64(m[b:, h:, -2:])
    assert (np.abs(got_m - ref_m) <= 2.0 ** -8 * np.abs(ref_m) + 130 * 2.0 ** -24).all()
    # All other blocks have summary 0: the two with the larger score are taken if positive.
    ref = oracle.block_select_ref(f64(q[b:, -2:]), f64(m[b:, h:]), S, 5, bs, 1, 2)
    assert np.array_equal(lists[b:, h:].cpu().numpy(), ref)
    # The listed blocks as a cache of their own; the last query sees it all, the one before all
    # but the last key.
    kc = torch.cat([k[b, h, n * bs:(n + 1) * bs] for n in blocks])[None, None]
    vc = torch.cat([v[b, h, n * bs:(n + 1) * bs] for n in blocks])[None, None]
    a = [f64(t) for t in (q[b:, -2:], kc, vc)]
    ref = oracle.attention_ref(*a, D ** -0.5, True)
    mag = oracle.attention_ref(*a[:2], np.abs(a[2]), D ** -0.5, True)
    close(out[b:, -2:], ref, mag, "large cache")
    # Dense: all keys but those of the listed blocks are 0 and have score 0 and value 0.
    x = np.einsum("hid,kd->hik", a[0][0], a[1][0, 0]) * D ** -0.5
    x[:, 0, -1] = -np.inf
    w = np.exp(x)
    zeros = S + 64 - len(blocks) * bs
    tot = w.sum(-1, keepdims=True) + zeros
    ref = np.einsum("hik,kd->hid", w, a[2][0, 0]) / tot
    mag = np.einsum("hik,kd->hid", w, np.abs(a[2][0, 0])) / tot
    close(dense[b, -2:], ref, mag, "large dense")

"""Performance cases of the long-context operators: block summaries, block selection, attention
over selected blocks, and attention of a batch over one shared prefix.

With ``own`` false ``run`` computes an operator in its plain form, elementary torch operations in
32 bits (the selection, which compares values next to each other, in 64), rounded once at the end.
With ``own`` true it makes the calls of ``paper_2609_12330_amd.ef_attention`` that an inference
program makes, on tensors and workspaces that such a program keeps between calls.

q, k and v are N(0, 1) rounded to bf16, drawn on the GPU from a seeded generator. Keys of one
block lean towards a common direction, so that its mean says something about them. Caches have a
capacity; the sequences of a batch fill it to different lengths. Head layouts are those of the
workloads and tests of this repository.
"""

import math

import torch

own = False

SUMMARY, SELECT, BLOCKS, PREFIX = "summary", "select", "blocks", "prefix"


def _case(name, op, B, Hq, Hkv, Sq, Skv, D, low=None, block=64, topk=0, sinks=1, local=2, new=0,
          pool=1.5, Lp=0, causal=True):
    """low: length of the shortest sequence, Skv being the longest's; pool: blocks that 64
    neighbouring queries choose theirs from, over topk (0: each from all blocks)."""
    c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, Sq=Sq, Skv=Skv, D=D, low=Skv if low is None else low,
             block=block, topk=topk, sinks=sinks, local=local, new=new, pool=pool, Lp=Lp,
             causal=causal)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # After a decode step: the last block of every sequence has a new key. All latency.
        _case("summary_step", SUMMARY, 16, 32, 8, 1, 8192, 128, low=4001, new=1),
        # After the prefill of a batch of long prompts of different lengths: a pass over all keys.
        _case("summary_prompt", SUMMARY, 8, 32, 8, 1, 32768, 128, low=20011),
        # Decode step of a batch over long contexts: 32 of up to 1024 blocks.
        _case("select_step", SELECT, 16, 32, 8, 1, 65536, 128, low=30001, topk=32),
        # Chunk of a long prompt of odd length, one kv head for two heads of 64, wider blocks.
        _case("select_chunk_d64", SELECT, 2, 8, 4, 777, 20001, 64, block=128, topk=12),
        # Chunk of a very long prompt: every query of it chooses 16 of up to 1024 blocks.
        _case("select_prompt", SELECT, 1, 32, 8, 4096, 65536, 128, topk=16),
        # One decode step of one sequence, few blocks.
        _case("blocks_single", BLOCKS, 1, 32, 8, 1, 16001, 128, topk=16),
        # Decode step of a batch of different lengths.
        _case("blocks_step", BLOCKS, 16, 32, 8, 1, 32768, 128, low=12001, topk=64),
        # Several query tokens per sequence (speculative decoding), 64-wide heads, wider blocks.
        _case("blocks_draft_d64", BLOCKS, 8, 64, 8, 5, 16384, 64, low=7001, block=128, topk=24),
        # Chunk of a long prompt: neighbouring queries agree on most of their blocks.
        _case("blocks_prompt", BLOCKS, 1, 32, 8, 4096, 32768, 128, topk=16),
        # A small batch answers questions about one short document.
        _case("prefix_small", PREFIX, 4, 32, 8, 1, 300, 128, low=5, Lp=2011),
        # Decode step of a large batch over one long document, with answers of different lengths.
        _case("prefix_step", PREFIX, 64, 32, 8, 1, 2048, 128, low=64, Lp=32768),
        # Prefill of a batch of questions behind a system prompt.
        _case("prefix_prompts", PREFIX, 16, 32, 8, 384, 384, 128, low=384, Lp=8192),
    ]


# Head layouts (Hq, Hkv) of the workloads and tests.
_HEADS = ((4, 4), (8, 2), (12, 12), (16, 4), (32, 8), (32, 32), (64, 8))
# A drawn case costs no more than the listed ones.
_MAX_BYTES = 1.1e9
_MAX_FLOPS = 400e9


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("summary", "summary_step", "select_step", "select", "blocks_step",
                       "blocks_draft", "blocks", "prefix_step", "prefix_draft", "prefix"))
    Hq, Hkv = rng.choice(_HEADS)
    D = rng.choice((64, 128, 128))
    B = _log(rng, 1, 32)
    block = rng.choice((64, 64, 128))
    topk = rng.choice((8, 13, 16, 32, 64))
    sinks, local = rng.choice((0, 1, 1)), rng.choice((1, 2, 3))

    def low(S):
        return max(1, S - rng.randrange(0, S)) if rng.random() < 0.7 else S

    if kind == "summary":
        S = _log(rng, 64, 65536)
        return _case(None, SUMMARY, B, Hq, Hkv, 1, S, D, low(S), block)
    if kind == "summary_step":
        S = _log(rng, 64, 65536)
        return _case(None, SUMMARY, B, Hq, Hkv, 1, S, D, low(S), block, new=_log(rng, 1, 300))
    if kind == "select_step":
        S = _log(rng, 1024, 131072)
        return _case(None, SELECT, B, Hq, Hkv, _log(rng, 1, 8), S, D, low(S), block, topk, sinks,
                     local)
    if kind == "select":
        S = _log(rng, 2048, 65536)
        return _case(None, SELECT, _log(rng, 1, 4), Hq, Hkv, min(S, _log(rng, 64, 4096)), S, D, S,
                     block, topk, sinks, local)
    if kind in ("blocks_step", "blocks_draft"):
        S = _log(rng, 1024, 65536)
        Sq = 1 if kind == "blocks_step" else _log(rng, 2, 16)
        return _case(None, BLOCKS, B, Hq, Hkv, Sq, S, D, low(S), block, topk, sinks, local,
                     pool=rng.choice((0, 1.5)))
    if kind == "blocks":
        S = _log(rng, 1024, 32768)
        return _case(None, BLOCKS, _log(rng, 1, 4), Hq, Hkv, min(S, _log(rng, 64, 4096)), S, D, S,
                     block, rng.choice((8, 13, 16)), sinks, local, pool=rng.choice((1.5, 2.5, 0)))
    S = _log(rng, 1, 4096)
    Lp = _log(rng, 64, 65536)
    B = _log(rng, 2, 64)
    if kind == "prefix_step":
        return _case(None, PREFIX, B, Hq, Hkv, 1, S, D, low(S), Lp=Lp)
    if kind == "prefix_draft":
        S = max(S, 16)
        return _case(None, PREFIX, B, Hq, Hkv, _log(rng, 2, 16), S, D, max(16, low(S)), Lp=Lp)
    S = _log(rng, 16, 512)
    return _case(None, PREFIX, B, Hq, Hkv, S, S, D, S, Lp=_log(rng, 64, 16384),
                 causal=rng.random() < 0.8)


def _gathered(c):
    """Bytes of the keys that a query-by-query gather makes in 32 bits."""
    return 4 * c["B"] * c["Hkv"] * c["Sq"] * c["topk"] * c["block"] * c["D"]


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        held = 4 * c["B"] * c["Hkv"] * c["Skv"] * c["D"] + 4 * c["Hkv"] * c["Lp"] * c["D"]
        scores = 8 * c["B"] * c["Hq"] * c["Sq"] * _keys_of_plain(c)
        if (w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES and held <= 6e9 and
                scores <= 20e9 and (c["op"] != BLOCKS or _gathered(c) <= 18e9)):
            return c


def _keys_of_plain(c):
    if c["op"] == SUMMARY:
        return 0
    if c["op"] == SELECT:
        return -(-c["Skv"] // c["block"])
    return c["topk"] * c["block"] if c["op"] == BLOCKS else c["Lp"] + c["Skv"]


def _lengths(case):
    """Lengths of the sequences: spread evenly from the shortest to the capacity, out of order."""
    B, S, low = case["B"], case["Skv"], case["low"]
    if low == S:
        return [S] * B
    if B == 1:
        return [S]
    a = [low + (S - low) * b // (B - 1) for b in range(B)]
    return a[::2][::-1] + a[1::2]


def _diagonals(case):
    """Key position of every query of every sequence (negative: before the first key)."""
    return [[i + n - case["Sq"] for i in range(case["Sq"])] for n in _lengths(case)]


def _blocks_of(case):
    return -(-case["Skv"] // case["block"])


def _scale(case):
    return 1.0 / math.sqrt(case["D"])


# ------------------------------------------------------------------------------------ inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for b in range(shape[0]):
        t[b] = torch.randn(shape[1:], generator=g, device="cuda")
    return t


def _keys(g, case):
    """[B][Hkv][Skv][D]: each key leans towards a direction of its block."""
    B, H, S, D = case["B"], case["Hkv"], case["Skv"], case["D"]
    bs, nb = case["block"], _blocks_of(case)
    t = torch.empty(B, H, S, D, dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        x = torch.randn(H, S, D, generator=g, device="cuda")
        lean = torch.randn(H, nb, D, generator=g, device="cuda")
        t[b] = x + 0.5 * lean.repeat_interleave(bs, 1)[:, :S]
    return t


def _means(k, block):
    """Mean key of each block of a whole cache."""
    B, H, S, D = k.shape
    nb = -(-S // block)
    x = torch.nn.functional.pad(k.float(), (0, 0, 0, nb * block - S)).view(B, H, nb, block, D)
    count = (S - torch.arange(nb, device="cuda") * block).clamp(max=block).view(1, 1, nb, 1)
    return (x.sum(3) / count).to(torch.bfloat16)


def _lists(g, case):
    """Block lists as a selection makes them: the first `sinks` blocks, the last `local` up to the
    query's own, and others from a pool that 64 neighbouring queries share, in ascending order,
    filled with -1."""
    B, H, Sq, K, bs = (case[x] for x in ("B", "Hkv", "Sq", "topk", "block"))
    nb = _blocks_of(case)
    cur = torch.tensor(_diagonals(case), device="cuda")
    cur = torch.where(cur >= 0, cur // bs, -1)[:, None, :, None]       # [B][1][Sq][1]
    n = torch.arange(nb, device="cuda")
    rank = torch.rand(B, H, Sq, nb, generator=g, device="cuda")
    if case["pool"]:
        liked = torch.rand(B, H, -(-Sq // 64), nb, generator=g, device="cuda")
        size = min(nb, max(K, int(K * case["pool"])))
        cut = torch.sort(liked, dim=-1, descending=True).values[..., size - 1:size]
        rank = rank + (liked >= cut).float().repeat_interleave(64, 2)[:, :, :Sq]
    rank = torch.where((n < case["sinks"]) | (n > cur - case["local"]), 9.0, rank)
    rank = torch.where(n <= cur, rank, -1.0)
    best = torch.sort(rank, dim=-1, descending=True, stable=True)
    idx = torch.where(best.values >= 0, best.indices, nb)[..., :K]
    idx = torch.nn.functional.pad(idx, (0, K - idx.shape[-1]), value=nb)
    idx = torch.sort(idx, -1).values
    return torch.where(idx < nb, idx, -1).to(torch.int32).contiguous()


def _inputs(case, seed):
    g = _generator(seed)
    op, B, Hq, Hkv, Sq, D = (case[x] for x in ("op", "B", "Hq", "Hkv", "Sq", "D"))
    t = dict(lengths=torch.tensor(_lengths(case), dtype=torch.int32, device="cuda"))
    if op != SUMMARY:
        t["q"] = _normal(g, B, Hq, Sq, D)
    t["k"] = _keys(g, case)
    if op == SUMMARY:
        t["summary"] = torch.zeros(B, Hkv, _blocks_of(case), D, dtype=torch.bfloat16,
                                   device="cuda")
    if op == SELECT:
        t["summary"] = _means(t["k"], case["block"])
        del t["k"]
    if op in (BLOCKS, PREFIX):
        t["v"] = _normal(g, B, Hkv, case["Skv"], D)
    if op == BLOCKS:
        t["blocks"] = _lists(g, case)
    if op == PREFIX:
        t["kp"], t["vp"] = _normal(g, Hkv, case["Lp"], D), _normal(g, Hkv, case["Lp"], D)
    return t


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] in (BLOCKS, PREFIX):
        s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    if case["op"] == SELECT:
        s["out"] = torch.empty(case["B"], case["Hkv"], case["Sq"], case["topk"],
                               dtype=torch.int32, device="cuda")
    s["workspace"] = None
    if own and case["op"] in (BLOCKS, PREFIX):
        from paper_2609_12330_amd import ef_attention as ef
        if case["op"] == BLOCKS:
            s["workspace"] = ef.make_blocks_workspace(s["q"], s["k"], case["topk"], case["block"])
        else:
            s["workspace"] = ef.make_shared_prefix_workspace(s["q"], s["kp"], s["k"])
    return s


# --------------------------------------------------------------------------------- plain forms


def _plain_summary(s):
    c, k, out = s["case"], s["k"], s["summary"]
    B, H, S, D = k.shape
    bs, nb, new = c["block"], _blocks_of(c), c["new"]
    n = s["lengths"].long()
    # Blocks of each sequence that are written: all, or those of its last `new` keys.
    T = nb if new == 0 else min(nb, (new + bs - 2) // bs + 1)
    first = torch.zeros_like(n) if new == 0 else (n - new).clamp(min=0) // bs
    blk = first[:, None] + torch.arange(T, device=k.device)                   # [B][T]
    written = (blk < nb) & ((blk * bs < n[:, None]) | (new == 0))
    key = blk[:, :, None] * bs + torch.arange(bs, device=k.device)            # [B][T][bs]
    valid = (key < n[:, None, None]).float()
    at = key.clamp(max=S - 1).view(B, 1, T * bs, 1).expand(B, H, T * bs, D)
    x = torch.gather(k, 2, at).float().view(B, H, T, bs, D)
    total = (x * valid[:, None, :, :, None]).sum(3)
    mean = total / valid.sum(2).clamp(min=1)[:, None, :, None]
    to = blk.clamp(max=nb - 1)
    old = torch.gather(out, 2, to[:, None, :, None].expand(B, H, T, D))
    new_rows = torch.where(written[:, None, :, None], mean.to(torch.bfloat16), old)
    if new == 0:
        return out.copy_(new_rows)
    # A clamped block past the end repeats the last one: write each with its own rows only.
    sel = torch.nonzero(written)
    out[sel[:, 0], :, blk[sel[:, 0], sel[:, 1]]] = new_rows[sel[:, 0], :, sel[:, 1]]
    return out


def _plain_select(s):
    c, q, m = s["case"], s["q"], s["summary"]
    B, Hq, Sq, D = q.shape
    H, nb, K, bs = c["Hkv"], m.shape[2], c["topk"], c["block"]
    x = torch.matmul(q.double().reshape(B, H, -1, D), m.double().transpose(2, 3).contiguous())
    x = x.view(B, H, Hq // H, Sq, nb).amax(2)
    cur = s["lengths"].long()[:, None] - Sq + torch.arange(Sq, device=q.device)
    cur = torch.where(cur >= 0, cur // bs, -1)[:, None, :, None]
    n = torch.arange(nb, device=q.device)
    x = torch.where((n < c["sinks"]) | (n > cur - c["local"]), math.inf, x)
    x = torch.where(n <= cur, x, -math.inf)
    idx = torch.sort(x, dim=-1, descending=True, stable=True).indices
    idx = torch.where(idx <= cur, idx, nb)[..., :K]
    idx = torch.sort(torch.nn.functional.pad(idx, (0, K - idx.shape[-1]), value=nb), -1).values
    return torch.where(idx < nb, idx, -1).to(torch.int32)


def _plain_blocks(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    B, Hq, Sq, D = q.shape
    H, S, bs, K = c["Hkv"], c["Skv"], c["block"], c["topk"]
    G = Hq // H
    blk = s["blocks"].long()                                                  # [B][H][Sq][K]
    key = (blk.clamp(min=0)[..., None] * bs + torch.arange(bs, device=q.device)).flatten(3)
    diag = s["lengths"].long()[:, None] - Sq + torch.arange(Sq, device=q.device)
    seen = (blk >= 0).repeat_interleave(bs, -1) & (key <= diag[:, None, :, None])
    at = key.clamp(max=S - 1).flatten(2)[..., None].expand(B, H, Sq * K * bs, D)
    kg = torch.gather(k, 2, at).float().view(B * H * Sq, K * bs, D)
    qg = q.float().view(B, H, G, Sq, D).transpose(2, 3).reshape(B * H * Sq, G, D)
    x = torch.matmul(qg, kg.transpose(1, 2)).view(B, H, Sq, G, K * bs) * _scale(c)
    del kg
    x = torch.where(seen[..., None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total = w.sum(-1, keepdim=True)
    vg = torch.gather(v, 2, at).float().view(B * H * Sq, K * bs, D)
    o = torch.matmul(w.view(B * H * Sq, G, K * bs), vg).view(B, H, Sq, G, D)
    o = o / torch.where(total > 0, total, 1.0)
    return s["out"].copy_(o.transpose(2, 3).reshape(B, Hq, Sq, D))


def _plain_prefix(s):
    c, q, k, v, kp, vp = s["case"], s["q"], s["k"], s["v"], s["kp"], s["vp"]
    B, Hq, Sq, D = q.shape
    H, S, Lp = c["Hkv"], c["Skv"], c["Lp"]
    G = Hq // H
    qg = q.float().view(B, H, G * Sq, D)
    qp = qg.transpose(0, 1).reshape(H, B * G * Sq, D)
    xp = torch.matmul(qp, kp.float().transpose(1, 2)).view(H, B, G, Sq, Lp).transpose(0, 1)
    xs = torch.matmul(qg, k.float().transpose(2, 3)).view(B, H, G, Sq, S)
    x = torch.cat([xp, xs], -1) * _scale(c)
    n = s["lengths"].long()[:, None, None]
    key = torch.arange(Lp + S, device=q.device)
    seen = key < Lp + n
    if c["causal"]:
        seen = seen & (key <= Lp + n - Sq + torch.arange(Sq, device=q.device)[:, None])
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total = w.sum(-1, keepdim=True)
    wp = w[..., :Lp].transpose(0, 1).reshape(H, B * G * Sq, Lp)
    o = torch.matmul(wp, vp.float()).view(H, B, G, Sq, D).transpose(0, 1)
    o = o + torch.matmul(w[..., Lp:].reshape(B, H, G * Sq, S), v.float()).view(B, H, G, Sq, D)
    o = o / torch.where(total > 0, total, 1.0)
    return s["out"].copy_(o.reshape(B, Hq, Sq, D))


_PLAIN = {SUMMARY: _plain_summary, SELECT: _plain_select, BLOCKS: _plain_blocks,
          PREFIX: _plain_prefix}


def run(state):
    c = state["case"]
    if not own:
        return _PLAIN[c["op"]](state)
    from paper_2609_12330_amd import ef_attention as ef
    if c["op"] == SUMMARY:
        return ef.block_summary(state["k"], c["block"], lengths=state["lengths"],
                                new_keys=c["new"], out=state["summary"])
    if c["op"] == SELECT:
        return ef.block_select(state["q"], state["summary"], c["Skv"], c["topk"], c["block"],
                               c["sinks"], c["local"], lengths=state["lengths"],
                               out=state["out"])
    if c["op"] == BLOCKS:
        return ef.attention_blocks(state["q"], state["k"], state["v"], state["blocks"],
                                   c["block"], lengths=state["lengths"],
                                   workspace=state["workspace"], out=state["out"])
    return ef.attention_shared_prefix(state["q"], state["kp"], state["vp"], state["k"],
                                      state["v"], causal=c["causal"], lengths=state["lengths"],
                                      workspace=state["workspace"], out=state["out"])


# ---------------------------------------------------------------------------------------- work


def _scored(case, diag):
    """Blocks whose score decides for the query whose own key is `diag`."""
    cur = diag // case["block"]
    if diag < 0 or cur + 1 <= case["topk"]:
        return 0
    return max(0, cur - case["local"] + 1 - case["sinks"])


def work(case):
    op, B, Hq, Hkv, Sq, Skv, D = (case[x] for x in ("op", "B", "Hq", "Hkv", "Sq", "Skv", "D"))
    bs, K, Lp = case["block"], case["topk"], case["Lp"]
    lengths = _lengths(case)
    if op == SUMMARY:
        if case["new"]:
            keys = [n - (max(n - case["new"], 0) // bs) * bs for n in lengths]
            blocks = sum(-(-m // bs) for m in keys)
        else:
            keys, blocks = lengths, B * _blocks_of(case)
        return {"bytes": Hkv * D * 2 * (sum(keys) + blocks), "flops": Hkv * D * sum(keys)}
    diags = _diagonals(case)
    qo = 4 * B * Hq * Sq * D  # q and o in bf16
    if op == SELECT:
        scored = sum(_scored(case, d) for row in diags for d in row)
        read = sum(max(_scored(case, d) for d in row) for row in diags)
        return {"bytes": qo // 2 + Hkv * read * D * 2 + 4 * B * Hkv * Sq * K,
                "flops": 2 * D * Hq * scored}
    if op == BLOCKS:
        pairs, read = 0, 0
        for row in diags:
            seen = [min(d + 1, (K - 1) * bs + d % bs + 1) if d >= 0 else 0 for d in row]
            pairs += sum(seen)
            # Keys some query of the sequence reads: those of one list, or where lists differ of
            # the pools of each 64 queries, or of all blocks, at most all keys.
            groups = 1 if Sq == 1 else (-(-Sq // 64) * max(case["pool"], 1) if case["pool"] else Sq)
            read += min(max(row) + 1, int(max(seen) * groups)) if max(row) >= 0 else 0
        return {"bytes": qo + 4 * D * Hkv * read + 4 * B * Hkv * Sq * K,
                "flops": 4 * D * Hq * pairs}
    if case["causal"]:
        pairs = sum(max(0, Lp + d + 1) for row in diags for d in row)
    else:
        pairs = Sq * sum(Lp + n for n in lengths)
    return {"bytes": qo + 4 * D * Hkv * (Lp + sum(lengths)), "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------------------- in 64 bits


def _attend64(q, k, v, seen, scale):
    """Rows q [R][D] over keys [N][D], seen [R][N]."""
    x = (q @ k.t()) * scale
    x = x.masked_fill(~seen, -math.inf)
    w = torch.softmax(x, -1)
    return torch.nan_to_num(w, nan=0.0) @ v


def exact(case, seed):
    t = _inputs(case, seed)
    op, B, Hq, Hkv, Sq, Skv, D = (case[x] for x in ("op", "B", "Hq", "Hkv", "Sq", "Skv", "D"))
    bs, nb, lengths, G = case["block"], _blocks_of(case), _lengths(case), Hq // Hkv
    if op == SUMMARY:
        out = t["summary"].double()
        for b, n in enumerate(lengths):
            start = max(0, n - case["new"]) // bs * bs if case["new"] else 0
            for j in range(start, n if case["new"] else nb * bs, bs):
                m = min(j + bs, n) - j
                row = t["k"][b, :, j:j + m].double().mean(1) if m > 0 else 0.0
                out[b, :, j // bs] = row
        return out
    if op == SELECT:
        return None  # whole numbers: they have to equal the plain form's
    out = torch.empty(B, Hq, Sq, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            k, v = t["k"][b, h, :n].double(), t["v"][b, h, :n].double()
            if op == PREFIX:
                k = torch.cat([t["kp"][h].double(), k])
                v = torch.cat([t["vp"][h].double(), v])
            N = k.shape[0]
            step = max(1, (1 << 27) // max(1, G * N))
            for i in range(0, Sq, step):
                e = min(i + step, Sq)
                q = t["q"][b, h * G:(h + 1) * G, i:e].double().reshape(-1, D)
                diag = torch.arange(i, e, device="cuda") + (N - Sq)
                seen = torch.arange(N, device="cuda") <= diag[:, None]
                if op == PREFIX and not case["causal"]:
                    seen = torch.ones_like(seen)
                if op == BLOCKS:
                    lists = t["blocks"][b, h, i:e].long()
                    on = torch.zeros(e - i, nb + 1, dtype=torch.bool, device="cuda")
                    on.scatter_(1, torch.where(lists >= 0, lists, nb), True)
                    seen &= on[:, :nb].repeat_interleave(bs, 1)[:, :N]
                out[b, h * G:(h + 1) * G, i:e] = _attend64(
                    q, k, v, seen.repeat(G, 1), _scale(case)).view(G, e - i, D)
    return out

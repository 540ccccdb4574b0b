"""The cache's life between prefill and the end of a long dialogue, call by call.

A decoder that revisits image regions appends the K/V rows of its new tokens to the cache, attends with chunks of new
tokens (a whole prompt, the next piece of one, a few drafted tokens, a single token) over what the cache holds, adds up
how much attention each slot gets, and, as revisits make the cache grow, evicts the slots that get the least. Each case
is one such call on inputs of the shapes of ``workloads/configs.py`` or of generic odd ones:

  op        call                                                           sizes
  append    append_kv: new tokens' keys rotated and written with values    1..16 sequences, 1..8192 tokens in all, 1..36 layers
  chunk     chunk_attention of one layer over the cache                    1..32 sequences, 1..8192 new tokens each, contexts up to 32,768
  weights   accumulate_weights of one decode step, every layer             1..16 sequences of up to 16,384 slots
  evict     evict to a budget of slots per sequence, every layer           1..16 sequences of up to 16,384 slots

with 1..8 KV heads, GQA groups of 1..8, head_dim 64, 128 (the usual one) and 256, contiguous caches and paged ones of
several block sizes, and both M-RoPE band layouts. K/V and queries are bf16 N(0, 1), made on the GPU from the seed. What
decides how much work a case is (token counts, lengths) follows from the case alone.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
THETA = 1.0e6


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def listed():
    b8 = dict(kv_heads=8, group=4, head_dim=128, sec_t=24, layout="sectioned")   # Qwen3-VL-8B geometry
    b7 = dict(kv_heads=4, group=7, head_dim=128, sec_t=16, layout="sectioned")   # Qwen2.5-VL-7B geometry
    paged = dict(cache="paged", block=16)
    flat = dict(cache="contiguous", block=1)
    return [
        # one decode step of a serving batch: every sequence's new text token, all layers (latency)
        dict(name="append-8b-step", op="append", layers=36, seqs=16, q_max=1, ctx_max=4000, pad=0, **b8, **paged),
        # the packed prompts of six requests, all layers at once: the most rows an append moves
        dict(name="append-7b-prompts", op="append", layers=28, seqs=6, q_max=2116, ctx_max=0, pad=12, **b7, **paged),
        # a single new token of one user over a short context: the smallest attention, latency alone
        dict(name="chunk-8b-token", op="chunk", layers=1, seqs=1, q_max=1, ctx_max=932, pad=0, **b8, **flat),
        # drafted tokens of a serving batch checked in one pass: a few queries each over a long cache, bound by memory
        dict(name="chunk-8b-verify", op="chunk", layers=1, seqs=16, q_max=6, ctx_max=8192, pad=0, **b8, **paged),
        # packed prompts of six requests with images of about 2116 tokens, an odd group, ragged lengths, padded rows
        dict(name="chunk-7b-prompts", op="chunk", layers=1, seqs=6, q_max=2116, ctx_max=0, pad=12, **b7, **flat),
        # the next 1024 tokens of each of four long prompts over what the cache holds of them (chunked prefill)
        dict(name="chunk-8b-extend", op="chunk", layers=1, seqs=4, q_max=1024, ctx_max=15360, pad=0, **b8, **paged),
        # one whole prompt of two 4096-token images, causal: the most operations
        dict(name="chunk-8b-prompt", op="chunk", layers=1, seqs=1, q_max=8192, ctx_max=0, pad=0, **b8, **paged),
        # head_dim 256, eight query heads per KV head, a prompt's second half
        dict(name="chunk-d256", op="chunk", layers=1, seqs=2, q_max=1500, ctx_max=2000, pad=0, kv_heads=4, group=8, head_dim=256,
             sec_t=48, layout="sectioned", **paged),
        # one user's decode step: which slots of a short context get attention, every layer
        dict(name="weights-8b-b1", op="weights", layers=36, seqs=1, len_max=933, **b8, **flat),
        # the same for a serving batch of long contexts
        dict(name="weights-8b-b16", op="weights", layers=36, seqs=16, len_max=4096, **b8, **paged),
        # one user's cache of 4096 slots cut to 1024
        dict(name="evict-8b-b1", op="evict", layers=36, seqs=1, len_max=4096, budget=1024, sink=4, recent=128, **b8, **paged),
        # a serving batch's caches of up to 8192 slots cut to 2048, odd block size: the most rows an eviction moves
        dict(name="evict-7b-b8", op="evict", layers=28, seqs=8, len_max=8192, budget=2048, sink=16, recent=500,
             **b7, cache="paged", block=7),
    ]


_MOST_BYTES = 2.8e9   # of a drawn case's pass: below the largest listed one's
_MOST_FLOPS = 5.0e11


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "chunk", "chunk", "chunk", "chunk", "weights", "weights", "evict", "evict"])
    D = rng.choice([64, 128, 128, 128, 128, 256])
    H = rng.choice([1, 2, 3, 4, 4, 5, 8, 8])
    g = rng.choice([1, 2, 3, 4, 4, 6, 7, 8])
    while H * g * D > 8192 or H * g > 64:
        g = max(1, g // 2)
    c = dict(op=op, kv_heads=H, group=g, head_dim=D, sec_t=rng.randint(D // 16, D // 4), layout=rng.choice(["sectioned", "sectioned", "interleaved"]))
    c.update(rng.choice([dict(cache="contiguous", block=1), dict(cache="paged", block=16),
                         dict(cache="paged", block=rng.choice([8, 16, 32, 64, 7]))]))
    if op == "append":
        c.update(layers=_log_int(rng, 1, 36), seqs=_log_int(rng, 1, 16), q_max=_log_int(rng, 1, 2500), ctx_max=_log_int(rng, 1, 6000),
                 pad=rng.choice([0, 0, 5]))
    elif op == "chunk":
        kind = rng.choice(["prompt", "extend", "few", "few"])
        q = _log_int(rng, 16, 8192) if kind == "prompt" else _log_int(rng, 16, 2048) if kind == "extend" else rng.randint(1, 12)
        c.update(layers=rng.choice([1, 2]), seqs=_log_int(rng, 1, 32 if kind == "few" else 8), q_max=q,
                 ctx_max=0 if kind == "prompt" else _log_int(rng, 64, 32768), pad=rng.choice([0, 0, 9]))
    else:
        c.update(layers=_log_int(rng, 1, 36), seqs=_log_int(rng, 1, 16), len_max=_log_int(rng, 64, 16384))
        if op == "evict":
            budget = max(8, int(c["len_max"] * rng.uniform(0.1, 0.9)))
            c.update(budget=budget, sink=rng.choice([0, 4, budget // 8]), recent=rng.choice([0, budget // 8, budget // 3]))
    while work(c)["bytes"] > _MOST_BYTES or work(c)["flops"] > _MOST_FLOPS or _plain_bytes(c) > 10.0e9:
        if c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
        elif c["layers"] > 1:
            c["layers"] = (c["layers"] + 1) // 2
        elif c["ctx_max"] > 1:
            c["ctx_max"] //= 2
        else:
            c["q_max"] = (c["q_max"] + 1) // 2
    return c


# ----------------------------------------------------------------------------
# what follows from the case alone
# ----------------------------------------------------------------------------
def _sections(c):
    P = c["head_dim"] // 2
    h = (P - c["sec_t"]) // 2
    return (c["sec_t"], h, P - c["sec_t"] - h)


def _spread(c, what, most):
    """A number of each sequence, from a quarter of `most` to `most`; the last one's is `most`."""
    rng = np.random.default_rng([sum(map(ord, what)), c["seqs"], most])
    n = rng.integers(max(1, most // 4) if most else 0, most + 1, size=c["seqs"])
    n[-1] = most
    return [int(x) for x in n]


def _new(c):
    return _spread(c, "new", c["q_max"])


def _before(c):
    return _spread(c, "before", c["ctx_max"])


def _lengths(c):
    """Slots that each sequence's cache holds (behind an append: with the new ones)."""
    if c["op"] in ("append", "chunk"):
        return [a + b for a, b in zip(_before(c), _new(c))]
    return _spread(c, "lengths", c["len_max"])


def _plain_bytes(c):
    """About the memory of the plain form's largest array."""
    H, D, g, B = c["kv_heads"], c["head_dim"], c["group"], c["seqs"]
    if c["op"] == "chunk":
        return 4.0 * B * H * g * c["q_max"] * max(_lengths(c))
    return 4.0 * B * c["layers"] * H * D * max(_lengths(c))


def work(c):
    H, D, L, B = c["kv_heads"], c["head_dim"], c["layers"], c["seqs"]
    Hq, row = H * c["group"], 2 * H * D
    if c["op"] == "append":  # K and V rows read and written
        T = sum(_new(c))
        return {"bytes": float(T * (L * 4 * row + 12) + 12 * B), "flops": float(T * L * H * D * 3)}
    if c["op"] == "chunk":  # queries, the slots' K and V read; outputs written
        T, S = sum(_new(c)), sum(_lengths(c))
        seen = sum(n * (s - n) + n * (n + 1) // 2 for n, s in zip(_new(c), _lengths(c)))
        return {"bytes": float(T * (4 * Hq * D + 12) + S * 2 * row + 8 * B), "flops": float(seen * Hq * (4 * D + 8))}
    S = sum(_lengths(c))
    if c["op"] == "weights":  # keys and queries read, scores read and written
        return {"bytes": float(S * L * (row + 8 * H) + B * L * Hq * D * 2), "flops": float(S * L * Hq * (2 * D + 8))}
    kept = sum(min(n, c["budget"]) for n in _lengths(c))  # scores read, kept rows moved, scores and indices written
    return {"bytes": float(L * H * (4 * S + kept * 8 * D + B * 4 * (max(_lengths(c)) + c["budget"]))), "flops": float(S * L * H)}


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _gen(seed, which):
    return torch.Generator(device=DEV).manual_seed(1000003 * (int(seed) % (1 << 40)) + which)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _to(a, dtype):
    return torch.as_tensor(np.asarray(a), dtype=dtype).to(DEV)


def _tables(c, rng, counts):
    """Block tables of one pool: a row of blocks for each sequence of each list of slot counts, and the pool's size."""
    bs = c["block"]
    need = [[-(-n // bs) for n in ns] for ns in counts]
    total = sum(map(sum, need))
    perm, at, out = rng.permutation(total + 3), 0, []  # a few blocks of the pool stay unused
    for blocks in need:
        table = np.full((c["seqs"], max(blocks) + 1), -1, dtype=np.int32)
        for b, n in enumerate(blocks):
            table[b, :n] = perm[at:at + n]
            at += n
        out.append(_to(table, torch.int32))
    return out, total + 3


def _cache(c, rng, gens, counts):
    """(k, v, block tables): a cache whose rows are N(0, 1), as a model's context is; one table for each list of counts."""
    H, D, L = c["kv_heads"], c["head_dim"], c["layers"]
    if c["cache"] == "contiguous":
        tables, shape = [None] * len(counts), (c["seqs"], L, max(map(max, counts)) + 8, H, D)
    else:
        tables, blocks = _tables(c, rng, counts)
        shape = (L, blocks, c["block"], H, D)
    return _normal(shape, gens[0]), _normal(shape, gens[1]), tables


def _coords(c, rng):
    """[T + pad, 3]: the first half of a sequence's new tokens an image (rows of 46 patches), the rest text behind it."""
    out = []
    for n, before in zip(_new(c), _before(c)):
        p, i = before + int(rng.integers(0, 20000)), np.arange(n)
        m = n // 2
        img = np.stack([np.full(m, p), p + i[:m] // 46, p + i[:m] % 46], 1)
        text = p + 46 + i[m:]
        out += [img, np.stack([text] * 3, 1)]
    out.append(np.zeros((c["pad"], 3), dtype=np.int64))
    return _to(np.concatenate(out), torch.int32)


def prepare(case, seed):
    c, rng = case, np.random.default_rng([int(seed) % (1 << 32), 77])
    H, D, L, B = c["kv_heads"], c["head_dim"], c["layers"], c["seqs"]
    s = dict(c=c, op=c["op"])
    lens = _lengths(c)
    gens = [_gen(seed, 1), _gen(seed, 2)]
    if c["op"] in ("append", "chunk"):
        T = sum(_new(c)) + c["pad"]
        s["coords"] = _coords(c, rng)
        s["off"] = _to(np.concatenate([[0], np.cumsum(_new(c))]), torch.int32)
        s["k"], s["v"], (s["table"],) = _cache(c, rng, gens, [lens])
        if c["op"] == "append":
            s["len_in"] = _to(_before(c), torch.int32)
            s["k_new"], s["v_new"] = (_normal((L, T, H, D), _gen(seed, w)) for w in (3, 4))
        else:
            s["len"] = _to(lens, torch.int32)
            s["q"] = _normal((T, H * c["group"], D), _gen(seed, 3))
        return s
    s["len"] = _to(lens, torch.int32)
    top = max(lens) + 16
    # attention so far: most slots little, a few much (a product of uniforms)
    u = torch.rand((2, B, L, H, top), generator=_gen(seed, 5), device=DEV)
    s["score"] = torch.where(torch.arange(top, device=DEV) < s["len"].view(B, 1, 1, 1), u[0] * u[1] * u[1], 0.0)
    if c["op"] == "weights":
        s["k"], s["v"], (s["table"],) = _cache(c, rng, gens, [lens])
        s["q"] = _normal((B, L, H * c["group"], D), _gen(seed, 3))
        s["q_pos"] = _to(np.asarray(lens) + rng.integers(0, 20000, B), torch.int64)
        return s
    kept = [min(n, c["budget"]) for n in lens]
    if c["cache"] == "contiguous":  # into another cache
        s["k"], s["v"], _ = _cache(c, rng, gens, [lens])
        s["table"] = s["to_table"] = None
        s["to_k"], s["to_v"] = (torch.zeros((B, L, c["budget"] + 8, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:  # into other blocks of the pool
        s["k"], s["v"], (s["table"], s["to_table"]) = _cache(c, rng, gens, [lens, kept])
        s["to_k"], s["to_v"] = s["k"], s["v"]
    return s


# ----------------------------------------------------------------------------
# the framework's calls
# ----------------------------------------------------------------------------
def _kept(s):
    """What a program makes once and keeps: descriptors, outputs, workspace."""
    import paper_2606_26631_gb300 as prcr
    c = s["c"]
    B, Hq = c["seqs"], c["kv_heads"] * c["group"]
    cfg = prcr.rope_cfg(c["layers"], c["kv_heads"], c["head_dim"], _sections(c), THETA,
                        prcr.LAYOUT_INTERLEAVED if c["layout"] == "interleaved" else prcr.LAYOUT_SECTIONED)

    def desc(k, v, table):
        return prcr.cache_contiguous(k, v) if table is None else prcr.cache_paged(k, v, table)

    h = dict(prcr=prcr, cfg=cfg, cache=desc(s["k"], s["v"], s["table"]), status=torch.zeros(1, dtype=torch.int32, device=DEV),
             top=max(_lengths(c)))
    nbytes = 0
    if s["op"] == "append":
        h["len_out"] = torch.zeros_like(s["len_in"])
    elif s["op"] == "chunk":
        h["out"] = torch.zeros_like(s["q"])
        nbytes = prcr.chunk_workspace_size(cfg, B, Hq, s["q"].shape[0], h["top"])
    elif s["op"] == "weights":
        nbytes = prcr.weights_workspace_size(cfg, B, Hq, h["top"])
    else:
        h["dst"] = desc(s["to_k"], s["to_v"], s["to_table"])
        h["keep"] = torch.zeros((B, c["layers"], c["kv_heads"], c["budget"]), dtype=torch.int32, device=DEV)
        h["score_out"] = torch.zeros_like(s["score"])
        h["len_out"] = torch.zeros_like(s["len"])
    h["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)
    return h


def _run_own(s):
    if "own" not in s:
        s["own"] = _kept(s)
    h, c = s["own"], s["c"]
    prcr = h["prcr"]
    if s["op"] == "append":
        prcr.append_kv(h["cfg"], h["cache"], 0, s["k_new"], s["v_new"], s["coords"], s["off"], s["len_in"], h["len_out"], h["status"])
        return {"k": s["k"], "v": s["v"], "len": h["len_out"]}
    if s["op"] == "chunk":
        prcr.chunk_attention(h["cfg"], h["cache"], c["layers"] - 1, s["q"], s["coords"], s["off"], s["len"], h["top"], h["out"],
                             h["status"], h["ws"])
        return {"out": h["out"]}
    if s["op"] == "weights":
        prcr.accumulate_weights(h["cfg"], h["cache"], s["q"], s["q_pos"], s["len"], h["top"], s["score"], h["status"], 1.0, h["ws"])
        return {"score": s["score"]}
    prcr.evict(h["cfg"], h["cache"], s["len"], h["top"], c["budget"], c["sink"], c["recent"], s["score"], h["keep"], h["len_out"],
               h["status"], dst=h["dst"], score_out=h["score_out"])
    return {"keep": h["keep"], "len": h["len_out"], "k": s["to_k"], "v": s["to_v"], "score": h["score_out"]}


# ----------------------------------------------------------------------------
# the plain form: elementary torch operations in 32 bits
# ----------------------------------------------------------------------------
def _rotate(x, pos, c):
    """x [..., n, heads, D] at pos [n, 3]: pairs (i, i + D/2); the angles in 64 bits, the rest in 32."""
    D, (st, sh, sw) = c["head_dim"], _sections(c)
    i = torch.arange(D // 2, device=x.device)
    if c["layout"] == "interleaved":
        axis = torch.where((i % 3 == 1) & (i < 3 * sh), 1, torch.where((i % 3 == 2) & (i < 3 * sw), 2, 0))
    else:
        axis = (i >= st).long() + (i >= st + sh).long()
    ang = pos.double()[:, axis] * THETA ** (-2.0 * i.double() / D)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _row_index(c, table, shape, slots):
    """Rows of a cache seen as [rows, H, D]: of slot `slots` [B, 1 or L, n] of every sequence, at every layer: [B, L, n]."""
    B, L = c["seqs"], c["layers"]
    layer, seq = torch.arange(L, device=DEV).view(1, L, 1), torch.arange(B, device=DEV).view(B, 1, 1)
    if table is None:
        return (seq * L + layer) * shape[2] + slots
    blocks, bs = shape[1], shape[2]
    blk = table.long()[seq, slots // bs].clamp(min=0)
    return (layer * blocks + blk) * bs + slots % bs


def _flat(x):
    return x.view(-1, x.shape[-2], x.shape[-1])


def _plain_append(s):
    c, off = s["c"], s["off"].long()
    T = s["k_new"].shape[1]
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    t = t[b < c["seqs"]]
    b = b[b < c["seqs"]]
    slot = s["len_in"].long()[b] + t - off[b]
    layer = torch.arange(c["layers"], device=DEV).view(-1, 1)
    if s["table"] is None:
        rows = (b * c["layers"] + layer) * s["k"].shape[2] + slot
    else:
        bs = c["block"]
        rows = (layer * s["k"].shape[1] + s["table"].long()[b, slot // bs]) * bs + slot % bs
    _flat(s["k"])[rows] = _rotate(s["k_new"][:, t], s["coords"][t], c).bfloat16()
    _flat(s["v"])[rows] = s["v_new"][:, t]
    return {"k": s["k"], "v": s["v"], "len": s["len_in"] + (off[1:] - off[:-1]).int()}


def _plain_chunk(s):
    c, off, n_slots = s["c"], s["off"].long(), s["len"].long()
    B, H, g, D = c["seqs"], c["kv_heads"], c["group"], c["head_dim"]
    N, S = max(_new(c)), max(_lengths(c))
    t = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    t, b = t[b < B], b[b < B]
    i = t - off[b]
    one = dict(c, layers=1)
    k, v = (x[:, -1:] if s["table"] is None else x[-1:] for x in (s["k"], s["v"]))
    rows = _row_index(one, s["table"], k.shape, torch.arange(S, device=DEV).view(1, 1, S).expand(B, 1, S))[:, 0]
    k, v = (_flat(x.contiguous())[rows].float().permute(0, 2, 1, 3) for x in (k, v))  # [B, H, S, D]
    q = torch.zeros((B, N, H * g, D), device=DEV)
    q[b, i] = _rotate(s["q"][t], s["coords"][t], c)
    q = q.view(B, N, H, g, D).permute(0, 2, 3, 1, 4).reshape(B, H, g * N, D)
    n_new = off[1:] - off[:-1]
    last = (n_slots - n_new).view(B, 1) + torch.arange(N, device=DEV)  # the last slot that each query sees
    hidden = torch.arange(S, device=DEV) > last.view(B, 1, 1, N, 1)
    x = (q @ k.transpose(-1, -2)).view(B, H, g, N, S) / math.sqrt(D)
    x.masked_fill_(hidden, -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp_()
    o = (x.view(B, H, g * N, S) @ v).view(B, H, g, N, D) / x.sum(-1, keepdim=True)
    out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    out[t] = o.permute(0, 3, 1, 2, 4).reshape(B, N, H * g, D)[b, i].bfloat16()
    return {"out": out}


def _plain_weights(s):
    c = s["c"]
    B, L, H, g, D = c["seqs"], c["layers"], c["kv_heads"], c["group"], c["head_dim"]
    S = max(_lengths(c))
    rows = _row_index(c, s["table"], s["k"].shape, torch.arange(S, device=DEV).view(1, 1, S).expand(B, 1, S))
    k = _flat(s["k"])[rows].float().permute(0, 1, 3, 2, 4)  # [B, L, H, S, D]
    pos = s["q_pos"].view(B, 1).expand(B, 3)
    q = _rotate(s["q"].transpose(0, 1), pos, c).transpose(0, 1).reshape(B, L, H, g, D)
    x = (k @ q.transpose(-1, -2)).transpose(-1, -2) / math.sqrt(D)
    x.masked_fill_(torch.arange(S, device=DEV) >= s["len"].view(B, 1, 1, 1, 1), -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp_()
    s["score"][..., :S] += (x / x.sum(-1, keepdim=True)).sum(3)
    return {"score": s["score"]}


def _plain_evict(s):
    c = s["c"]
    B, L, H, D, budget = c["seqs"], c["layers"], c["kv_heads"], c["head_dim"], c["budget"]
    n, slot = s["len"].long().view(B, 1, 1, 1), torch.arange(s["score"].shape[-1], device=DEV)
    safe = (slot < c["sink"]) | (slot >= n - c["recent"])
    rank = torch.where(slot >= n, -1.0, torch.where(safe, math.inf, s["score"]))
    best = rank.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    best = torch.where(n > budget, best, torch.arange(budget, device=DEV)).sort(-1).values
    there = torch.arange(budget, device=DEV) < n
    keep = torch.where(there, best, -1)
    score = torch.zeros_like(s["score"])
    score[..., :budget] = torch.where(there, s["score"].gather(-1, best.clamp(max=s["score"].shape[-1] - 1)), 0.0)
    # rows: [B, L, H, budget] of one head each
    head = torch.arange(H, device=DEV).view(1, 1, H, 1).expand(B, L, H, budget)[there.expand(B, L, H, budget)]
    src = torch.where(there, best, 0).reshape(B, L, H * budget)
    dst = torch.where(there, torch.arange(budget, device=DEV), 0).expand(B, L, H, budget).reshape(B, L, H * budget)
    ok = there.expand(B, L, H, budget).reshape(-1)
    src = _row_index(c, s["table"], s["k"].shape, src).reshape(-1)[ok]
    dst = _row_index(c, s["to_table"], s["to_k"].shape, dst).reshape(-1)[ok]
    for a, b in ((s["k"], s["to_k"]), (s["v"], s["to_v"])):
        _flat(b)[dst, head] = _flat(a)[src, head]
    return {"keep": keep.int(), "len": s["len"].clamp(max=budget), "k": s["to_k"], "v": s["to_v"], "score": score}


_PLAIN = {"append": _plain_append, "chunk": _plain_chunk, "weights": _plain_weights, "evict": _plain_evict}


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["op"]](state)


# ----------------------------------------------------------------------------
# the definition in 64 bits, a sequence and a head at a time
# ----------------------------------------------------------------------------
def _turned(x, pos, c):
    """RoPE of x [..., D] (64 bits) by complex numbers: pair i of a token at (t, h, w) turns by its axis' coordinate."""
    D, secs = c["head_dim"], _sections(c)
    axis = np.repeat([0, 1, 2], secs)
    if c["layout"] == "interleaved":
        axis = np.array([1 if i % 3 == 1 and i < 3 * secs[1] else 2 if i % 3 == 2 and i < 3 * secs[2] else 0 for i in range(D // 2)])
    rate = torch.from_numpy(np.exp(-2.0 * np.arange(D // 2) / D * np.log(THETA))).to(DEV)
    a = pos.to(torch.float64)[..., torch.from_numpy(axis).to(DEV)] * rate
    z = torch.complex(x[..., : D // 2], x[..., D // 2:]) * torch.polar(torch.ones_like(a), a)
    return torch.cat([z.real, z.imag], -1)


def _slots(c, s, x, b, layer, n, table="table"):
    """Rows of slots 0 .. n - 1 of sequence b at `layer`: [n, H, D] in 64 bits."""
    if s[table] is None:
        return x[b, layer, :n].double()
    blocks = s[table][b, : -(-n // c["block"])].long()
    return x[layer, blocks].flatten(0, 1)[:n].double()


def exact(case, seed):
    s, c = prepare(case, seed), case
    H, g, D = c["kv_heads"], c["group"], c["head_dim"]
    if c["op"] == "append":
        k, v = s["k"].double(), s["v"].clone()
        at = 0
        for b, (n, before) in enumerate(zip(_new(c), _before(c))):
            new = _turned(s["k_new"][:, at:at + n].double(), s["coords"][at:at + n].unsqueeze(1), c)
            slot = torch.arange(before, before + n, device=DEV)
            if s["table"] is None:
                k[b, :, slot], v[b, :, slot] = new, s["v_new"][:, at:at + n]
            else:
                blk, o = s["table"][b, slot // c["block"]].long(), slot % c["block"]
                k[:, blk, o], v[:, blk, o] = new, s["v_new"][:, at:at + n]
            at += n
        return {"k": k, "v": v, "len": _to(_lengths(c), torch.int32)}
    if c["op"] == "chunk":
        out, at = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), 0
        for b, (n, total) in enumerate(zip(_new(c), _lengths(c))):
            K, V = (_slots(c, s, s[x], b, c["layers"] - 1, total) for x in "kv")
            q = _turned(s["q"][at:at + n].double(), s["coords"][at:at + n].unsqueeze(1), c)
            sees = torch.arange(total, device=DEV) <= torch.arange(total - n, total, device=DEV).view(n, 1)
            for h in range(H * g):
                x = q[:, h] @ K[:, h // g].T / D ** 0.5
                out[at:at + n, h] = torch.softmax(torch.where(sees, x, -torch.inf), -1) @ V[:, h // g]
            at += n
        return {"out": out}
    if c["op"] == "weights":
        score = s["score"].double()
        for b, total in enumerate(_lengths(c)):
            for l in range(c["layers"]):
                K = _slots(c, s, s["k"], b, l, total)
                q = _turned(s["q"][b, l].double(), s["q_pos"][b].expand(1, 3), c).view(H, g, D)
                score[b, l, :, :total] += torch.softmax(torch.einsum("hgd,shd->hgs", q, K) / D ** 0.5, -1).sum(1)
        return {"score": score}
    # evict: which slots stay, by numpy's sort; the rows and scores are copies
    keep = np.full((c["seqs"], c["layers"], H, c["budget"]), -1, dtype=np.int64)
    sc, score = s["score"].cpu().numpy(), np.zeros(tuple(s["score"].shape), dtype=np.float32)
    to_k, to_v = s["to_k"].clone(), s["to_v"].clone()
    for b, total in enumerate(_lengths(c)):
        n = min(total, c["budget"])
        if total > n:
            end, free = total - c["recent"], n - c["sink"] - c["recent"]
            order = np.argsort(-sc[b, :, :, c["sink"]:end], axis=-1, kind="stable")[..., :free] + c["sink"]
            ends = np.concatenate([np.arange(c["sink"]), np.arange(end, total)])
            keep[b] = np.sort(np.concatenate([order, np.broadcast_to(ends, order.shape[:2] + ends.shape)], -1), -1)
        else:
            keep[b, :, :, :n] = np.arange(n)
        score[b, :, :, :n] = np.take_along_axis(sc[b], keep[b, :, :, :n], -1)
        at = _to(keep[b, :, :, :n], torch.int64)
        for l in range(c["layers"]):
            for x, to in (("k", to_k), ("v", to_v)):
                rows = _slots(c, s, s[x], b, l, total).gather(0, at[l].T.unsqueeze(-1).expand(n, H, D)).bfloat16()
                if s["to_table"] is None:
                    to[b, l, :n] = rows
                else:
                    i = torch.arange(n, device=DEV)
                    to[l, s["to_table"][b, i // c["block"]].long(), i % c["block"]] = rows
    return {"keep": _to(keep, torch.int32), "len": _to([min(n, c["budget"]) for n in _lengths(c)], torch.int32), "k": to_k, "v": to_v,
            "score": _to(score, torch.float32)}

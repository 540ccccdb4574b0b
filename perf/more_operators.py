"""A decoder cache held in 8 or 4 bits, call by call: rows quantised as they are written, read back, and attended to.

A decoder that revisits image regions grows its cache with every revisit; held in fewer bits, it takes half or a quarter of
the memory, and of the time that a decode step spends on reading it. Each case is one step of such a decoder, on inputs of the
shapes of ``workloads/configs.py`` or of generic odd ones:

  op        calls                                                            sizes
  append    append_kv_quant: new tokens' keys rotated, K and V rounded into   1..32 sequences, 1..16,384 tokens in all, 1..36 layers
            the cache; dequantize_cache of those rows for the model's own
            attention over them
  cast      quantize_cache: slots of a bf16 cache (a revisit's rows, a whole   1..32 sequences of up to 8192 slots
            context) into the cache; dequantize_cache of them
  read      dequantize_cache: the rows that chunks of tokens attend over        1..32 sequences of up to 16,384 slots
  decode    decode_attention_quant: one new token of each sequence over the     1..64 sequences of up to 32,768 slots, one layer or all
            whole cache

with 1..8 KV heads, GQA groups of 1..8, head_dim 64, 128 (the usual one) and 256 (8-bit rows alone: also 80, 96 and 192),
contiguous caches and paged ones of several block sizes.

Formats: "e4m3" holds a value in a byte and a scale for each (slot, KV head) row; "e2m1" holds a value in four bits (dim 2i
in the low half of byte i) and a scale for each of D/32 groups of 32 dims, group j the dims d with d / 4 mod D/32 = j. A scale
is a power of two, 2^e with the least e >= -117 for which the group's largest magnitude is at most 448 * 2^e (6 * 2^e), and
is held as the byte e + 127; a value is rounded to the nearest one of the format, ties to even. New rows are N(0, 1) bf16
with a magnitude of each row's own. Cases of op append and cast return what the written rows stand for, in bf16, which holds
every such value exactly. Rounding to 4 bits is op cast's alone: there both sides start from the same numbers, where a rotated
key that lies next to a border between two values may fall to either side of it, which are up to half of the value apart.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
THETA = 1.0e6
LEAST = -117  # the least exponent of a scale


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
        dict(name="append-8b-step", op="append", fmt="e4m3", layers=36, seqs=16, n_max=1, ctx_max=4000, pad=0, empty=False, **b8, **paged),
        # the packed prompts of six requests with images, all layers at once: the most rows an append moves
        dict(name="append-7b-prompts", op="append", fmt="e4m3", layers=28, seqs=6, n_max=2116, ctx_max=0, pad=12, empty=False, **b7, **paged),
        # the next piece of two users' prompts, an odd head_dim and an odd number of heads
        dict(name="append-d80", op="append", fmt="e4m3", layers=24, seqs=2, n_max=500, ctx_max=3001, pad=5, empty=False, kv_heads=5,
             group=2, head_dim=80, sec_t=16, layout="interleaved", **flat),
        # a revisit's rows (four regions of up to 1024 tokens in all for each of 16 sequences), rebound into bf16 rows, join the cache
        dict(name="cast-8b-revisit", op="cast", fmt="e4m3", layers=36, seqs=16, n_max=1024, ctx_max=4000, empty=False, **b8, **paged),
        # one user's whole context goes from bf16 to four bits
        dict(name="cast-8b-e2m1", op="cast", fmt="e2m1", layers=36, seqs=1, n_max=933, ctx_max=0, empty=False, **b8, **flat),
        # one layer's rows of four long prompts, before the next piece of each attends over them
        dict(name="read-8b-layer", op="read", fmt="e4m3", layers=1, seqs=4, n_max=16384, empty=False, **b8, **paged),
        # every layer's rows of a serving batch, to be weighed and evicted from
        dict(name="read-7b-e2m1", op="read", fmt="e2m1", layers=28, seqs=8, n_max=4096, empty=False, **b7, cache="paged", block=7),
        # one user's decode step over a short context, every layer: latency
        dict(name="decode-8b-b1", op="decode", fmt="e4m3", layers=36, seqs=1, n_max=933, empty=False, **b8, **flat),
        # the same for a serving batch: the most bytes a step reads
        dict(name="decode-8b-b16", op="decode", fmt="e4m3", layers=36, seqs=16, n_max=4096, empty=False, **b8, **paged),
        # a serving batch in four bits, an odd group
        dict(name="decode-7b-e2m1", op="decode", fmt="e2m1", layers=28, seqs=8, n_max=8192, empty=False, **b7, **paged),
        # one layer, as a decoder calls it layer by layer: long contexts of ragged lengths, one sequence without any slot
        dict(name="decode-8b-layer", op="decode", fmt="e4m3", layers=1, seqs=32, n_max=16384, empty=True, **b8, **paged),
        # head_dim 256, eight query heads per KV head
        dict(name="decode-d256", op="decode", fmt="e4m3", layers=1, seqs=8, n_max=8000, empty=False, kv_heads=4, group=8, head_dim=256,
             sec_t=48, layout="sectioned", cache="paged", block=32),
    ]


_MOST_BYTES = 2.5e9   # of a drawn case's pass: below the largest listed one's


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "cast", "read", "decode", "decode", "decode"])
    fmt = "e4m3" if op == "append" else rng.choice(["e4m3", "e4m3", "e2m1"])
    D = rng.choice([64, 128, 128, 128, 256] + [80, 96, 192] * (op != "decode" and fmt == "e4m3"))
    H = rng.choice([1, 2, 3, 4, 4, 5, 8, 8])
    g = rng.choice([1, 2, 3, 4, 4, 6, 7, 8])
    while H * g * D > 8192:
        g = max(1, g // 2)
    c = dict(op=op, fmt=fmt, kv_heads=H, group=g, head_dim=D, sec_t=rng.randint(D // 16, D // 4),
             layout=rng.choice(["sectioned", "sectioned", "interleaved"]), empty=rng.random() < 0.2)
    c.update(rng.choice([dict(cache="contiguous", block=1), dict(cache="paged", block=16),
                         dict(cache="paged", block=rng.choice([8, 16, 32, 64, 7]))]))
    if op == "decode":
        one = rng.random() < 0.5
        c.update(layers=1 if one else _log_int(rng, 2, 36), seqs=_log_int(rng, 1, 64 if one else 16), n_max=_log_int(rng, 1, 32768))
    else:
        c.update(layers=_log_int(rng, 1, 36), seqs=_log_int(rng, 1, 32))
        c.update(n_max=_log_int(rng, 1, 2500 if op == "append" else 8192 if op == "cast" else 16384))
        if op != "read":
            c.update(ctx_max=_log_int(rng, 1, 6000))
        if op == "append":
            c.update(pad=rng.choice([0, 0, 5]))
    c["empty"] = c["empty"] and c["seqs"] > 1
    while work(c)["bytes"] > _MOST_BYTES or _plain_bytes(c) > 10.0e9:
        if c["seqs"] > 2:
            c["seqs"] = (c["seqs"] + 1) // 2
        elif c["layers"] > 1:
            c["layers"] = (c["layers"] + 1) // 2
        else:
            c["n_max"] = (c["n_max"] + 1) // 2
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
    """Rows of each sequence that are written, read back or attended over."""
    n = _spread(c, "new", c["n_max"])
    if c["empty"]:
        n[0] = 0
    return n


def _before(c):
    """Slots that the sequences' caches held before."""
    return _spread(c, "before", c["ctx_max"]) if c["op"] in ("append", "cast") else [0] * c["seqs"]


def _lengths(c):
    return [a + b for a, b in zip(_before(c), _new(c))]


def _code_bytes(c):
    """Bytes of a head's row of codes, and of its scales."""
    return (c["head_dim"], 1) if c["fmt"] == "e4m3" else (c["head_dim"] // 2, c["head_dim"] // 32)


def _plain_bytes(c):
    """About the memory of the plain form's largest array."""
    rows = c["seqs"] * c["n_max"] * c["layers"] * c["kv_heads"]
    return 4.0 * rows * (c["head_dim"] + (c["group"] if c["op"] == "decode" else 0))


def work(c):
    H, D, L, B, T = c["kv_heads"], c["head_dim"], c["layers"], c["seqs"], sum(_new(c))
    codes, values = 2 * sum(_code_bytes(c)), 4 * D  # bytes of K and V of a head, held in few bits and in bf16
    if c["op"] == "decode":  # the cache and the queries read, outputs written
        Hq = H * c["group"]
        return {"bytes": float(T * L * H * codes + B * L * Hq * 6 * D + 12 * B), "flops": float(T * L * Hq * (4 * D + 8) + 1)}
    if c["op"] == "read":  # codes read, values written
        return {"bytes": float(T * L * H * (codes + values) + 4 * B), "flops": float(T * L * H * 2 * D)}
    # values read, codes written, what these stand for written
    return {"bytes": float(T * L * H * (2 * values + codes) + 12 * (T + B)), "flops": float(T * L * H * 8 * D)}


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _gen(seed, which):
    return torch.Generator(device=DEV).manual_seed(1000003 * (int(seed) % (1 << 40)) + which)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _rows(shape, gen):
    """N(0, 1) rows, each with a magnitude of its own (a factor of 1/4 to 4)."""
    x = _normal(shape, gen)
    return x.mul_(torch.rand(shape[:-1] + (1,), generator=gen, device=DEV).mul_(4).sub_(2).exp2_().bfloat16())


def _to(a, dtype):
    return torch.as_tensor(np.asarray(a), dtype=dtype).to(DEV)


def _tables(c, rng, counts):
    """A block table and the pool's size: a row of blocks for each sequence of `counts` slots; a few blocks stay unused."""
    need = [-(-n // c["block"]) for n in counts]
    perm, at = rng.permutation(sum(need) + 3), 0
    table = np.full((c["seqs"], max(need) + 1), -1, dtype=np.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return _to(table, torch.int32), sum(need) + 3


def _codes(c, lead, gen, filled):
    """(codes, scales) of rows [*lead, H]: zeros, or what rows of a model's context are held as."""
    H, D = c["kv_heads"], c["head_dim"]
    width, scales = _code_bytes(c)
    dtype = torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.uint8
    codes = torch.zeros((*lead, H, width), dtype=torch.uint8, device=DEV)
    scale = torch.full((*lead, H, scales), 127, dtype=torch.uint8, device=DEV)
    if filled:
        least = 118 if c["fmt"] == "e4m3" else 124  # so that values are about 1
        scale.copy_(torch.randint(least, least + 6, scale.shape, generator=gen, device=DEV, dtype=torch.uint8))
        edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV, dtype=torch.bfloat16)
        for i in range(lead[0]):  # a part at a time: the values take several times the codes' memory
            x = _normal((*lead[1:], H, D), gen)
            if c["fmt"] == "e4m3":
                codes[i] = x.mul_(130).clamp_(-448, 448).to(dtype).view(torch.uint8)
            else:
                x.mul_(1.9)
                q = torch.bucketize(x.abs(), edges, out_int32=True).to(torch.uint8) | (x < 0).to(torch.uint8) << 3
                codes[i] = q[..., 0::2] | q[..., 1::2] << 4
    return codes.view(dtype), scale


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
    H, D, L, B, lens = c["kv_heads"], c["head_dim"], c["layers"], c["seqs"], _lengths(case)
    s = dict(c=c, op=c["op"], count=_to(_new(c), torch.int32), before=_to(_before(c), torch.int32), len=_to(lens, torch.int32))
    s["table"] = None
    if c["cache"] == "contiguous":
        lead = (B, L, max(lens) + 8)
    else:
        s["table"], blocks = _tables(c, rng, lens)
        lead = (L, blocks, c["block"])
    held = c["op"] in ("read", "decode")  # the others write every row that they return
    (s["k"], s["k_scale"]), (s["v"], s["v_scale"]) = (_codes(c, lead, _gen(seed, w), held) for w in (1, 2))
    if c["op"] == "append":
        s["coords"] = _coords(c, rng)
        s["off"] = _to(np.concatenate([[0], np.cumsum(_new(c))]), torch.int32)
        s["k_new"], s["v_new"] = (_rows((L, sum(_new(c)) + c["pad"], H, D), _gen(seed, w)) for w in (3, 4))
    elif c["op"] == "cast":
        s["k_src"], s["v_src"] = (_rows((B, L, c["n_max"], H, D), _gen(seed, w)) for w in (3, 4))
    elif c["op"] == "decode":
        s["q"] = _normal((B, L, H * c["group"], D), _gen(seed, 3))
        s["q_pos"] = _to(np.asarray(lens) + rng.integers(0, 20000, B), torch.int64)
    return s


# ----------------------------------------------------------------------------
# the framework's calls
# ----------------------------------------------------------------------------
def _kept(s):
    """What a program makes once and keeps: descriptors, outputs, workspace."""
    import paper_2606_26631_gb300 as prcr
    c = s["c"]
    H, D, L, B = c["kv_heads"], c["head_dim"], c["layers"], c["seqs"]
    cfg = prcr.rope_cfg(L, H, D, _sections(c), THETA, prcr.LAYOUT_INTERLEAVED if c["layout"] == "interleaved" else prcr.LAYOUT_SECTIONED)
    if s["table"] is None:
        cache = prcr.qcache_contiguous(s["k"], s["v"], s["k_scale"], s["v_scale"])
    else:
        cache = prcr.qcache_paged(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"])
    h = dict(prcr=prcr, cfg=cfg, cache=cache, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if s["op"] == "decode":
        h["out"] = torch.empty(s["q"].shape, dtype=torch.float32, device=DEV)
        h["max_len"] = max(_lengths(c))
        nbytes = prcr.decode_quant_workspace_size(cfg, cache, B, L, H * c["group"], h["max_len"])
        h["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)
        return h
    h["k"], h["v"] = (torch.zeros((B, L, c["n_max"], H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    h["rows"] = prcr.cache_contiguous(h["k"], h["v"])
    h["zero"], h["len"] = torch.zeros_like(s["len"]), torch.zeros_like(s["len"])
    if s["op"] == "cast":
        h["src"] = prcr.cache_contiguous(s["k_src"], s["v_src"])
    return h


def _run_own(s):
    if "own" not in s:
        s["own"] = _kept(s)
    h, c = s["own"], s["c"]
    prcr = h["prcr"]
    if s["op"] == "decode":
        prcr.decode_attention_quant(h["cfg"], h["cache"], 0, s["q"], s["q_pos"], s["len"], h["max_len"], h["out"], h["status"], h["ws"])
        return {"out": h["out"]}
    out = {"k": h["k"], "v": h["v"]}
    if s["op"] == "append":
        prcr.append_kv_quant(h["cfg"], h["cache"], 0, s["k_new"], s["v_new"], s["coords"], s["off"], s["before"], h["len"], h["status"])
        out["len"] = h["len"]
    elif s["op"] == "cast":
        prcr.quantize_cache(h["cfg"], h["src"], 0, h["cache"], 0, c["layers"], h["zero"], s["before"], s["count"], c["n_max"], h["status"])
    prcr.dequantize_cache(h["cfg"], h["cache"], 0, h["rows"], 0, c["layers"], s["before"], h["zero"], s["count"], c["n_max"], h["status"])
    return out


# ----------------------------------------------------------------------------
# the plain form: elementary torch operations in 32 bits
# ----------------------------------------------------------------------------
def _rotate(x, pos, c):
    """x [..., n, heads, D] at pos [n, 3]: pairs (i, i + D/2), in 64 bits (what comes may lie next to a border)."""
    D, (st, sh, sw) = c["head_dim"], _sections(c)
    i = torch.arange(D // 2, device=x.device)
    if c["layout"] == "interleaved":
        axis = torch.where((i % 3 == 1) & (i < 3 * sh), 1, torch.where((i % 3 == 2) & (i < 3 * sw), 2, 0))
    else:
        axis = (i >= st).long() + (i >= st + sh).long()
    ang = pos.double()[:, axis] * THETA ** (-2.0 * i.double() / D)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x.double().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _rounded(x, c):
    """What rows x [..., D] are held as, in bf16."""
    shape, dims = x.shape, -1
    if c["fmt"] == "e4m3":
        top, lowest, bits, wide, narrow = 0.875, -6, 3, 9, 8  # 448 = 0.875 * 2^9; subnormals below 2^-6; 3 bits behind the first
    else:
        top, lowest, bits, wide, narrow = 0.75, 0, 1, 3, 2
        x, dims = x.reshape(*shape[:-1], 8, -1, 4), (-3, -1)
    frac, exp = torch.frexp(x.abs().amax(dims, keepdim=True))
    e = torch.where(frac <= top, exp - wide, exp - narrow).clamp(min=LEAST)
    y = torch.ldexp(x, -e)
    step = (torch.frexp(y).exponent - 1).clamp(min=lowest) - bits  # the format's steps at y are 2^step
    return torch.ldexp(torch.ldexp(y, -step).round(), step + e).bfloat16().reshape(shape)


def _values(c, codes, scale):
    """What codes [..., bytes] with scales [..., n] stand for, in 32 bits."""
    if c["fmt"] == "e4m3":
        return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), scale.int() - 127)
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    m, s = q & 7, 1.0 - 2.0 * (q >> 3)
    x = s * torch.where(m < 2, m * 0.5, torch.ldexp(1.0 + 0.5 * (m & 1), (m >> 1) - 1))
    return torch.ldexp(x.unflatten(-1, (8, -1, 4)), scale.int()[..., None, :, None] - 127).flatten(-3)


def _slots(s, b, slot, layers):
    """Places, as rows of [rows, H, bytes], of slots `slot` [n] of sequences `b` [n] at every layer: [L, n]."""
    c, layer = s["c"], torch.arange(layers, device=DEV).view(-1, 1)
    shape = s["k"].shape
    if s["table"] is None:
        return (b * shape[1] + layer) * shape[2] + slot
    return (layer * shape[1] + s["table"].long()[b, slot // c["block"]]) * c["block"] + slot % c["block"]


def _each_row(s):
    """The sequence and the place among its rows of each written or read row, in order."""
    n = s["count"].long()
    b = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n)
    return b, torch.arange(b.numel(), device=DEV) - (n.cumsum(0) - n)[b]


def _laid_out(s, rows):
    """Rows [L, n, H, D] as [B, L, n_max, H, D], zeros behind each sequence's."""
    c = s["c"]
    b, i = _each_row(s)
    out = torch.zeros((c["seqs"], c["layers"], c["n_max"], c["kv_heads"], c["head_dim"]), dtype=torch.bfloat16, device=DEV)
    out[b, :, i] = rows.transpose(0, 1)
    return out


def _gathered(s, which, rows):
    """What the cache's rows `rows` stand for, in 32 bits: [*rows.shape, H, D]."""
    codes, scale = s[which].view(torch.uint8), s[which + "_scale"]
    return _values(s["c"], codes.view(-1, *codes.shape[-2:])[rows], scale.view(-1, *scale.shape[-2:])[rows])


def _plain_append(s):
    c, T = s["c"], sum(_new(s["c"]))
    return {"k": _laid_out(s, _rounded(_rotate(s["k_new"][:, :T], s["coords"][:T], c), c)),
            "v": _laid_out(s, _rounded(s["v_new"][:, :T].float(), c)), "len": s["before"] + s["count"]}


def _plain_cast(s):
    b, i = _each_row(s)
    return {x: _laid_out(s, _rounded(s[x + "_src"][b, :, i].transpose(0, 1).float(), s["c"])) for x in "kv"}


def _plain_read(s):
    b, i = _each_row(s)
    rows = _slots(s, b, i, s["c"]["layers"])
    return {x: _laid_out(s, _gathered(s, x, rows).bfloat16()) for x in "kv"}


def _plain_decode(s):
    c = s["c"]
    B, L, H, g, D, S = c["seqs"], c["layers"], c["kv_heads"], c["group"], c["head_dim"], max(_lengths(c))
    b = torch.arange(B, device=DEV).repeat_interleave(S)
    slot = torch.arange(S, device=DEV).repeat(B)
    slot = torch.where(slot < s["len"].long()[b], slot, 0)
    if s["table"] is not None:  # (a sequence without any slot: its table is empty)
        b = torch.where(s["len"].long()[b] > 0, b, B - 1)
    rows = _slots(s, b, slot, L).view(L, B, S)
    k, v = (_gathered(s, x, rows).permute(1, 0, 3, 2, 4) for x in "kv")  # [B, L, H, S, D]
    q = _rotate(s["q"].transpose(0, 1), s["q_pos"].view(B, 1).expand(B, 3), c).float().transpose(0, 1).reshape(B, L, H, g, D)
    x = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    seen = torch.arange(S, device=DEV) < s["len"].view(B, 1, 1, 1, 1)
    x = torch.where(seen, (x - torch.where(seen, x, -math.inf).amax(-1, keepdim=True)).exp(), 0.0)
    out = (x @ v) / x.sum(-1, keepdim=True)
    return {"out": torch.where(s["len"].view(B, 1, 1, 1, 1) > 0, out, 0.0).view(B, L, H * g, D)}


_PLAIN = {"append": _plain_append, "cast": _plain_cast, "read": _plain_read, "decode": _plain_decode}


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


def _format(c):
    """Every magnitude of the format, ascending (64 bits): the code's place in the list is the code without its sign."""
    if c["fmt"] == "e4m3":
        m = [(f / 8) * 2.0 ** -6 if not e else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)][:-1]
    else:
        m = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(m, dtype=torch.float64, device=DEV)


def _nearest(x, c):
    """x [..., D] (64 bits) by search among the format's values: the nearer neighbour, the even code of two as near."""
    values, shape = _format(c), x.shape
    apart = c["fmt"] == "e2m1"
    y = x.reshape(-1, 8, shape[-1] // 32, 4).transpose(1, 2).reshape(-1, 32) if apart else x.reshape(-1, shape[-1])
    out = torch.empty(y.shape, dtype=torch.bfloat16, device=DEV)
    for at in range(0, y.shape[0], 1 << 17):  # some rows at a time: the search takes several times their memory
        z = y[at:at + (1 << 17)]
        need = z.abs().amax(-1, keepdim=True) / values[-1]
        scale = torch.exp2(torch.ceil(torch.log2(need.clamp(min=2.0 ** LEAST))))
        scale = torch.where(scale < need, scale * 2, torch.where((scale / 2 >= need) & (scale > 2.0 ** LEAST), scale / 2, scale))
        w = z.abs() / scale
        hi = torch.searchsorted(values, w).clamp(max=values.numel() - 1)
        lo = (hi - 1).clamp(min=0)
        up, down = values[hi] - w, w - values[lo]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        out[at:at + (1 << 17)] = (torch.sign(z) * values[pick] * scale).bfloat16()
    return (out.view(-1, shape[-1] // 32, 8, 4).transpose(1, 2) if apart else out).reshape(shape)


def _stands_for(c, codes, scale):
    """What rows of codes stand for (64 bits), by the format's list of values."""
    values = _format(c)
    if c["fmt"] == "e4m3":
        values = torch.cat([values, values.new_tensor([math.nan])])
        q, at = codes.view(torch.uint8).long(), torch.zeros(c["head_dim"], dtype=torch.long, device=DEV)
        x = torch.where(q >= 128, -1.0, 1.0) * values[q % 128]
    else:
        q, at = codes.long(), torch.arange(c["head_dim"], device=DEV) // 4 % (c["head_dim"] // 32)
        q = torch.stack([q % 16, q // 16], -1).flatten(-2)
        x = torch.where(q >= 8, -1.0, 1.0) * values[q % 8]
    return x * torch.exp2(scale.double() - 127)[..., at]


def _held(c, s, which, b, layer, n):
    """Slots 0 .. n - 1 of sequence b at `layer`: [n, H, D] in 64 bits."""
    codes, scale = s[which].view(torch.uint8), s[which + "_scale"]
    if s["table"] is None:
        return _stands_for(c, codes[b, layer, :n], scale[b, layer, :n])
    blocks = s["table"][b, : -(-n // c["block"])].long()
    return _stands_for(c, codes[layer][blocks].flatten(0, 1)[:n], scale[layer][blocks].flatten(0, 1)[:n])


def exact(case, seed):
    s, c = prepare(case, seed), case
    H, g, D, L, B = c["kv_heads"], c["group"], c["head_dim"], c["layers"], c["seqs"]
    if c["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        for b, n in enumerate(_lengths(c)):
            for l in range(L if n else 0):
                K, V = (_held(c, s, x, b, l, n) for x in "kv")
                q = _turned(s["q"][b, l].double(), s["q_pos"][b].expand(1, 3), c).view(H, g, D)
                p = torch.softmax(torch.einsum("hgd,shd->hgs", q, K) / D ** 0.5, -1)
                out[b, l] = torch.einsum("hgs,shd->hgd", p, V).reshape(H * g, D)
        return {"out": out}
    k, v = (torch.zeros((B, L, c["n_max"], H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    at = 0
    for b, n in enumerate(_new(c)):
        for l in range(L if n else 0):
            if c["op"] == "append":
                k[b, l, :n] = _nearest(_turned(s["k_new"][l, at:at + n].double(), s["coords"][at:at + n].unsqueeze(1), c), c)
                v[b, l, :n] = _nearest(s["v_new"][l, at:at + n].double(), c)
            elif c["op"] == "cast":
                k[b, l, :n], v[b, l, :n] = (_nearest(s[x][b, l, :n].double(), c) for x in ("k_src", "v_src"))
            else:
                k[b, l, :n], v[b, l, :n] = (_held(c, s, x, b, l, n).bfloat16() for x in "kv")
        at += n
    out = {"k": k, "v": v}
    if c["op"] == "append":
        out["len"] = _to(_lengths(c), torch.int32)
    return out

"""Caches, packed batches and 64-bit references for the tests of append_kv,
chunk_attention, accumulate_weights and evict.

A Cache holds the device tensors of a decoder cache and says where a slot's row
lies; its rows are compared on the host in float64.
"""
import numpy as np
import torch

import paper_2606_26631_gb300 as prcr
from oracle import prcr_oracle as O

DEV = "cuda:0"
CANARY = 12345.0  # exact in bf16: 12352 is its neighbour, so it is written and read as 12352


def sections(D):
    t = D // 8
    h = (D // 2 - t) // 2
    return (t, h, D // 2 - t - h)


def cfg_of(L, H, D, layout=prcr.LAYOUT_SECTIONED):
    return prcr.rope_cfg(L, H, D, sections(D), 1e6, layout)


def f64(t):
    return O.bf16_bits_to_f64(t.contiguous().view(torch.int16).cpu().numpy())


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def normal(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


class Cache:
    """k, v of a cache for `caps[b]` slots a sequence; block 0: contiguous. `gap` elements more
    between slots. Rows are N(0, 1), or `fill` everywhere."""

    def __init__(self, L, H, D, caps, block, seed=0, fill=None, gap=0, unmapped=()):
        self.L, self.H, self.D, self.block, self.caps = L, H, D, block, list(caps)
        B, row = len(caps), H * D
        if block == 0:
            shape = (B, L, max(caps), row + gap)
            self.table = None
        else:
            need = [-(-c // block) for c in caps]
            rng = np.random.default_rng(seed + 5)
            perm = rng.permutation(sum(need) + 2)
            table = np.full((B, max(need)), -1, dtype=np.int32)
            at = 0
            for b, n in enumerate(need):
                table[b, :n] = perm[at:at + n]
                at += n
            for b, j in unmapped:
                table[b, j] = -1
            self.np_table, self.table = table, torch.from_numpy(table).to(DEV)
            shape = (L, sum(need) + 2, block, row + gap)
        make = (lambda s: normal(shape, s)) if fill is None else (lambda s: torch.full(shape, fill, dtype=torch.bfloat16, device=DEV))
        self.k_all, self.v_all = make(seed + 1), make(seed + 2)
        self.k, self.v = (x[..., :row].unflatten(-1, (H, D)) for x in (self.k_all, self.v_all))

    def desc(self):
        return prcr.cache_contiguous(self.k, self.v) if self.table is None else prcr.cache_paged(self.k, self.v, self.table)

    def where(self, b, slots):
        """Index of the [L, len(slots), H, D] rows of sequence b."""
        s = torch.as_tensor(slots, device=DEV).long()
        if self.table is None:
            return (b, slice(None), s)
        return (slice(None), torch.from_numpy(self.np_table).to(DEV)[b][s // self.block].long(), s % self.block)

    def rows(self, x, b, n):
        """Slots 0 .. n - 1 of sequence b of the tensor x (k or v), [L, n, H, D] on the device."""
        return x[self.where(b, np.arange(n))]


def offsets(lens):
    return i32(np.concatenate([[0], np.cumsum(lens)]))


def rope64(x, pos, D, layout=prcr.LAYOUT_SECTIONED):
    """x [..., n, heads, D] at pos [n, 3] (the oracle's angles), 64 bits."""
    ang = O.angles(np.asarray(pos, dtype=np.float64), D, sections(D), 1e6, layout)[:, None, :]
    c, s, a, b = np.cos(ang), np.sin(ang), x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def softmax64(x):
    m = x.max(-1, keepdims=True)
    w = np.exp(x - m)
    return w / w.sum(-1, keepdims=True)


def chunk64(q, pos, K, V, sees, layout=prcr.LAYOUT_SECTIONED):
    """out [n, Hq, D] and a bound on its error: q [n, Hq, D], K / V [S, H, D], sees [n, S] bool.

    The bound counts the kernel's roundings, each by at most half a bf16 step (2^-8 of the value): of the
    rotated query (which moves a logit by at most e = 2^-8 sum |q k| / sqrt(D), and so a weight by a factor within
    exp(+-2 e)), of the probabilities (2^-8 of sum w |v|), of the output; float32 sums add under 1e-4 of that."""
    n, Hq, D = q.shape
    H = K.shape[1]
    g = Hq // H
    qr = rope64(q, pos, D, layout)
    out, bound = np.zeros_like(qr), np.zeros_like(qr)
    for h in range(Hq):
        k, v = K[:, h // g], V[:, h // g]
        x = qr[:, h] @ k.T / np.sqrt(D)
        e = 2.0 ** -8 * (np.abs(qr[:, h]) @ np.abs(k).T) / np.sqrt(D)
        for i in range(n):
            s = sees[i]
            if not s.any():
                continue
            w = softmax64(x[i, s])
            out[i, h] = w @ v[s]
            mean = w @ np.abs(v[s])
            bound[i, h] = 2.0 ** -8 * np.abs(out[i, h]) + (2.0 ** -8 + np.expm1(2 * e[i, s].max())) * mean * 1.001 + 1e-30
    return out, bound


def causal(n, length, S):
    """[n, S]: query i of the last n of `length` slots sees slots up to its own."""
    return np.arange(S)[None, :] <= (length - n + np.arange(n))[:, None]


def score_order(score, lo, hi, count):
    """The `count` slots of [lo, hi) of the highest score, equal ones by index, NaN last."""
    x = np.where(np.isnan(score[lo:hi]), -np.inf, score[lo:hi].astype(np.float64))
    nan = np.isnan(score[lo:hi])
    order = sorted(range(hi - lo), key=lambda i: (nan[i], -x[i], i))
    return [lo + i for i in order[:count]]


def evict64(score, n, budget, sink, recent):
    if n <= budget:
        return list(range(n))
    mid = score_order(score, sink, n - recent, budget - sink - recent)
    return sorted(list(range(sink)) + mid + list(range(n - recent, n)))


def chunk64_exact(q, K, V, sees):
    """out [n, Hq, D] and a bound on its error as chunk64 gives them, for queries at position 0: these are not rotated, so the
    kernel's bf16 ones are exact, and large logits do not blur the bound.

    A float32 dot of D products is off by at most e = D 2^-23 sum |q k| / sqrt(D) (its D additions by 2^-23 of a partial sum
    each), whatever their order. That moves a weight w by a factor within exp(+-2 e), and so 1 - w, the others' sum: by at most
    expm1(2 e) min(w, 1 - w). The probabilities and the output are rounded by 2^-8."""
    n, Hq, D = q.shape
    g = Hq // K.shape[1]
    out, bound = np.zeros_like(q), np.zeros_like(q)
    for h in range(Hq):
        k, v = K[:, h // g], V[:, h // g]
        x = q[:, h] @ k.T / np.sqrt(D)
        e = D * 2.0 ** -23 * (np.abs(q[:, h]) @ np.abs(k).T) / np.sqrt(D)
        for i in range(n):
            s = sees[i]
            if not s.any():
                continue
            w = softmax64(x[i, s])
            out[i, h] = w @ v[s]
            off = 2.0 ** -8 * w + np.expm1(2 * e[i, s].max()) * np.minimum(w, 1 - w)
            bound[i, h] = (2.0 ** -8 * np.abs(out[i, h]) + off @ np.abs(v[s])) * 1.001 + 1e-30
    return out, bound


EXACT_NORM = 3.5e-3  # two roundings, of 1.6e-3 in the mean square each, make 2.3e-3 of the 2-norm; half as much again


def assert_close(got, ref, bound):
    """Every element within its bound, and the whole within EXACT_NORM of the 2-norm."""
    d = np.abs(got - ref)
    assert (d <= bound).all(), (np.unravel_index((d - bound).argmax(), d.shape), (d / bound).max())
    norm = np.sqrt((ref ** 2).sum())
    assert np.sqrt((d ** 2).sum()) <= EXACT_NORM * norm, np.sqrt((d ** 2).sum()) / norm

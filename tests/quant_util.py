"""Quantised caches and 64-bit references for the tests of append_kv_quant, quantize_cache,
dequantize_cache and decode_attention_quant.

The formats are written out here as lists of their values, and a value is rounded by search among
them; nothing here uses the library's conversions.
"""
import numpy as np
import torch

import cache_ops_util as U
import paper_2606_26631_gb300 as prcr
from cache_ops_util import DEV, i32

E4M3 = np.array([f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)][:-1])
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = {"e4m3": E4M3, "e2m1": E2M1}
LEAST = 10  # the least byte of a scale that is written
NAN = 255


def groups(fmt, D):
    """The group of each dim."""
    return np.zeros(D, dtype=int) if fmt == "e4m3" else np.arange(D) // 4 % (D // 32)


def n_scales(fmt, D):
    return 1 if fmt == "e4m3" else D // 32


def width(fmt, D):
    return D if fmt == "e4m3" else D // 2


def scale64(byte):
    s = np.exp2(np.asarray(byte, dtype=np.float64) - 127)
    return np.where(np.asarray(byte) == NAN, np.nan, s)


def scale_of(fmt, amax):
    """The scale's byte of a largest magnitude (64 bits): by trying them all."""
    bytes_ = np.arange(LEAST, 255)
    enough = VALUES[fmt][-1] * scale64(bytes_) >= np.asarray(amax)[..., None]
    return np.where(np.isfinite(amax), LEAST + np.argmax(enough, -1), NAN)


def nearest(fmt, x, byte):
    """The place in VALUES of |x| in units of the scale (64 bits): ties to the even one, never one that stands for 2^128."""
    v = VALUES[fmt]
    y = np.abs(x) / scale64(byte)
    hi = np.clip(np.searchsorted(v, y), 1, len(v) - 1)
    up, down = v[hi] - y, y - v[hi - 1]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return np.where(v[pick] * scale64(byte) >= 2.0 ** 128, pick - 1, pick)


def quantize(fmt, x):
    """(codes [..., D], one per dim, bytes of scales [..., n]) of x [..., D] (64 bits, which hold bf16 exactly)."""
    D = x.shape[-1]
    g = groups(fmt, D)
    amax = np.stack([np.abs(x[..., g == j]).max(-1) for j in range(n_scales(fmt, D))], -1)
    with np.errstate(invalid="ignore"):
        amax = np.where(np.stack([np.isnan(x[..., g == j]).any(-1) for j in range(n_scales(fmt, D))], -1), np.nan, amax)
    byte = scale_of(fmt, amax)
    b = byte[..., g]
    nan = b == NAN
    safe, bs = np.where(nan, 0.0, np.where(np.isfinite(x), x, 0.0)), np.where(nan, 127, b)
    sign = np.signbit(safe) & ~nan
    codes = nearest(fmt, safe, bs) | np.where(sign, 128 if fmt == "e4m3" else 8, 0)
    return codes.astype(np.uint8), byte.astype(np.uint8)


def stand_for(fmt, codes, byte):
    """What codes [..., D] with scales [..., n] stand for (64 bits)."""
    D = codes.shape[-1]
    if fmt == "e4m3":
        v = np.concatenate([E4M3, [np.nan]])
        x = np.where(codes >= 128, -1.0, 1.0) * v[codes & 127]
    else:
        x = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes & 7]
    return x * scale64(byte)[..., groups(fmt, D)]


def pack(fmt, codes):
    """Codes, one per dim, as the cache holds them."""
    return codes if fmt == "e4m3" else (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(fmt, held):
    """The inverse of pack."""
    return held if fmt == "e4m3" else np.stack([held & 15, held >> 4], -1).reshape(*held.shape[:-1], 2 * held.shape[-1])


class QCache:
    """Codes and scales of a quantised cache for `caps[b]` slots a sequence; block 0: contiguous. `gap` codes' rows have
    16 * gap bytes more between slots, scales' 8 * gap. Random codes and scales of about 2^-6 (finite values of about 1), or `fill`."""

    def __init__(self, fmt, L, H, D, caps, block, seed=0, fill=None, gap=0, unmapped=()):
        self.fmt, self.L, self.H, self.D, self.block, self.caps = fmt, L, H, D, block, list(caps)
        self.W, self.n = width(fmt, D), n_scales(fmt, D)
        B = len(caps)
        if block == 0:
            lead, self.table = (B, L, max(caps)), None
        else:
            need = [-(-c // block) for c in caps]
            rng = np.random.default_rng(seed + 5)
            perm = rng.permutation(sum(need) + 2)
            table = np.full((B, max(max(need), 1)), -1, dtype=np.int32)
            at = 0
            for b, n in enumerate(need):
                table[b, :n] = perm[at:at + n]
                at += n
            for b, j in unmapped:
                table[b, j] = -1
            self.np_table, self.table = table, torch.from_numpy(table).to(DEV)
            lead = (L, sum(need) + 2, block)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)

        def codes():
            x = torch.randint(0, 256, lead + (H * self.W + 16 * gap,), generator=g, device=DEV, dtype=torch.uint8)
            if fmt == "e4m3":  # finite, below 2^6: exponents 0 .. 12
                x = (x & 0x80) | ((x & 0x7f) % 104)
            return x

        def scales():
            low, high = (118, 122) if fmt == "e4m3" else (124, 129)
            return torch.randint(low, high, lead + (H * self.n + 8 * gap,), generator=g, device=DEV, dtype=torch.uint8)

        if fill is None:
            self.k_all, self.v_all, self.ks_all, self.vs_all = codes(), codes(), scales(), scales()
        else:
            self.k_all, self.v_all = (torch.full(lead + (H * self.W + 16 * gap,), fill, dtype=torch.uint8, device=DEV) for _ in range(2))
            self.ks_all, self.vs_all = (torch.full(lead + (H * self.n + 8 * gap,), fill, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.k, self.v = (x[..., :H * self.W].unflatten(-1, (H, self.W)) for x in (self.k_all, self.v_all))
        self.ks, self.vs = (x[..., :H * self.n].unflatten(-1, (H, self.n)) for x in (self.ks_all, self.vs_all))

    def all(self):
        return self.k_all, self.v_all, self.ks_all, self.vs_all

    def desc(self):
        k, v = (x.view(torch.float8_e4m3fn) if self.fmt == "e4m3" else x for x in (self.k, self.v))
        if self.table is None:
            return prcr.qcache_contiguous(k, v, self.ks, self.vs)
        return prcr.qcache_paged(k, v, self.ks, self.vs, self.table)

    where = U.Cache.where

    def held(self, which, b, slots):
        """(codes one per dim [L, n, H, D], bytes of scales [L, n, H, n_scales]) of those slots, on the host."""
        x, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        w = self.where(b, slots)
        return unpack(self.fmt, x[w].cpu().numpy()), s[w].cpu().numpy()

    def values(self, which, b, n):
        """What slots 0 .. n - 1 stand for, [L, n, H, D] (64 bits)."""
        return stand_for(self.fmt, *self.held(which, b, np.arange(n)))


def decode64(q, pos, K, V, layout=prcr.LAYOUT_SECTIONED):
    """out [Hq, D] of one sequence and layer, and a bound on the kernel's error: q [Hq, D], K / V [S, H, D].

    The bound counts, each by the most that it can be: the query's rotation in float32 with float32 cos/sin of an angle exact to
    2^-24 of half a turn (2^-21 of the pair), its two fp16 pieces (2^-21 of it, and 2^-36 of the head's largest), and the
    float32 sums of a logit (D additions of 2^-23 each, which may truncate): a logit is off by at most
    e = ((D + 16) 2^-23 sum |q||k| + 2^-36 max |q| sum |k|) / sqrt(D) with |q| the pair's norm; the logit in units of log 2 and its difference from the reference
    are rounded too (2^-22 of |x| and of the largest |x|). All of that moves a weight by a factor within exp(+-2 e). The weights' exponentials are
    off by 2^-21, their two pieces by 2^-21 and by 2^-35 of the largest product weight, sums over S slots and 64 parts by (S + 64) 2^-23."""
    Hq, D = q.shape
    S, H, _ = K.shape
    g = Hq // H
    qr = U.rope64(q[None], np.array([[pos] * 3]), D, layout)[0]
    norm = np.sqrt(q[:, :D // 2] ** 2 + q[:, D // 2:] ** 2)
    norm = np.concatenate([norm, norm], -1)
    out, bound = np.zeros((Hq, D)), np.zeros((Hq, D))
    if S == 0:
        return out, bound + 1e-37
    for h in range(Hq):
        k, v = K[:, h // g], V[:, h // g]
        x = k @ qr[h] / np.sqrt(D)
        e = ((D + 16) * 2.0 ** -23 * (np.abs(k) @ norm[h]) + 2.0 ** -36 * norm[h].max() * np.abs(k).sum(-1)) / np.sqrt(D)
        e = e.max() + 2.0 ** -21 * np.abs(x).max()
        w = U.softmax64(x)
        out[h] = w @ v
        mean = w @ np.abs(v)
        most = (w * np.abs(v).max(-1)).max()
        bound[h] = (np.expm1(2 * e) + (S + 80) * 2.0 ** -23) * mean * 1.001 + S * 2.0 ** -34 * most + 1e-37
    return out, bound


def run_decode(cfg, cache, layer0, q, pos, lens, max_len, out=None, ws=None, stream=None, status=None):
    """(out, status) of a call with a workspace of what the library asks for, filled with NaN."""
    B, L, Hq, D = q.shape
    d = cache.desc()
    out = torch.full((B, L, Hq, D), float("nan"), device=DEV) if out is None else out
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    if ws is None:
        ws = torch.full((max(16, prcr.decode_quant_workspace_size(cfg, d, B, L, Hq, max_len)),), 0xff, dtype=torch.uint8, device=DEV)
    prcr.decode_attention_quant(cfg, d, layer0, q, torch.as_tensor(np.asarray(pos), dtype=torch.int64).to(DEV), i32(lens), max_len, out, status,
                                ws, stream=stream)
    return out, status

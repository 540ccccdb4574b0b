"""Numbers at which the quantised cache's operators can go wrong: keys whose rotation cancels next to a border between two codes,
groups of a value's dims that lie far below its others, logits and codes that are not finite, the longest sequences."""
import numpy as np
import pytest
import torch

import cache_ops_util as U
import paper_2606_26631_gb300 as prcr
import quant_util as Q
from cache_ops_util import DEV, i32, normal

pytestmark = pytest.mark.gpu


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


# (pair, position, first, second): pairs of head_dim 128 at theta 1e6 of which one rotated value is some 2^-9 to 2^-17 of the pair's norm and
# 2^-26 to 2^-21 units of an E4M3 scale from a border between two codes, on the side that sin and cos off by 2^-29 miss.
NEAR_BORDERS = [
    (12, 9876, 1.6328125, 1.75), (20, 16313, 1.984375, -1.9140625), (5, 39792, 1.828125, -1.65625), (4, 2483, 1.90625, -2.515625),
    (24, 25524, 1.296875, 1.9375), (11, 8954, 1.2578125, -1.0859375), (6, 2567, 1.140625, 1.09375), (7, 33160, 1.140625, -1.0859375),
    (16, 24466, 1.0546875, -1.203125), (29, 32521, 1.890625, 1.546875), (13, 11293, 1.96875, -1.6796875), (14, 27886, 1.8515625, -1.8671875),
    (19, 23496, 1.1171875, 1.0234375), (21, 36628, 1.71875, -2.203125), (2, 23668, 1.09375, -1.359375), (22, 25664, 1.578125, 1.6640625),
    (17, 29559, 1.0625, 0.953125), (8, 16284, 1.859375, 1.90625), (31, 34701, 1.9609375, 2.578125), (0, 39877, 1.1484375, -1.1015625),
    (0, 6416, 1.0234375, 0.8671875), (1, 21825, 1.1796875, -1.3984375), (1, 21825, 1.3984375, 1.1796875), (11, 38900, 1.0390625, 0.98828125)]


def append_keys(fmt, k, pos):
    """(codes [n, H, D], scales' bytes) of keys k [n, H, D] appended at (p, p, p)."""
    n, H, D = k.shape
    cache = Q.QCache(fmt, 1, H, D, [n], 0, fill=0x5a)
    out, st = i32([0]), status_word()
    prcr.append_kv_quant(U.cfg_of(1, H, D), cache.desc(), 0, k[None].contiguous(), torch.zeros_like(k)[None], i32(np.stack([pos] * 3, 1)), i32([0, n]),
                         i32([0]), out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and out.tolist() == [n]
    codes, byte = cache.held("k", 0, np.arange(n))
    return codes[0], byte[0]


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_append_next_to_borders(fmt):
    """The code nearest to the exact rotation, however far a pair cancels. (The 64-bit rotation is off by 2^-38 of the pair's norm at these positions,
    2^-28 units; the nearest of these values lies 2^-26 from its border.)"""
    D, H = 128, 4
    pos = np.array([c[1] for c in NEAR_BORDERS])
    k = np.zeros((len(pos), H, D))
    for t, (i, _, x, y) in enumerate(NEAR_BORDERS):
        for h, e in enumerate((0, -30, 60, 127)):  # (at 2^127: those that stay below 2^128; their scale is the highest)
            top = np.hypot(x, y) * 2.0 ** e
            k[t, h, i], k[t, h, i + D // 2] = (x * 2.0 ** e, y * 2.0 ** e) if top < 3.38e38 else (0.0, 0.0)
    assert np.count_nonzero(k[:, 3]) > 0
    k = torch.from_numpy(k).float().bfloat16().to(DEV)
    codes, byte = append_keys(fmt, k, pos)
    ref = Q.quantize(fmt, U.rope64(U.f64(k), np.stack([pos] * 3, 1), D))
    assert np.array_equal(byte, ref[1])
    mag = 127 if fmt == "e4m3" else 7
    assert np.array_equal(codes & mag, ref[0] & mag)
    assert np.array_equal((codes > mag) & (codes & mag > 0), (ref[0] > mag) & (ref[0] & mag > 0))


@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("e4m3", 80), ("e2m1", 64)])
def test_append_of_pairs_that_cancel(fmt, D):
    """Rows all of whose pairs cancel to 2^-7 of their norm and less in one value or the other. (Values that the 64-bit rotation, off by 2^-38 of the
    norm, cannot place on a side of a border, and groups whose scale it cannot, are left out.)"""
    n, H, P = 600, 4, D // 2
    rng = np.random.default_rng(D)
    pos = rng.integers(1, 40000, n)
    ang = U.O.angles(np.stack([pos] * 3, 1).astype(np.float64), D, U.sections(D), 1e6, prcr.LAYOUT_SECTIONED)[:, None, :]
    c, s = np.cos(ang), np.sin(ang)
    p = rng.integers(128, 256, (n, H, P)) / 128.0 * rng.choice([-1, 1], (n, H, P))
    which = rng.random((n, H, P)) < 0.5
    with np.errstate(divide="ignore"):
        q = np.clip(np.where(which, p * c / s, -p * s / c), -4, 4)
    k = torch.from_numpy(np.concatenate([p, q], -1)).float().bfloat16().to(DEV)
    codes, byte = append_keys(fmt, k, pos)
    x = U.f64(k)
    exact = U.rope64(x, np.stack([pos] * 3, 1), D)
    pair = np.hypot(x[..., :P], x[..., P:])
    e = 2.0 ** -36 * np.concatenate([pair, pair], -1)
    low, high = (Q.quantize(fmt, np.abs(exact) + z * e) for z in (-1, 1))
    sure = low[1] == high[1]
    assert sure.mean() > 0.99 and np.array_equal(byte[sure], low[1][sure])
    ok = sure[..., Q.groups(fmt, D)] & (low[0] == high[0])
    mag = 127 if fmt == "e4m3" else 7
    assert ok.mean() > 0.99 and np.array_equal((codes & mag)[ok], low[0][ok] & mag)


@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("e4m3", 48), ("e2m1", 128), ("e2m1", 64)])
def test_append_at_position_zero(fmt, D):
    """Pairs whose axis is at 0 (an image's first row, column or frame) are not turned: their keys are rounded as they are, ties among them."""
    n, H, L = 48, 3, 2
    rng = np.random.default_rng(D)
    pos = rng.integers(1, 3000, (n, 3)) * rng.integers(0, 2, (n, 3))
    pos[:6] = [[0, 0, 0], [0, 5, 9], [7, 0, 0], [0, 0, 1], [0, 1, 0], [1, 0, 0]]
    v = Q.VALUES[fmt]
    edges = np.concatenate([v, (v[1:] + v[:-1]) / 2])
    x = rng.choice(edges, (L, n, H, D)) * rng.choice([-1, 1], (L, n, H, D)) * 2.0 ** rng.integers(-30, 30, (L, n, H, 1))
    k = torch.from_numpy(x).float().bfloat16().to(DEV)
    cache = Q.QCache(fmt, L, H, D, [n], 16, fill=0x5a)
    out, st = i32([0]), status_word()
    prcr.append_kv_quant(U.cfg_of(L, H, D), cache.desc(), 0, k, k, i32(pos), i32([0, n]), i32([0]), out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    codes, byte = cache.held("k", 0, np.arange(n))
    x = U.f64(k)
    ref = Q.quantize(fmt, U.rope64(x, pos, D))
    assert np.array_equal(byte, ref[1])
    axis = np.repeat([0, 1, 2], U.sections(D))
    still = np.tile(pos[:, axis] == 0, (1, 2))[None, :, None]
    assert np.array_equal(codes[np.broadcast_to(still, codes.shape)], ref[0][np.broadcast_to(still, codes.shape)])
    mag = 127 if fmt == "e4m3" else 7
    assert np.array_equal(codes & mag, ref[0] & mag)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_append_at_position_zero_takes_no_longer(fmt):
    """Keys that are not turned lie on borders between codes in great numbers; computing them again in float64 took 20 to 50 times as long."""
    L, H, D, n = 8, 4, 128, 8192
    cache, k = Q.QCache(fmt, L, H, D, [n], 16, fill=0), normal((L, n, H, D), 1)
    c, d, off, len_in, len_out, st = U.cfg_of(L, H, D), cache.desc(), i32([0, n]), i32([0]), i32([0]), status_word()
    took = []
    for pos in (i32(np.random.default_rng(1).integers(5000, 40000, (n, 3))), i32(np.zeros((n, 3)))):
        ms = []
        for _ in range(8):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            prcr.append_kv_quant(c, d, 0, k, k, pos, off, len_in, len_out, st)
            b.record()
            torch.cuda.synchronize()
            ms.append(a.elapsed_time(b))
        took.append(min(ms))
    assert took[1] < 6 * took[0], took


# ----------------------------------------------------------------------------
# one new token: values' groups far apart
# ----------------------------------------------------------------------------
def decode_by_group(q, pos, K, V, byte):
    """decode64's result and a bound that holds for each group of dims by itself: what fp16 loses of a slot's product weight, 2^-25 for each of its two
    pieces' products and of itself, is 3 2^-29 of a group's largest one at most (groups lie less than 2^8 below their row's largest, or are
    worked on apart; the largest of a row is 2^11 at least), of each of S slots, times a code's 6: S 2^-27 of the largest."""
    Hq, D = q.shape
    S, H, _ = K.shape
    G, norm = Q.groups("e2m1", D), U.rope64(q[None], np.array([[pos] * 3]), D)[0]
    out, bar = np.zeros((Hq, D)), np.zeros((Hq, D))
    for j in range(D // 32):
        ref, b = Q.decode64(q, pos, K, np.where(G == j, V, 0.0))
        for h in range(Hq):
            w = U.softmax64(K[:, h // (Hq // H)] @ norm[h] / np.sqrt(D))
            b[h] += S * 2.0 ** -27 * 6 * (w * Q.scale64(byte[:, h // (Hq // H), j])).max()
        out[:, G == j], bar[:, G == j] = ref[:, G == j], b[:, G == j]
    return out, bar


def spread_scales(kind, shape, rng):
    """Bytes of values' scales, [..., groups of a row]: groups far apart in every slot, in any slot by chance, in few slots, by steps, zeros among them."""
    n = shape[-1]
    s = rng.integers(120, 126, shape)
    if kind == "every slot":
        s[..., 0] += 60
    elif kind == "by chance":
        s = rng.integers(20, 240, shape)
    elif kind == "a few slots":  # in which the others' groups count for nothing beside the first, and as much as any slot's for themselves
        s[rng.random(shape[:-1]) < 0.01, 0] += 45
    elif kind == "steps":
        s = s - 9 * np.arange(n)
    elif kind == "zeros":
        s[..., n - 1] = np.where(rng.random(shape[:-1]) < 0.5, 10, s[..., n - 1])
        s[..., 0] = 10
    return s.astype(np.uint8)


@pytest.mark.parametrize("kind", ["every slot", "by chance", "a few slots", "steps", "zeros"])
@pytest.mark.parametrize("D,H,g,block,lens,L", [(128, 2, 3, 16, [300, 0, 17], 2), (128, 3, 7, 7, [1, 140], 1), (64, 2, 8, 0, [200, 65], 2), (64, 1, 4, 5, [90], 1),
                                               (256, 1, 8, 16, [250, 2], 1), (256, 2, 2, 4, [70], 1), (128, 4, 4, 32, [2500], 1), (128, 2, 6, 16, [40] * 700, 1)])
def test_decode_of_groups_far_apart(D, H, g, block, lens, L, kind):
    B, rng = len(lens), np.random.default_rng(len(lens) + D)
    cache = Q.QCache("e2m1", L, H, D, [n + 1 for n in lens], block, seed=D + g)
    cache.vs.copy_(torch.from_numpy(spread_scales(kind, tuple(cache.vs.shape), rng)).to(DEV))
    if kind == "zeros":
        cache.v[..., torch.from_numpy(Q.groups("e2m1", D)[::2] == 0).to(DEV)] = 0
        last = torch.from_numpy(Q.groups("e2m1", D)[::2] == D // 32 - 1).to(DEV)
        cache.v[:] = torch.where(last & (cache.vs[..., -1:] == 10), torch.zeros_like(cache.v), cache.v)
    q, pos = normal((B, L, H * g, D), 7), rng.integers(0, 60000, B)
    out, st = Q.run_decode(U.cfg_of(L, H, D), cache, 0, q, pos, lens, max(lens))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    got = out.double().cpu().numpy()
    for b in range(B) if B < 20 else (0, 1, 350, B - 1):
        n = lens[b]
        (K, V), byte = (cache.values(w, b, n) for w in "kv"), cache.held("v", b, np.arange(n))[1]
        for l in range(L):
            ref, bar = decode_by_group(U.f64(q[b, l]), int(pos[b]), K[l], V[l], byte[l]) if n else (0.0, 0.0)
            off = np.abs(got[b, l] - ref)
            assert (off <= bar).all(), (b, l, np.nanmax(off / (bar + 1e-300)))
        if kind == "zeros":
            assert (got[b][..., Q.groups("e2m1", D) == 0] == 0).all()


def test_decode_of_groups_far_apart_and_nan():
    """A group far below the others in a slot, another that reads as NaN: the second's dims are NaN, the first's as without it."""
    H, g, D, n = 2, 4, 128, 100
    cache = Q.QCache("e2m1", 1, H, D, [n], 0, seed=3)
    cache.vs[..., 1] = 60
    q = normal((1, 1, H * g, D), 1)
    want, _ = Q.run_decode(U.cfg_of(1, H, D), cache, 0, q, [5], [n], n)
    cache.vs[0, 0, 33, 1, 2] = Q.NAN
    got, st = Q.run_decode(U.cfg_of(1, H, D), cache, 0, q, [5], [n], n)
    hit = torch.zeros((H, g, D), dtype=torch.bool, device=DEV)
    hit[1] = torch.from_numpy(Q.groups("e2m1", D) == 2).to(DEV)
    hit = hit.view(H * g, D)
    assert int(st.item()) == 0 and torch.equal(got[0, 0].isnan(), hit)
    for j in range(4):  # the references differ, so the weights' and the sums' roundings: 2 (2^-21 + (n + 80) 2^-23) of the group's largest
        dims = torch.from_numpy(Q.groups("e2m1", D) == j).to(DEV) & ~hit
        off, most = (got[0, 0] - want[0, 0]).abs()[dims], want[0, 0].abs()[dims].max()
        assert bool((off <= 5e-5 * most).all())


def test_decode_of_the_longest_sequences():
    """32 sequences of 2^30 slots, 2^31 tiles together: blocks of their own that their tables repeat, all values of sequence b's 2^(b - 16). (Keys are
    zeros, so that weights are one and the parts' sums exact up to 2^24 times their unit; joining 58 parts rounds twice 61 times: 2^-17.)"""
    B, S, block, H, D = 32, 1 << 30, 4096, 1, 128
    k = torch.zeros((1, B, block, H, D), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    v = torch.full((1, B, block, H, D), 1.0, device=DEV).to(torch.float8_e4m3fn)
    ks = torch.full((1, B, block, H, 1), 127, dtype=torch.uint8, device=DEV)
    vs = (torch.arange(B, device=DEV) + 111).to(torch.uint8).view(1, B, 1, 1, 1).expand(1, B, block, H, 1).contiguous()
    table = torch.arange(B, dtype=torch.int32, device=DEV).view(B, 1).expand(B, S // block).contiguous()
    c, d, q = U.cfg_of(1, H, D), prcr.qcache_paged(k, v, ks, vs, table), normal((B, 1, 1, D), 1)
    out, st = torch.full((B, 1, 1, D), float("nan"), device=DEV), status_word()
    ws = torch.empty(prcr.decode_quant_workspace_size(c, d, B, 1, 1, S), dtype=torch.uint8, device=DEV)
    prcr.decode_attention_quant(c, d, 0, q, torch.arange(B, device=DEV), i32([S] * B), S, out, st, ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want = torch.exp2(torch.arange(B, device=DEV) - 16.0).view(B, 1, 1, 1)
    assert bool(((out - want).abs() <= 2.0 ** -17 * want).all())


# ----------------------------------------------------------------------------
# one new token: codes and logits that are not finite
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("D,g", [(128, 4), (64, 7), (256, 8)])
def test_decode_nan_codes(D, g, code):
    """E4M3's codes for NaN: in a key all of its KV head's outputs are NaN, in a value that dim's; the others as without it."""
    H, n, slot, c = 3, 90, 41, U.cfg_of(1, 3, D)
    q, base = normal((1, 1, H * g, D), 3), Q.QCache("e4m3", 1, H, D, [n], 16, seed=8)
    want, _ = Q.run_decode(c, base, 0, q, [5], [n], n)
    for what in ("k", "v"):
        cache = Q.QCache("e4m3", 1, H, D, [n], 16, seed=8)
        x, w = cache.k if what == "k" else cache.v, cache.where(0, [slot])
        rows = x[w]
        rows[:, :, 1, 37] = code
        x[w] = rows
        got, st = Q.run_decode(c, cache, 0, q, [5], [n], n)
        hit = torch.zeros((H, g, D), dtype=torch.bool, device=DEV)
        if what == "k":
            hit[1] = True
        else:
            hit[1, :, 37] = True
        hit = hit.view(H * g, D)
        assert int(st.item()) == 0 and torch.equal(got[0, 0].isnan(), hit)
        assert torch.equal(got[0, 0][~hit], want[0, 0][~hit])


@pytest.mark.parametrize("fmt,D,g,n", [("e4m3", 128, 1, 70), ("e4m3", 64, 8, 2000), ("e2m1", 128, 7, 70), ("e2m1", 64, 2, 2000), ("e2m1", 256, 1, 33)])
def test_decode_logits_beyond_float32(fmt, D, g, n):
    """A logit of minus infinity has no weight and the other slots have theirs; where all of a head's are, its outputs are zeros; one of plus
    infinity makes them NaN. (Queries are ones at position 0, keys -1 or 1 in every dim times 2^127.)"""
    H, c, minus, plus = 1, U.cfg_of(1, 1, D), 0xb8 if fmt == "e4m3" else 0xaa, 0x38 if fmt == "e4m3" else 0x22
    q = torch.ones((1, 1, g, D), dtype=torch.bfloat16, device=DEV)
    hit = [0, 3, n // 2, n - 1]

    def run(at, code):
        cache = Q.QCache(fmt, 1, H, D, [n], 16, seed=n)
        w = cache.where(0, at)
        cache.k[w], cache.ks[w] = code, 254
        out, st = Q.run_decode(c, cache, 0, q, [0], [n], n)
        assert int(st.item()) == 0
        return cache, out[0, 0].double().cpu().numpy()

    cache, got = run(hit, minus)
    left = np.setdiff1d(np.arange(n), hit)
    K, V = (Q.stand_for(fmt, *cache.held(w, 0, left))[0] for w in "kv")
    ref, bar = Q.decode64(U.f64(q[0, 0]), 0, K, V)
    assert (np.abs(got - ref) <= bar).all()
    assert (run(np.arange(n), minus)[1] == 0).all()
    assert np.isnan(run([hit[2]], plus)[1]).all()

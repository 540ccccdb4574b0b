"""GPU parity of append_kv_quant, quantize_cache, dequantize_cache and decode_attention_quant
against 64-bit references (quant_util).

Rounding of values that both sides have exactly (values, slots of a bf16 cache) and reading back are
compared bit for bit. A rotated key may lie next to a border between two codes: it is held to half a step
of the format and what float32 is off by before."""
import numpy as np
import pytest
import torch

import cache_ops_util as U
import paper_2606_26631_gb300 as prcr
import quant_util as Q
from cache_ops_util import DEV, Cache, i32, normal

pytestmark = pytest.mark.gpu
CANARY = 0x5a


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def rows_like(shape, seed):
    """bf16 rows, each of a magnitude of its own, from 2^-6 to 2^6."""
    x = normal(shape, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 100)
    return x * torch.exp2(torch.randint(-6, 7, shape[:-1] + (1,), generator=g, device=DEV)).bfloat16()


# ----------------------------------------------------------------------------
# new tokens' rows
# ----------------------------------------------------------------------------
def check_keys(fmt, codes, byte, y, pair):
    """codes [..., D] and scales' bytes against exact rotated keys y (64 bits) of pairs of norm `pair`.

    float32 is off by e = 2^-21 of the pair's norm: cos and sin of an angle rounded to 2^-24 of half a turn (2^-22.3 together), two products and
    their sum (3 2^-24). So the scale is that of a largest magnitude within e of the exact one, and a value is within e and half the way to the
    next code of the exact one, on either side."""
    D, e = y.shape[-1], 2.0 ** -21 * pair
    g, v = Q.groups(fmt, D), Q.VALUES[fmt]
    for j in range(byte.shape[-1]):
        mag = np.abs(y[..., g == j])
        low, high = (mag - e[..., g == j]).max(-1), (mag + e[..., g == j]).max(-1)
        assert (byte[..., j] >= Q.scale_of(fmt, low)).all() and (byte[..., j] <= Q.scale_of(fmt, high)).all()
    s = Q.scale64(byte)[..., g]
    got = Q.stand_for(fmt, codes, byte)
    place = (codes & (127 if fmt == "e4m3" else 7)).astype(int)
    up = v[np.minimum(place + 1, len(v) - 1)] - v[place]
    down = v[place] - v[np.maximum(place - 1, 0)]
    far = (np.abs(y) - np.abs(got)) * np.where(np.signbit(got) == np.signbit(y), 1, -1)
    assert (far <= 0.5 * up * s + e).all() or (place[far > 0.5 * up * s + e] == len(v) - 1).all()
    assert (-far <= 0.5 * down * s + e).all() or (place[-far > 0.5 * down * s + e] == 0).all()
    assert (np.abs(got - y) <= 0.5 * np.maximum(up, down) * s + e).all()


@pytest.mark.parametrize("fmt,L,l0,nl,H,D,block,layout,lens,gap", [
    ("e4m3", 3, 0, 3, 8, 128, 16, prcr.LAYOUT_SECTIONED, [1, 0, 40], 0),
    ("e2m1", 3, 0, 3, 8, 128, 16, prcr.LAYOUT_SECTIONED, [1, 0, 40], 0),
    ("e4m3", 5, 1, 3, 2, 64, 0, prcr.LAYOUT_INTERLEAVED, [7, 1, 3], 1),
    ("e2m1", 5, 1, 3, 2, 64, 0, prcr.LAYOUT_INTERLEAVED, [7, 1, 3], 1),
    ("e4m3", 2, 0, 2, 4, 256, 7, prcr.LAYOUT_SECTIONED, [1, 1, 1], 3),
    ("e2m1", 2, 0, 2, 4, 256, 7, prcr.LAYOUT_SECTIONED, [1, 130, 1], 2),
    ("e4m3", 2, 1, 1, 1, 16, 1, prcr.LAYOUT_SECTIONED, [0, 0, 9], 0),
    ("e4m3", 2, 0, 2, 3, 48, 5, prcr.LAYOUT_SECTIONED, [20], 0),
    ("e4m3", 2, 0, 2, 5, 80, 16, prcr.LAYOUT_INTERLEAVED, [300, 2, 0, 77], 0),
    ("e4m3", 1, 0, 1, 102, 80, 16, prcr.LAYOUT_SECTIONED, [3, 2], 0),
    ("e4m3", 2, 0, 2, 7, 192, 16, prcr.LAYOUT_SECTIONED, [33], 1),
    ("e4m3", 36, 0, 36, 8, 128, 16, prcr.LAYOUT_SECTIONED, [1] * 5, 0),
    ("e2m1", 20, 3, 17, 1, 128, 0, prcr.LAYOUT_SECTIONED, [70], 0),
    ("e2m1", 2, 0, 2, 128, 64, 4, prcr.LAYOUT_SECTIONED, [9, 2], 0),
])
def test_append(fmt, L, l0, nl, H, D, block, layout, lens, gap):
    rng = np.random.default_rng(3)
    B, T = len(lens), sum(lens)
    len_in = rng.integers(0, 40, B)
    cache = Q.QCache(fmt, L, H, D, [int(a + b + 2) for a, b in zip(len_in, lens)], block, fill=CANARY, gap=gap)
    src = rows_like((nl, T + 3, 3, H, D), 11)
    ks, vs = src[:, :, 0], src[:, :, 1]
    pos = rng.integers(-2 ** 31, 2 ** 31, (T + 3, 3)).astype(np.int32) if D == 80 else rng.integers(0, 40000, (T + 3, 3))
    before = [x.clone() for x in cache.all()]
    li, st = i32(len_in), status_word()
    lo = torch.full_like(li, -7)
    prcr.append_kv_quant(U.cfg_of(L, H, D, layout), cache.desc(), l0, ks, vs, i32(pos), U.offsets(lens), li, lo, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and np.array_equal(lo.cpu().numpy(), len_in + lens)
    at = 0
    for b, n in enumerate(lens):
        slots = np.arange(len_in[b], len_in[b] + n)
        if n:
            codes, byte = (x[l0:l0 + nl] for x in cache.held("v", b, slots))
            ref = Q.quantize(fmt, U.f64(vs[:, at:at + n]))
            assert np.array_equal(byte, ref[1]) and np.array_equal(codes, ref[0])
            codes, byte = (x[l0:l0 + nl] for x in cache.held("k", b, slots))
            x = U.f64(ks[:, at:at + n])
            pair = np.sqrt(x[..., :D // 2] ** 2 + x[..., D // 2:] ** 2)
            exact = U.rope64(x, pos[at:at + n], D, layout)
            check_keys(fmt, codes, byte, exact, np.concatenate([pair, pair], -1))
            if np.abs(pos).max() <= 40000:  # where the oracle's angles are exact to 2^-36 the codes are those of the exact rotation
                ref = Q.quantize(fmt, exact)
                assert np.array_equal(byte, ref[1]) and np.array_equal(codes, ref[0])
        for x_ in (cache.k, cache.v, cache.ks, cache.vs):  # back to what they were: nothing else may differ
            w = cache.where(b, slots)
            rows = x_[w]
            rows[l0:l0 + nl] = CANARY
            x_[w] = rows
        at += n
    for x, y in zip(cache.all(), before):
        assert torch.equal(x, y)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_append_errors(fmt):
    """Full cache, unmapped block, negative length: those rows are skipped and reported; malformed
    offsets: nothing is written and lengths stay."""
    L, H, D = 2, 2, 64
    c = U.cfg_of(L, H, D)
    ks, vs = normal((L, 12, H, D), 1), normal((L, 12, H, D), 2)
    pos = i32(np.zeros((12, 3)))
    cache = Q.QCache(fmt, L, H, D, [32, 32, 32], 8, fill=CANARY, unmapped=[(1, 2)])
    st, li = status_word(), i32([30, 14, -1])
    lo = torch.full_like(li, -7)
    prcr.append_kv_quant(c, cache.desc(), 0, ks, vs, pos, U.offsets([4, 4, 4]), li, lo, st)
    torch.cuda.synchronize()
    assert int(st.item()) == prcr.ST_CAPACITY | prcr.ST_NO_BLOCK and lo.tolist() == [34, 18, 3]
    ref = Q.quantize(fmt, U.f64(vs))
    for b, slots, n in ((0, [30, 31], 0), (1, [14, 15], 4)):
        codes, byte = cache.held("v", b, slots)
        assert np.array_equal(codes, ref[0][:, n:n + 2]) and np.array_equal(byte, ref[1][:, n:n + 2])
        for x in (cache.k, cache.v, cache.ks, cache.vs):
            x[cache.where(b, slots)] = CANARY
    assert all(bool((x == CANARY).all()) for x in cache.all())
    for off in ([1, 4, 8, 12], [0, 8, 4, 12], [0, 4, 8, 13], [0, -3, 8, 12], [0, 2 ** 30, 8, 12]):
        st, li = status_word(), i32([3, 4, 5])
        lo = torch.full_like(li, -7)
        prcr.append_kv_quant(c, cache.desc(), 0, ks, vs, pos, i32(off), li, lo, st)
        torch.cuda.synchronize()
        assert int(st.item()) == prcr.ST_CSR and torch.equal(lo, li)
        assert all(bool((x == CANARY).all()) for x in cache.all())


def test_append_of_nothing():
    """No tokens at all: lengths are passed on."""
    c, cache = U.cfg_of(2, 2, 64), Q.QCache("e2m1", 2, 2, 64, [8, 8], 0, fill=CANARY)
    li, st = i32([3, 0]), status_word()
    lo = torch.full_like(li, -7)
    empty = torch.empty((2, 0, 2, 64), dtype=torch.bfloat16, device=DEV)
    prcr.append_kv_quant(c, cache.desc(), 0, empty, empty, torch.empty((0, 3), dtype=torch.int32, device=DEV), i32([0, 0, 0]), li, lo, st)
    torch.cuda.synchronize()
    assert torch.equal(lo, li) and int(st.item()) == 0 and all(bool((x == CANARY).all()) for x in cache.all())


# ----------------------------------------------------------------------------
# slots of a bf16 cache and back
# ----------------------------------------------------------------------------
def hard_rows(fmt, n, H, D, seed):
    """[n, H, D] bf16 rows with borders of the format, zeros of both signs, the smallest and the largest numbers, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, H, D)) * np.exp2(rng.integers(-140, 128, (n, H, 1)).astype(np.float64))
    v = Q.VALUES[fmt]
    mid = (v[1:] + v[:-1]) / 2
    for i in range(0, n, 3):  # halves between codes, with the largest code for the scale
        s = 2.0 ** rng.integers(-100, 100)
        x[i] = rng.choice(np.concatenate([mid, v]), (H, D)) * s * rng.choice([-1, 1], (H, D))
        x[i, :, ::7] = v[-1] * s
    if n > 12:
        x[1], x[2] = 0.0, -0.0
        x[4] = 2.0 ** -133
        x[5] = np.where(rng.random((H, D)) < 0.5, 3.3895e38, -1e38)
        x[7, 0, 3], x[8, -1, D - 1], x[10, 0, 0] = np.inf, np.nan, -np.inf
        x[11] = 1e-30
        x[11, :, 5] = 3e38
    return torch.from_numpy(x).float().bfloat16().to(DEV)


CASTS = [
    # fmt, layers of the two caches and of the call, H, D, blocks, counts, begins
    ("e4m3", 2, 3, 2, 8, 128, 16, 16, [1, 0, 45], ([0, 3, 7], [5, 0, 0]), 0),
    ("e2m1", 2, 3, 2, 8, 128, 16, 16, [1, 0, 45], ([0, 3, 7], [5, 0, 0]), 0),
    ("e4m3", 3, 2, 1, 2, 64, 0, 7, [33, 20], ([1, 0], [0, 9]), 1),
    ("e2m1", 3, 2, 1, 2, 64, 7, 0, [33, 20], ([1, 0], [0, 9]), 2),
    ("e4m3", 1, 1, 1, 4, 256, 0, 0, [300], ([0], [0]), 0),
    ("e2m1", 1, 1, 1, 4, 256, 32, 8, [300], ([5], [2]), 1),
    ("e4m3", 12, 12, 12, 3, 80, 5, 0, [40, 2, 0, 1], ([0, 1, 2, 3], [3, 2, 1, 0]), 0),
    ("e4m3", 1, 2, 1, 1, 16, 1, 1, [50], ([0], [0]), 0),
    ("e4m3", 1, 1, 1, 102, 80, 16, 0, [4, 3], ([0, 0], [1, 0]), 0),
    ("e4m3", 2, 2, 2, 32, 256, 4, 4, [5], ([0], [0]), 0),
    ("e2m1", 2, 2, 2, 128, 64, 4, 4, [5], ([0], [0]), 0),
]


@pytest.mark.parametrize("fmt,LS,LD,nl,H,D,block,qblock,counts,begins,gap", CASTS)
def test_cast_and_read(fmt, LS, LD, nl, H, D, block, qblock, counts, begins, gap):
    B, (sb, db) = len(counts), begins
    c = U.cfg_of(max(LS, LD), H, D)
    src = Cache(LS, H, D, [n + s + 1 for n, s in zip(counts, sb)], block, seed=3, gap=8 * gap)
    dst = Q.QCache(fmt, LD, H, D, [n + d + 1 for n, d in zip(counts, db)], qblock, fill=CANARY, gap=gap)
    for b, n in enumerate(counts):
        w = src.where(b, np.arange(sb[b], sb[b] + n))
        for x, seed in ((src.k, 10), (src.v, 20)):
            x[w] = torch.stack([hard_rows(fmt, n, H, D, seed + b + 100 * l) for l in range(LS)])
    ls, ld = LS - nl, LD - nl
    st = status_word()
    prcr.quantize_cache(c, src.desc(), ls, dst.desc(), ld, nl, i32(sb), i32(db), i32(counts), max(counts), st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    back = Cache(LS, H, D, [n + s + 1 for n, s in zip(counts, sb)], block, seed=3, fill=U.CANARY, gap=8 * gap)  # (src's table)
    back_before = back.k_all.clone()
    prcr.dequantize_cache(c, dst.desc(), ld, back.desc(), ls, nl, i32(db), i32(sb), i32(counts), max(counts), st)
    again = Q.QCache(fmt, LD, H, D, dst.caps, qblock, fill=CANARY, gap=gap)
    prcr.quantize_cache(c, back.desc(), ls, again.desc(), ld, nl, i32(sb), i32(db), i32(counts), max(counts), st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    untouched = [torch.full_like(x, CANARY) for x in dst.all()]
    for b, n in enumerate(counts):
        slots, w = np.arange(db[b], db[b] + n), src.where(b, np.arange(sb[b], sb[b] + n))
        for which, x, y in (("k", src.k, back.k), ("v", src.v, back.v)):
            if n == 0:
                continue
            ref = Q.quantize(fmt, U.f64(x[w][ls:]))
            codes, byte = (z[ld:] for z in dst.held(which, b, slots))
            assert np.array_equal(byte, ref[1])
            assert np.array_equal(codes, ref[0])
            val = Q.stand_for(fmt, *ref)
            got = U.f64(y[w][ls:])
            assert np.array_equal(got, val, equal_nan=True) and np.array_equal(np.signbit(got[val == 0]), np.signbit(val[val == 0]))
            # quantising what was read back gives values that are the same
            codes, byte = (z[ld:] for z in again.held(which, b, slots))
            assert np.array_equal(Q.stand_for(fmt, codes, byte), val, equal_nan=True)
        for x in (dst.k, dst.v, dst.ks, dst.vs):
            wd = dst.where(b, slots)
            rows = x[wd]
            rows[ld:] = CANARY
            x[wd] = rows
        for x in (back.k, back.v):
            rows = x[w]
            rows[ls:] = U.CANARY
            x[w] = rows
    assert all(torch.equal(x, y) for x, y in zip(dst.all(), untouched))
    assert torch.equal(back.k_all, back_before) and torch.equal(back.v_all, back_before)


@pytest.mark.parametrize("fmt,nl,H,D,counts", [("e4m3", 1, 3, 128, [26001, 70]), ("e2m1", 1, 4, 64, [3, 26100, 0]), ("e2m1", 2, 6, 64, [26007])])
def test_cast_and_read_of_few_layers(fmt, nl, H, D, counts):
    """So many rows of so few layers that a CTA takes several rounds of them."""
    test_cast_and_read(fmt, nl, nl, nl, H, D, 16, 7, counts, ([2] * len(counts), [1] * len(counts)), 0)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_read_every_code(fmt):
    """Every code with every scale's byte, whoever wrote them: rounded to bf16 where that does not hold the value."""
    H, D, S = 2, 128, 256
    cache = Q.QCache(fmt, 1, H, D, [S], 0, fill=0)
    rng = np.random.default_rng(0)
    codes = rng.permuted(np.tile(np.arange(256 if fmt == "e4m3" else 16, dtype=np.uint8), S * H * D // (256 if fmt == "e4m3" else 16))).reshape(1, 1, S, H, D)
    byte = np.broadcast_to(np.arange(S, dtype=np.uint8)[None, None, :, None, None], (1, 1, S, H, cache.n)).copy()
    if cache.n > 1:
        byte = byte + np.arange(cache.n, dtype=np.uint8)
    for x, s in ((cache.k, cache.ks), (cache.v, cache.vs)):
        x.copy_(torch.from_numpy(Q.pack(fmt, codes)))
        s.copy_(torch.from_numpy(byte))
    out, st = Cache(1, H, D, [S], 0, fill=U.CANARY), status_word()
    prcr.dequantize_cache(U.cfg_of(1, H, D), cache.desc(), 0, out.desc(), 0, 1, i32([0]), i32([0]), i32([S]), S, st)
    torch.cuda.synchronize()
    want = torch.from_numpy(Q.stand_for(fmt, codes, byte)).float().bfloat16()  # (float32 holds them all but those that are infinite in bf16 too)
    for x in (out.k, out.v):
        got = x.cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(got.float(), nan=7.0), torch.nan_to_num(want.float(), nan=7.0))


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_cast_errors(fmt, read):
    """Counts and begins out of range, full caches, unmapped blocks in either: reported, those rows left as they were."""
    L, H, D, c = 2, 2, 64, U.cfg_of(2, 2, 64)

    def go(sb, db, n, top, unmapped=(), qunmapped=()):
        wide = Cache(L, H, D, [24, 24], 8, seed=1, fill=U.CANARY if read else None, unmapped=unmapped)
        few = Q.QCache(fmt, L, H, D, [24, 24], 8, seed=1, fill=None if read else CANARY, unmapped=qunmapped)
        st = status_word()
        if read:
            prcr.dequantize_cache(c, few.desc(), 0, wide.desc(), 0, L, i32(sb), i32(db), i32(n), top, st)
        else:
            prcr.quantize_cache(c, wide.desc(), 0, few.desc(), 0, L, i32(sb), i32(db), i32(n), top, st)
        torch.cuda.synchronize()
        canary = torch.tensor(U.CANARY, dtype=torch.bfloat16)
        out = []
        for b in range(2):
            mapped = [s for s in range(24) if (b, s // 8) not in (unmapped if read else qunmapped)]
            w = (wide if read else few).where(b, mapped)
            x = wide.k[w] != canary.item() if read else few.k[w] != CANARY
            out.append([s for s, hit in zip(mapped, x.any(-1).any(-1).all(0).tolist()) if hit])
        return int(st.item()), out

    full = list(range(4, 10))
    assert go([2, 2], [4, 4], [6, 6], 6) == (0, [full, full])
    assert go([2, 2], [4, 4], [-1, 6], 6) == (prcr.ST_CAPACITY, [[], full])
    assert go([2, 2], [4, 4], [6, 9], 6) == (prcr.ST_CAPACITY, [full, full])
    assert go([-1, 2], [4, 4], [6, 6], 6) == (prcr.ST_CAPACITY, [[], full])
    assert go([2, 2], [4, -3], [6, 6], 6) == (prcr.ST_CAPACITY, [full, []])
    assert go([20, 2], [4, 4], [6, 6], 6) == (prcr.ST_CAPACITY, [list(range(4, 8)), full])
    assert go([2, 2], [20, 4], [6, 6], 6) == (prcr.ST_CAPACITY, [list(range(20, 24)), full])
    assert go([2, 2], [4, 4], [6, 0], 6) == (0, [full, []])
    assert go([2 ** 31 - 1, 2], [4, 4], [6, 6], 6) == (prcr.ST_CAPACITY, [[], full])
    # an unmapped block in the cache that is read, and in the one that is written
    a, b = ([(1, 0)], []) if not read else ([], [(1, 0)])
    assert go([2, 2], [4, 4], [6, 8], 8, a, b) == (prcr.ST_NO_BLOCK, [full, list(range(10, 12))])
    assert go([2, 2], [4, 4], [6, 8], 8, b, a) == (prcr.ST_NO_BLOCK, [full, list(range(8, 12))])


# ----------------------------------------------------------------------------
# one new token
# ----------------------------------------------------------------------------
def check_decode(fmt, L, layers, H, g, D, lens, block, seed=0, gap=0, max_len=None, q_scale=1.0, caps=None, pos=None, layout=prcr.LAYOUT_SECTIONED):
    cache = Q.QCache(fmt, L, H, D, caps or [n + 3 for n in lens], block, seed=seed, gap=gap)
    c = U.cfg_of(L, H, D, layout)
    l0, nl = layers
    q = normal((len(lens), nl, H * g, D), seed + 7, q_scale)
    rng = np.random.default_rng(seed)
    pos = rng.integers(0, 60000, len(lens)) if pos is None else pos
    out, st = Q.run_decode(c, cache, l0, q, pos, lens, max(lens) if max_len is None else max_len)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    got = out.double().cpu().numpy()
    for b, n in enumerate(lens):
        K, V = (cache.values(w, b, n) for w in "kv")
        for l in range(nl):
            ref, bar = Q.decode64(U.f64(q[b, l]), int(pos[b]), K[l0 + l], V[l0 + l], layout)
            off = np.abs(got[b, l] - ref)
            assert (off <= bar).all(), (b, l, (off / bar).max())


@pytest.mark.parametrize("block,gap", [(0, 0), (16, 0), (7, 1)])
@pytest.mark.parametrize("H,g", [(1, 1), (2, 3), (3, 4), (2, 5), (4, 7), (1, 8)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_decode(fmt, D, H, g, block, gap):
    check_decode(fmt, 2, (0, 2), H, g, D, [1, 0, 17, 130], block, seed=H * 10 + g, gap=gap)


@pytest.mark.parametrize("fmt,D,H,g,lens,block", [
    ("e4m3", 128, 2, 4, [5000, 1, 777], 16), ("e2m1", 128, 2, 7, [5000, 2, 777], 16), ("e4m3", 64, 1, 8, [9001], 0),
    ("e2m1", 64, 1, 4, [9001], 7), ("e4m3", 256, 1, 8, [4100, 33], 32), ("e2m1", 256, 1, 2, [4100, 33], 16),
    ("e4m3", 128, 8, 4, [933], 0), ("e2m1", 128, 8, 1, [60, 61, 62, 63, 64, 65], 64)])
def test_decode_long(fmt, D, H, g, lens, block):
    check_decode(fmt, 3, (1, 2), H, g, D, lens, block, seed=5)
    check_decode(fmt, 2, (1, 1), H, g, D, lens, block, seed=6, max_len=max(lens) + 700, caps=[max(lens) + 700] * len(lens), layout=prcr.LAYOUT_INTERLEAVED)


@pytest.mark.parametrize("fmt,D,H,g,block,lens", [
    ("e4m3", 128, 2, 4, 16, [0] * 33 + [1, 40, 0, 17]),                      # nothing in the first 32 sequences
    ("e2m1", 64, 3, 5, 0, [(37 * i) % 150 for i in range(70)]),
    ("e4m3", 256, 1, 8, 7, [700 if i == 40 else 0 for i in range(65)]),      # all of the work in one of them
    ("e2m1", 128, 4, 7, 32, [33] * 32 + [0] * 32 + [500]),
    ("e4m3", 64, 2, 1, 16, [0] * 64)])
def test_decode_many_sequences(fmt, D, H, g, block, lens):
    check_decode(fmt, 2, (0, 2), H, g, D, lens, block, seed=len(lens), max_len=800, caps=[800] * len(lens))


@pytest.mark.parametrize("fmt,D,H,g,long", [("e4m3", 128, 2, 4, 0), ("e2m1", 64, 3, 1, 3000), ("e4m3", 256, 1, 5, 700), ("e2m1", 128, 1, 1, 0)])
def test_decode_of_many_rows(fmt, D, H, g, long):
    """Many more rows than warps: units that one warp has whole, units that two share, one that many do, sequences without a slot."""
    lens = [(29 * i) % 90 if i % 7 else 0 for i in range(299)] + [long]
    check_decode(fmt, 9, (1, 8), H, g, D, lens, 16, seed=2, max_len=3000, caps=[n + 1 for n in lens[:-1]] + [3000])


@pytest.mark.parametrize("fmt,g", [("e4m3", 4), ("e4m3", 8), ("e2m1", 2), ("e2m1", 7)])
def test_decode_sums_are_rounded(fmt, g):
    """Values of one sign over 8192 slots in one share (512 sequences of the same blocks): sums of 512 tiles or fewer that are rounded to
    nearest are off by 2^-24 / sqrt(3) sqrt(512) = 8e-7 in the mean square, without a sign; cut off, by 512 2^-25 = 1.5e-5 and more, all one way."""
    B, S, H, D, n = 512, 8192, 4, 128, 1 if fmt == "e4m3" else 4
    rng, blocks = np.random.default_rng(1), 8192 // 16
    shape = (1, blocks, 16, H, D)
    if fmt == "e4m3":
        k, v = normal(shape, 1).to(torch.float8_e4m3fn), (1 + normal(shape, 2).abs().clamp(max=1)).to(torch.float8_e4m3fn)
        K, V = k.double().cpu().numpy(), v.double().cpu().numpy()
    else:
        codes = [rng.integers(0, 16, shape), rng.integers(2, 8, shape)]
        K, V = (Q.VALUES[fmt][c & 7] * np.where(c > 7, -1.0, 1.0) for c in codes)
        k, v = (torch.from_numpy((c[..., ::2] | c[..., 1::2] << 4).astype(np.uint8)).to(DEV) for c in codes)
    scale = torch.full((1, blocks, 16, H, n), 127, dtype=torch.uint8, device=DEV)
    table = torch.arange(blocks, dtype=torch.int32, device=DEV).repeat(B, 1)
    c, d, q = U.cfg_of(1, H, D), prcr.qcache_paged(k, v, scale, scale.clone(), table), normal((B, 1, H * g, D), 3)
    out, st = torch.empty((B, 1, H * g, D), device=DEV), status_word()
    ws = torch.empty(prcr.decode_quant_workspace_size(c, d, B, 1, H * g, S), dtype=torch.uint8, device=DEV)
    prcr.decode_attention_quant(c, d, 0, q, torch.zeros(B, dtype=torch.int64, device=DEV), i32([S] * B), S, out, st, ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for b in (0, 300, B - 1):
        x = np.einsum("hgd,shd->hgs", U.f64(q[b, 0]).reshape(H, g, D), K.reshape(S, H, D)) / np.sqrt(D)
        p = np.exp(x - x.max(-1, keepdims=True))
        ref = (np.einsum("hgs,shd->hgd", p, V.reshape(S, H, D)) / p.sum(-1)[..., None]).reshape(H * g, D)
        off = out[b, 0].double().cpu().numpy() / ref - 1
        assert abs(off.mean()) < 2e-6 and np.abs(off).max() < 8e-6


def test_decode_repeats():
    """The same call gives the same bits, whatever the workspace held."""
    c, lens = U.cfg_of(3, 2, 128), [900, 3, 450, 0]
    cache, q, pos = Q.QCache("e2m1", 3, 2, 128, lens, 16, seed=2), normal((4, 3, 14, 128), 3), torch.tensor([9, 8, 7, 6], device=DEV)
    d, ln, st = cache.desc(), i32(lens), status_word()
    need = prcr.decode_quant_workspace_size(c, d, 4, 3, 14, 900)
    outs = []
    for fill in (0, 255, 127):
        ws, out = torch.full((need,), fill, dtype=torch.uint8, device=DEV), torch.full((4, 3, 14, 128), float("nan"), device=DEV)
        prcr.decode_attention_quant(c, d, 0, q, pos, ln, 900, out, st, ws)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and int(st.item()) == 0


@pytest.mark.parametrize("n", list(range(1, 20)) + [31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025])
@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("e2m1", 128), ("e2m1", 64), ("e4m3", 256)])
def test_decode_lengths(fmt, D, n):
    check_decode(fmt, 1, (0, 1), 1, 4, D, [n], 16, seed=n)


@pytest.mark.parametrize("q_scale", [2.0 ** -20, 0.01, 30.0, 300.0])
@pytest.mark.parametrize("fmt,g", [("e4m3", 4), ("e2m1", 6)])
def test_decode_of_small_and_large_queries(fmt, g, q_scale):
    check_decode(fmt, 1, (0, 1), 2, g, 128, [400], 16, q_scale=q_scale)


def test_decode_positions():
    """Far positions, and ones beyond what the rotation takes: those sequences read no slot."""
    check_decode("e4m3", 1, (0, 1), 2, 4, 128, [40, 50], 16, pos=[2 ** 31 - 1, -2 ** 31 + 1])
    cache, c = Q.QCache("e2m1", 1, 2, 64, [40, 40, 40], 16), U.cfg_of(1, 2, 64)
    q = normal((3, 1, 8, 64), 1)
    out, st = Q.run_decode(c, cache, 0, q, [2 ** 31, 5, -2 ** 31], [40, 40, 40], 40)
    assert int(st.item()) == prcr.ST_POS_RANGE
    assert bool((out[0] == 0).all()) and bool((out[2] == 0).all()) and bool((out[1] != 0).any())


@pytest.mark.parametrize("fmt,g", [("e4m3", 4), ("e4m3", 7), ("e2m1", 3), ("e2m1", 8)])
def test_decode_scales_far_apart(fmt, g):
    """Scales over many octaves: keys' rows, and values whose weights and scales compensate each other."""
    H, D, n, c = 1, 128, 300, U.cfg_of(1, 1, 128)
    for spread, at in ((12, "v"), (40, "v"), (6, "k"), (200, "v")):
        cache = Q.QCache(fmt, 1, H, D, [n], 0, seed=spread)
        rng = np.random.default_rng(spread)
        shape = (1, 1, n, H, cache.n)
        s = (122 if fmt == "e4m3" else 125) + rng.integers(-spread // 2, spread // 2 + 1, shape)
        (cache.vs if at == "v" else cache.ks).copy_(torch.from_numpy(np.clip(s, 10, 240).astype(np.uint8)))
        q = normal((1, 1, g, D), 4)
        out, st = Q.run_decode(c, cache, 0, q, [77], [n], n)
        ref, bar = Q.decode64(U.f64(q[0, 0]), 77, cache.values("k", 0, n)[0], cache.values("v", 0, n)[0])
        off = np.abs(out[0, 0].double().cpu().numpy() - ref)
        assert (off <= bar).all(), (spread, at, (off / bar).max())


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("g", [2, 6])
def test_decode_reads_nothing_else(fmt, g):
    """Slots past a sequence's length and in unmapped blocks hold NaN: no influence; unmapped blocks are reported."""
    L, H, D, c = 2, 2, 128, U.cfg_of(2, 2, 128)
    lens = [37, 64, 0, 5]
    cache = Q.QCache(fmt, L, H, D, [96] * 4, 16, seed=2)
    q = normal((4, L, H * g, D), 9)
    want, st = Q.run_decode(c, cache, 0, q, [9, 8, 7, 6], lens, 64)
    assert int(st.item()) == 0
    for b, n in enumerate(lens):
        w = cache.where(b, np.arange(n, 96))
        for x in (cache.ks, cache.vs):
            x[w] = Q.NAN
        for x in (cache.k, cache.v):
            x[w] = 0xff
    got, st = Q.run_decode(c, cache, 0, q, [9, 8, 7, 6], lens, 64)
    assert int(st.item()) == 0 and torch.equal(got, want) and bool((got[2] == 0).all())
    cache.np_table[1, 1] = -1
    cache.table.copy_(torch.from_numpy(cache.np_table))
    got, st = Q.run_decode(c, cache, 0, q, [9, 8, 7, 6], lens, 64)
    assert int(st.item()) == prcr.ST_NO_BLOCK and torch.equal(got[[0, 2, 3]], want[[0, 2, 3]])
    seen = np.r_[0:16, 32:64]
    K, V = (Q.stand_for(fmt, *cache.held(w, 1, seen)) for w in "kv")
    for l in range(L):
        ref, bar = Q.decode64(U.f64(q[1, l]), 8, K[l], V[l])
        assert (np.abs(got[1, l].double().cpu().numpy() - ref) <= bar).all()
    cache.table.fill_(10 ** 6)
    got, st = Q.run_decode(c, cache, 0, q, [9, 8, 7, 6], lens, 64)
    assert int(st.item()) == prcr.ST_NO_BLOCK and bool((got == 0).all())


def test_decode_lengths_out_of_range():
    c, cache = U.cfg_of(1, 1, 128), Q.QCache("e4m3", 1, 1, 128, [100, 100, 100], 0, seed=3)
    q = normal((3, 1, 4, 128), 5)
    want, _ = Q.run_decode(c, cache, 0, q, [1, 2, 3], [64, 64, 0], 64)
    got, st = Q.run_decode(c, cache, 0, q, [1, 2, 3], [64, 99, -5], 64)  # slots past max_len are left out
    assert int(st.item()) == prcr.ST_CAPACITY and torch.equal(got, want)
    got, st = Q.run_decode(c, cache, 0, q, [1, 2, 3], [0, 0, 0], 0)
    assert int(st.item()) == 0 and bool((got == 0).all())
    got, st = Q.run_decode(c, cache, 0, q, [1, 2, 3], [0, 4, 0], 0)
    assert int(st.item()) == prcr.ST_CAPACITY and bool((got == 0).all())


@pytest.mark.parametrize("g", [4, 5])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_decode_nan_and_infinity(fmt, g):
    """A key that reads as NaN makes its KV head's outputs NaN, a value (E2M1: a group of its dims) its dims, a query its head."""
    H, D, n, c = 3, 128, 90, U.cfg_of(1, 3, 128)
    q = normal((1, 1, H * g, D), 3)
    base = Q.QCache(fmt, 1, H, D, [n], 0, seed=8)
    want, _ = Q.run_decode(c, base, 0, q, [5], [n], n)
    groups = torch.from_numpy(Q.groups(fmt, D)).to(DEV)
    for what in ("k", "v"):
        cache = Q.QCache(fmt, 1, H, D, [n], 0, seed=8)
        (cache.ks if what == "k" else cache.vs)[0, 0, 71, 1, -1] = Q.NAN
        got, st = Q.run_decode(c, cache, 0, q, [5], [n], n)
        hit = torch.zeros((H, g, D), dtype=torch.bool, device=DEV)
        hit[1] = True if what == "k" else (groups == cache.n - 1)
        hit = hit.view(H * g, D)
        assert int(st.item()) == 0 and torch.equal(got[0, 0].isnan(), hit)
        assert torch.equal(got[0, 0][:g], want[0, 0][:g]) and torch.equal(got[0, 0][2 * g:], want[0, 0][2 * g:])
        assert torch.allclose(got[0, 0][~hit], want[0, 0][~hit], rtol=1e-4, atol=1e-5)  # (other references: other roundings)
    for bad in (float("nan"), float("inf")):
        p = q.clone()
        p[0, 0, g + 1, 9] = bad
        got, _ = Q.run_decode(c, base, 0, p, [5], [n], n)
        hit = torch.zeros((H * g, D), dtype=torch.bool, device=DEV)
        hit[g + 1] = True
        assert torch.equal(got[0, 0].isnan(), hit) and torch.allclose(got[0, 0][~hit], want[0, 0][~hit], rtol=1e-4, atol=1e-5)


def test_decode_query_alignment_and_strides():
    """Queries aligned to 4 bytes alone; scales and codes of views with strides of their own, single heads and slots."""
    c = U.cfg_of(2, 1, 64)
    cache = Q.QCache("e4m3", 2, 1, 64, [40], 0, seed=1)
    flat = normal((1 + 2 * 4 * 64 + 8,), 2)
    want = None
    for shift in (2, 8):
        q = flat[shift:shift + 2 * 4 * 64].view(1, 2, 4, 64)
        out, st = Q.run_decode(c, cache, 0, q, [3], [40], 40)
        for l in range(2):
            ref, bar = Q.decode64(U.f64(q[0, l]), 3, cache.values("k", 0, 40)[l], cache.values("v", 0, 40)[l])
            assert (np.abs(out[0, l].double().cpu().numpy() - ref) <= bar).all()


def test_decode_far_addresses():
    """A cache whose offsets pass 2^32 bytes."""
    H, D, n, c = 1, 128, 4400, U.cfg_of(1, 1, 128)
    far = 1 << 20
    big = torch.zeros(n * far, dtype=torch.uint8, device=DEV)
    small = Q.QCache("e4m3", 1, H, D, [n], 0, seed=4)
    view = lambda off, w: torch.as_strided(big, (1, 1, n, H, w), (n * far, n * far, far, w, 1), off)
    parts = [view(0, 128), view(256, 128), view(512, 1), view(640, 1)]
    for x, y in zip(parts, (small.k, small.v, small.ks, small.vs)):
        x.copy_(y)
    d = prcr.qcache_contiguous(parts[0].view(torch.float8_e4m3fn), parts[1].view(torch.float8_e4m3fn), parts[2], parts[3])
    q, st = normal((1, 1, 4, D), 1), status_word()
    want, _ = Q.run_decode(c, small, 0, q, [3], [n], n)
    out = torch.empty_like(want)
    ws = torch.empty(max(16, prcr.decode_quant_workspace_size(c, d, 1, 1, 4, n)), dtype=torch.uint8, device=DEV)
    prcr.decode_attention_quant(c, d, 0, q, torch.tensor([3], device=DEV), i32([n]), n, out, st, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    rows = Cache(1, H, D, [n], 0, fill=0.0)
    prcr.dequantize_cache(c, d, 0, rows.desc(), 0, 1, i32([0]), i32([0]), i32([n]), n, st)
    rows2 = Cache(1, H, D, [n], 0, fill=0.0)
    prcr.dequantize_cache(c, small.desc(), 0, rows2.desc(), 0, 1, i32([0]), i32([0]), i32([n]), n, st)
    assert torch.equal(rows.k, rows2.k) and torch.equal(rows.v, rows2.v) and int(st.item()) == 0
    for x in parts:
        x.zero_()
    prcr.quantize_cache(c, rows2.desc(), 0, d, 0, 1, i32([0]), i32([0]), i32([n]), n, st)
    prcr.dequantize_cache(c, d, 0, rows.desc(), 0, 1, i32([0]), i32([0]), i32([n]), n, st)
    torch.cuda.synchronize()
    assert torch.equal(rows.k, rows2.k) and torch.equal(rows.v, rows2.v) and int(st.item()) == 0


# ----------------------------------------------------------------------------
# together
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_a_dialogue(fmt):
    """A decoder's order: a prompt's rows appended, its chunk attention over rows read back, a revisit's rebound rows cast behind
    it, a decode step whose own token is appended first; against the same steps on the values that the cache stands for."""
    L, H, g, D, B, block = 2, 2, 4, 128, 2, 16
    c = U.cfg_of(L, H, D)
    cache = Q.QCache(fmt, L, H, D, [200] * B, block, fill=0)
    d, st = cache.desc(), status_word()
    new = [40, 23]
    T = sum(new)
    k, v = normal((L, T, H, D), 1), normal((L, T, H, D), 2)
    pos = np.concatenate([np.stack([np.arange(n)] * 3, 1) for n in new])
    zero, lens, more = i32([0] * B), i32([0] * B), i32([0] * B)
    prcr.append_kv_quant(c, d, 0, k, v, i32(pos), U.offsets(new), zero, lens, st)
    rows = Cache(L, H, D, [200] * B, 0, fill=0.0)
    prcr.dequantize_cache(c, d, 0, rows.desc(), 0, L, zero, zero, lens, 200, st)
    q = normal((T, H * g, D), 3)
    out = torch.empty_like(q)
    ws = torch.empty(max(16, prcr.chunk_workspace_size(c, B, H * g, T, 200)), dtype=torch.uint8, device=DEV)
    prcr.chunk_attention(c, rows.desc(), 1, q, i32(pos), U.offsets(new), lens, max(new), out, st, ws)
    torch.cuda.synchronize()
    at = 0
    for b, n in enumerate(new):
        K, V = (cache.values(w, b, n)[1] for w in "kv")
        assert np.array_equal(U.f64(rows.k[b, 1, :n]), K) and np.array_equal(U.f64(rows.v[b, 1, :n]), V)
        ref, bar = U.chunk64(U.f64(q[at:at + n]), pos[at:at + n], K, V, U.causal(n, n, n))
        assert (np.abs(U.f64(out[at:at + n]) - ref) <= bar).all()
        at += n
    # a revisit: six tokens of a raw store, rebound into bf16 rows, cast behind the prompt
    M, K6 = 30, 6
    sk, sv = normal((B, L, M, H, D), 5), normal((B, L, M, H, D), 6)
    coords = i32(np.broadcast_to(np.stack([np.zeros(M), np.arange(M) // 6, np.arange(M) % 6], 1), (B, M, 3)).copy())
    store = prcr.store_desc(sk, sv, coords)
    batch = prcr.revisit_batch(i32([0, 1, 2]), i32([0, K6, 2 * K6]), i32([1, 2, 8, 9, 15, 16] * 2),
                               torch.tensor(new, device=DEV), zero)
    staged = Cache(L, H, D, [K6] * B, 0, fill=0.0)
    got, nxt = torch.zeros_like(zero), torch.zeros(B, dtype=torch.int64, device=DEV)
    work = torch.empty(max(16, prcr.workspace_size(2 * K6)), dtype=torch.uint8, device=DEV)
    prcr.rebind_inject(c, store, staged.desc(), batch, prcr.outputs(got, nxt, st), workspace=work)
    prcr.quantize_cache(c, staged.desc(), 0, d, 0, L, zero, lens, got, K6, st)
    lens2 = lens + got
    # the step's own token, then the step
    k1, v1 = normal((L, B, H, D), 7), normal((L, B, H, D), 8)
    p1 = np.stack([nxt.cpu().numpy()] * 3, 1)
    prcr.append_kv_quant(c, d, 0, k1, v1, i32(p1), i32([0, 1, 2]), lens2, more, st)
    q1 = normal((B, L, H * g, D), 9)
    res, _ = Q.run_decode(c, cache, 0, q1, nxt.cpu().numpy(), more.cpu().numpy(), 200, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and more.tolist() == [n + K6 + 1 for n in new]
    for b, n in enumerate(more.tolist()):
        for w, x in (("k", staged.k), ("v", staged.v)):
            ref = Q.quantize(fmt, U.f64(x[b]))
            codes, byte = cache.held(w, b, np.arange(n - 1 - K6, n - 1))
            assert np.array_equal(codes, ref[0]) and np.array_equal(byte, ref[1])
        K, V = (cache.values(w, b, n) for w in "kv")
        for l in range(L):
            ref, bar = Q.decode64(U.f64(q1[b, l]), int(nxt[b]), K[l], V[l])
            assert (np.abs(res[b, l].double().cpu().numpy() - ref) <= bar).all()


def test_graph_and_streams():
    """Captured, replayed on new inputs in place, beside eager calls on another stream with its own workspace: the same results."""
    L, H, g, D, B, c = 2, 2, 4, 128, 3, U.cfg_of(2, 2, 128)
    cache, lens = Q.QCache("e4m3", L, H, D, [600] * B, 16, seed=1), [590, 100, 317]
    d = cache.desc()
    k, v, q = normal((L, B, H, D), 1), normal((L, B, H, D), 2), normal((B, L, H * g, D), 3)
    pos, off, ln, out_len = i32(np.full((B, 3), 700)), i32([0, 1, 2, 3]), i32(lens), i32([0] * B)
    qp, out, st = torch.full((B,), 700, dtype=torch.int64, device=DEV), torch.zeros((B, L, H * g, D), device=DEV), status_word()
    need = max(16, prcr.decode_quant_workspace_size(c, d, B, L, H * g, 600))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def step(out, ws, stream=None):
        prcr.append_kv_quant(c, d, 0, k, v, pos, off, ln, out_len, st, stream=stream)
        prcr.decode_attention_quant(c, d, 0, q, qp, out_len, 600, out, st, ws, stream=stream)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    for seed in (11, 12):
        for x, y in ((k, normal(k.shape, seed)), (v, normal(v.shape, seed + 1)), (q, normal(q.shape, seed + 2))):
            x.copy_(y)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out2, ws2 = torch.empty_like(out), torch.empty_like(ws)
        side.wait_stream(torch.cuda.current_stream())
        step(out2, ws2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, out2) and int(st.item()) == 0
        for b in range(B):
            K, V = (cache.values(w, b, lens[b] + 1) for w in "kv")
            ref, bar = Q.decode64(U.f64(q[b, 1]), 700, K[1], V[1])
            assert (np.abs(got[b, 1].double().cpu().numpy() - ref) <= bar).all()


@pytest.mark.parametrize("fmt,D,g", [("e4m3", 128, 4), ("e2m1", 64, 6)])
def test_graph_of_growing_lengths(fmt, D, g):
    """A captured step whose lengths, positions and blocks change in place between replays: what an eager call gives."""
    L, H, B, c = 3, 4, 40, U.cfg_of(3, 4, D)
    cache = Q.QCache(fmt, L, H, D, [300] * B, 16, seed=4)
    d, q, st = cache.desc(), normal((B, L, H * g, D), 3), status_word()
    ln, pos = i32([0] * B), torch.zeros(B, dtype=torch.int64, device=DEV)
    out = torch.zeros((B, L, H * g, D), device=DEV)
    ws = torch.empty(prcr.decode_quant_workspace_size(c, d, B, L, H * g, 300), dtype=torch.uint8, device=DEV)
    step = lambda out, ws: prcr.decode_attention_quant(c, d, 0, q, pos, ln, 300, out, st, ws)
    step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    rng = np.random.default_rng(5)
    for lens in ([0] * B, [1] * B, [0] * 39 + [300], rng.integers(0, 301, B), [300] * B):
        ln.copy_(i32(lens))
        pos.copy_(torch.from_numpy(rng.integers(0, 9000, B)))
        cache.table.copy_(cache.table[torch.from_numpy(rng.permutation(B)).to(DEV)])  # the same blocks, of other sequences
        out.fill_(float("nan"))
        graph.replay()
        want, ws2 = torch.full_like(out, float("nan")), torch.empty_like(ws)
        step(want, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and int(st.item()) == 0 and bool((out[ln == 0] == 0).all())

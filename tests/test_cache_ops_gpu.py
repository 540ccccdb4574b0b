"""GPU parity of append_kv, chunk_attention, accumulate_weights and evict against
64-bit references (cache_ops_util).

chunk_attention is held to two bars. Element by element to the sum of its
roundings' bounds (cache_ops_util.chunk64). And as a whole, as the 2-norm of the
difference over that of the result: an unbiased rounding to bf16 is off by
2^-8 / sqrt(3) of the step's binade, 1.6e-3 of the value in the mean square; the query's,
the probabilities' and the output's are independent and, for N(0, 1) inputs, move the output
by that much each, 2.9e-3 together; the bar is 5e-3."""
import numpy as np
import pytest
import torch

import cache_ops_util as U
import paper_2606_26631_gb300 as prcr
from cache_ops_util import DEV, Cache, i32, normal

pytestmark = pytest.mark.gpu
NORM = 5e-3


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def positions(n, p, rng):
    """Half an image of rows of 7, then text."""
    i = np.arange(n)
    img = np.stack([np.full(n, p), p + i // 7, p + i % 7], 1)
    txt = np.stack([p + 9 + i] * 3, 1)
    return np.where((i < n // 2)[:, None], img, txt).astype(np.int32)


# ----------------------------------------------------------------------------
# append
# ----------------------------------------------------------------------------
def run_append(c, desc, layer0, ks, vs, pos, lens, len_in, pad=0):
    off, li = U.offsets(lens), i32(len_in)
    lo, st = torch.full_like(li, -7), status_word()
    prcr.append_kv(c, desc, layer0, ks, vs, i32(pos), off, li, lo, st)
    torch.cuda.synchronize()
    return lo.cpu().numpy(), int(st.item())


@pytest.mark.parametrize("L,l0,nl,H,D,block,layout,lens,strided", [
    (3, 0, 3, 8, 128, 16, prcr.LAYOUT_SECTIONED, [1, 0, 40], False),
    (5, 1, 3, 2, 64, 0, prcr.LAYOUT_INTERLEAVED, [7, 1, 3], True),
    (2, 0, 2, 4, 256, 7, prcr.LAYOUT_SECTIONED, [1, 1, 1], True),
    (2, 1, 1, 1, 16, 1, prcr.LAYOUT_SECTIONED, [0, 0, 9], False),
    (36, 0, 36, 8, 128, 16, prcr.LAYOUT_SECTIONED, [1] * 5, False),
    (2, 0, 2, 5, 80, 16, prcr.LAYOUT_INTERLEAVED, [300, 2, 0, 77], False),
])
def test_append(L, l0, nl, H, D, block, layout, lens, strided):
    rng = np.random.default_rng(3)
    B, T, pad = len(lens), sum(lens), 3
    len_in = rng.integers(0, 40, B)
    cache = Cache(L, H, D, [int(a + b + 2) for a, b in zip(len_in, lens)], block, fill=U.CANARY, gap=8 if strided else 0)
    src = normal((nl, T + pad, 3 if strided else 2, H, D), 11)
    ks, vs = src[:, :, 0], src[:, :, 1]
    pos = rng.integers(-2 ** 31, 2 ** 31, (T + pad, 3)).astype(np.int32) if D == 80 else rng.integers(0, 40000, (T + pad, 3))
    before_k, before_v = cache.k_all.clone(), cache.v_all.clone()
    lo, st = run_append(U.cfg_of(L, H, D, layout), cache.desc(), l0, ks, vs, pos, lens, len_in)
    assert st == 0 and np.array_equal(lo, len_in + lens)
    at = 0
    for b, n in enumerate(lens):
        w = cache.where(b, np.arange(len_in[b], len_in[b] + n))
        got_k, got_v = cache.k[w][l0:l0 + nl], cache.v[w][l0:l0 + nl]
        assert torch.equal(got_v, vs[:, at:at + n])
        x = U.f64(ks[:, at:at + n])
        ref = U.rope64(x, pos[at:at + n], D, layout)
        # half a bf16 step, and float32 sums and cos/sin on the pair's norm
        pair = np.sqrt(x[..., :D // 2] ** 2 + x[..., D // 2:] ** 2)
        bar = 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.concatenate([pair, pair], -1) + 1e-38
        assert (np.abs(U.f64(got_k) - ref) <= bar).all()
        for x_ in (cache.k, cache.v):  # back to what they were: nothing else may differ
            rows = x_[w]
            rows[l0:l0 + nl] = U.CANARY
            x_[w] = rows
        at += n
    assert torch.equal(cache.k_all, before_k) and torch.equal(cache.v_all, before_v)


def test_append_errors():
    """Full cache, unmapped block, negative length: those rows are skipped and reported; malformed
    offsets: nothing is written and lengths stay."""
    L, H, D = 2, 2, 64
    c = U.cfg_of(L, H, D)
    ks, vs = normal((L, 12, H, D), 1), normal((L, 12, H, D), 2)
    pos = np.zeros((12, 3))
    cache = Cache(L, H, D, [32, 32, 32], 8, fill=U.CANARY, unmapped=[(1, 2)])
    lo, st = run_append(c, cache.desc(), 0, ks, vs, pos, [4, 4, 4], [30, 14, -1])
    assert st == prcr.ST_CAPACITY | prcr.ST_NO_BLOCK and list(lo) == [34, 18, 3]
    # the last block, 16..23, of sequence 1 is unmapped; block -1 of the table reads as the last pool block: untouched
    got = cache.v.clone()
    for b, slots, n in ((0, [30, 31], 0), (1, [14, 15], 4)):
        assert torch.equal(got[cache.where(b, slots)], vs[:, n:n + 2])
        got[cache.where(b, slots)] = U.CANARY
    assert bool((got == torch.tensor(U.CANARY, dtype=torch.bfloat16)).all())
    for off in ([1, 4, 8, 12], [0, 8, 4, 12], [0, 4, 8, 13], [0, -3, 8, 12], [0, 2 ** 30, 8, 12]):
        cache = Cache(L, H, D, [32, 32, 32], 8, fill=U.CANARY)
        st, li = status_word(), i32([3, 4, 5])
        lo = torch.full_like(li, -7)
        prcr.append_kv(c, cache.desc(), 0, ks, vs, i32(pos), i32(off), li, lo, st)
        torch.cuda.synchronize()
        assert int(st.item()) == prcr.ST_CSR and torch.equal(lo, li)
        assert bool((cache.k == torch.tensor(U.CANARY, dtype=torch.bfloat16)).all())


# ----------------------------------------------------------------------------
# chunk attention
# ----------------------------------------------------------------------------
class Chunk:
    """A packed batch: new[b] queries over lens[b] slots of a cache."""

    def __init__(self, H, g, D, new, lens, block, L=2, layer=1, layout=prcr.LAYOUT_SECTIONED, seed=0, pad=3, strided=False,
                 q_scale=1.0, caps=None, **cache):
        self.H, self.g, self.D, self.new, self.lens, self.layer, self.layout = H, g, D, list(new), list(lens), layer, layout
        self.cache = Cache(L, H, D, caps or [max(n, 1) + 3 for n in lens], block, seed=seed, **cache)
        T, Hq = sum(new) + pad, H * g
        self.T, rng = T, np.random.default_rng(seed + 9)
        big = normal((T, Hq + (2 * H if strided else 0), D), seed + 3, q_scale)
        self.q = big[:, :Hq]
        self.out_all = torch.full((T, Hq + (1 if strided else 0), D), U.CANARY, dtype=torch.bfloat16, device=DEV)
        self.out = self.out_all[:, :Hq]
        self.pos = np.concatenate([positions(n, int(rng.integers(0, 60000)), rng) for n in new] + [np.zeros((pad, 3), np.int32)])
        self.cfg = U.cfg_of(L, H, D, layout)
        self.args = (i32(self.pos), U.offsets(new), i32(lens))
        self.max_len = max(self.lens + [0])
        self.status = status_word()
        self.ws = self.workspace(self.max_len)

    def workspace(self, max_len):
        n = prcr.chunk_workspace_size(self.cfg, len(self.new), self.H * self.g, self.T, max_len)
        return torch.full((max(n, 16),), 0xff, dtype=torch.uint8, device=DEV)

    def run(self, max_len=None, q_off=None, seq_len=None, ws=None, stream=None):
        m = self.max_len if max_len is None else max_len
        prcr.chunk_attention(self.cfg, self.cache.desc(), self.layer, self.q, self.args[0], self.args[1] if q_off is None else q_off,
                             self.args[2] if seq_len is None else seq_len, m, self.out, self.status,
                             (self.ws if m == self.max_len else self.workspace(m)) if ws is None else ws, stream=stream)
        return self

    def done(self):
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, seqs=None, drop=None, top=None, rows=None):
        """Every query (or `rows` of them) of the sequences against the reference; drop(b): slots left out."""
        at, whole = 0, [0.0, 0.0]
        q, got = U.f64(self.q), U.f64(self.out)
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            if n and (seqs is None or b in seqs):
                S = max(1, min(length, top if top is not None else length))
                K, V = (U.f64(self.cache.rows(x, b, S)[self.layer]) for x in (self.cache.k, self.cache.v))
                i = np.arange(n) if rows is None else np.unique(np.linspace(0, n - 1, rows).astype(int))
                sees = U.causal(n, length, S)[i]
                if drop is not None:
                    sees[:, drop(b, np.arange(S))] = False
                live = sees.any(0)
                ref, bar = U.chunk64(q[at + i], self.pos[at + i], np.where(live[:, None, None], K, 0.0), np.where(live[:, None, None], V, 0.0),
                                     sees, self.layout)
                d = np.abs(got[at + i] - ref)
                assert (d <= bar).all(), (b, np.unravel_index((d - bar).argmax(), d.shape), (d / bar).max())
                whole[0] += (d ** 2).sum()
                whole[1] += (ref ** 2).sum()
            at += n
        if whole[1]:
            assert np.sqrt(whole[0] / whole[1]) <= NORM, np.sqrt(whole[0] / whole[1])
        tail = self.out_all.clone()
        tail[:at, :self.H * self.g] = U.CANARY
        assert bool((tail == torch.tensor(U.CANARY, dtype=torch.bfloat16)).all()), "rows or gaps that are not the call's"


SHAPES = [  # H, g, D, block
    (8, 4, 128, 16), (4, 7, 128, 0), (2, 1, 128, 7), (1, 8, 128, 64), (3, 3, 64, 16), (2, 8, 64, 0), (2, 4, 256, 16), (4, 8, 256, 0),
    (1, 1, 256, 1), (5, 6, 128, 128), (1, 5, 64, 8),
]


@pytest.mark.parametrize("H,g,D,block", SHAPES, ids=lambda v: str(v))
@pytest.mark.parametrize("kind", ["token", "few", "prompt", "extend", "ragged"])
def test_chunk(H, g, D, block, kind):
    new, lens = {"token": ([1, 1, 1], [1, 2, 300]), "few": ([6, 0, 3, 1], [700, 40, 3, 129]), "prompt": ([130, 1, 65], [130, 1, 65]),
                 "extend": ([70, 33], [400, 127 + 33]), "ragged": ([1, 128, 0, 40, 17], [257, 128, 0, 168, 1000])}[kind]
    c = Chunk(H, g, D, new, lens, block, strided=kind in ("few", "extend"), gap=16 if kind == "few" else 0,
              layout=prcr.LAYOUT_INTERLEAVED if kind == "extend" else prcr.LAYOUT_SECTIONED, seed=H * 100 + g)
    assert c.run().done() == 0
    c.check()


@pytest.mark.parametrize("H,g,D,block,new,lens", [
    (8, 4, 128, 16, [1], [9000]), (1, 1, 128, 16, [2], [40000]), (2, 7, 128, 0, [5, 1], [20011, 3]), (4, 4, 64, 32, [3], [12345]),
    (2, 8, 256, 16, [4, 2], [5000, 6001]), (2, 4, 128, 16, [300], [20000]), (1, 8, 128, 0, [1024], [1024]), (2, 2, 64, 16, [2500], [2500]),
    (1, 2, 256, 16, [1500], [1700]), (8, 4, 128, 16, [1900, 0, 800], [1900, 7, 3000]), (4, 8, 256, 0, [1000, 400], [1300, 400]),
    (8, 8, 64, 7, [1500], [1500]), (8, 4, 128, 64, [2600], [2600]), (8, 4, 128, 256, [300, 2300], [5000, 2300]),
    (4, 4, 128, 16, [50, 3, 20], [9000, 4100, 77]), (8, 2, 64, 0, [70, 79], [3000, 5000]), (1, 8, 128, 7, [6] * 24, [2000] * 24),  # few rows
    (3, 1, 64, 32, [160, 160], [160, 4000]), (1, 8, 64, 1, [16, 1], [5000, 130]),
    (8, 4, 128, 16, [6, 1, 0, 40] * 13, [300, 700, 20, 41] * 13), (16, 2, 64, 0, [3, 70] * 10, [500, 90] * 10),  # and many sequences
    (16, 2, 128, 7, [1] * 24, [1, 128, 129, 257] * 6),
], ids=lambda v: str(v))
def test_chunk_long(H, g, D, block, new, lens):
    c = Chunk(H, g, D, new, lens, block, seed=5)
    assert c.run().done() == 0
    c.check(rows=9)


def test_chunk_first_slot_is_exact():
    """A query that sees one slot gets its value, bit for bit (its weight is exactly 1)."""
    for D, g, block in ((128, 4, 16), (64, 7, 0), (256, 2, 7)):
        c = Chunk(2, g, D, [5, 1], [5, 1], block)
        assert c.run().done() == 0
        for b, t in ((0, 0), (1, 5)):
            v = c.cache.rows(c.cache.v, b, 1)[1, 0]
            assert torch.equal(c.out[t], v.repeat_interleave(g, 0))


@pytest.mark.parametrize("D,block", [(128, 16), (64, 0), (256, 7), (128, 0)])
def test_chunk_rows_that_see_nothing(D, block):
    """More new tokens than slots: the first ones see no slot and get zeros; a sequence of no slots."""
    c = Chunk(2, 4, D, [9, 3, 140], [4, 0, 2], block)
    assert c.run().done() == 0
    assert bool((c.out[:5] == 0).all()) and bool((c.out[9:12] == 0).all()) and bool((c.out[12:150] == 0).all())
    c.check()
    c = Chunk(2, 4, D, [9, 3], [0, 0], block)  # max_len 0
    assert c.run().done() == 0
    assert bool((c.out[:12] == 0).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H,g,D,block,new", [(2, 4, 128, 16, [40, 150, 1]), (1, 8, 64, 0, [40, 150, 1]), (2, 2, 256, 7, [40, 150, 1]),
                                             (2, 4, 128, 16, [12, 20, 1]), (1, 8, 64, 0, [12, 20, 1])])
def test_chunk_hidden_slots_do_not_matter(H, g, D, block, new, bad):
    """Slots behind the length, and slots of later tokens, have no influence whatever they hold; queries that see them do
    get what the formula gives."""
    lens = [300, 150, 17]
    c = Chunk(H, g, D, new, lens, block, seed=2)
    for b, n in enumerate(lens):  # rows behind the length
        w = c.cache.where(b, np.arange(n, n + 3))
        c.cache.k[w], c.cache.v[w] = bad, bad
    hidden = {0: 300 - new[0] // 4, 1: 150 - new[1] // 3}  # a slot that later queries see
    for b, s in hidden.items():
        w = c.cache.where(b, [s])
        c.cache.v[w] = bad
    assert c.run().done() == 0
    at = 0
    for b, (n, length) in enumerate(zip(new, lens)):
        K, V = (U.f64(c.cache.rows(x, b, length)[1]) for x in (c.cache.k, c.cache.v))
        free = n if b not in hidden else hidden[b] - (length - n)
        i = np.arange(free)
        S = length if b not in hidden else hidden[b]
        ref, bar = U.chunk64(U.f64(c.q[at:at + free]), c.pos[at:at + free], K[:S], V[:S], U.causal(n, length, S)[i])
        got = U.f64(c.out[at:at + free])
        assert (np.abs(got - ref) <= bar).all()
        seeing = U.f64(c.out[at + free:at + n])
        assert not np.isfinite(seeing).any()
        at += n


@pytest.mark.parametrize("H,g,D,block", [(8, 4, 128, 16), (4, 8, 256, 16), (8, 8, 64, 0)])
def test_chunk_many_rows_with_bad_slots(H, g, D, block):
    """Whole units (many rows): a value that is not finite reaches the queries that see it and no others; an unmapped block
    is left out of every query's slots."""
    c = Chunk(H, g, D, [1900, 40], [1900, 300], block, seed=3)
    w = c.cache.where(0, [1500])
    c.cache.v[w] = float("nan")
    assert c.run().done() == 0
    got = U.f64(c.out[:1940])
    assert np.isfinite(got[:1500]).all() and np.isnan(got[1500:1900]).all() and np.isfinite(got[1900:]).all()
    i = np.unique(np.r_[0:5, 700:705, 1490:1500])
    K, V = (U.f64(c.cache.rows(x, 0, 1500)[1]) for x in (c.cache.k, c.cache.v))
    ref, bar = U.chunk64(U.f64(c.q[i]), c.pos[i], K, V, U.causal(1900, 1900, 1500)[i])
    assert (np.abs(got[i] - ref) <= bar).all()
    c.check(seqs=[1], rows=5)
    if block:
        c = Chunk(H, g, D, [1900, 40], [1900, 300], block, seed=4, unmapped=[(0, 100)])
        assert c.run().done() == prcr.ST_NO_BLOCK
        c.check(rows=12, drop=lambda b, s: (s // block == 100) if b == 0 else s < 0)


@pytest.mark.parametrize("H,g,D,block", [(2, 4, 128, 16), (1, 8, 256, 7), (2, 3, 64, 0)])
def test_chunk_a_bad_element_reaches_its_dim_alone(H, g, D, block):
    """A NaN in one dim of a value that all queries see, an infinity in another dim of one that the later ones see: the
    other dims, and this one before them, are what the formula gives without the two."""
    c = Chunk(H, g, D, [300], [340], block, seed=6)
    first, late = c.cache.where(0, [5]), c.cache.where(0, [200])  # the late one is query 160's own
    K, V = (U.f64(c.cache.rows(x, 0, 340)[1]) for x in (c.cache.k, c.cache.v))
    for w, d, bad in ((first, 3, float("nan")), (late, 17, float("inf"))):
        rows = c.cache.v[w]
        rows[..., d] = bad
        c.cache.v[w] = rows
    assert c.run().done() == 0
    got = U.f64(c.out[:300])
    ref, bar = U.chunk64(U.f64(c.q[:300]), c.pos[:300], K, V, U.causal(300, 340, 340))
    ok = np.abs(got - ref) <= bar
    assert np.isnan(got[..., 3]).all() and not np.isfinite(got[160:, :, 17]).any()
    ok[..., 3] = ok[160:, :, 17] = True
    assert ok.all()


def test_chunk_nan_key_reaches_those_that_see_it():
    c = Chunk(2, 4, 128, [100], [400], 16, seed=4)
    c.cache.k[c.cache.where(0, [350])] = float("nan")
    assert c.run().done() == 0
    out = U.f64(c.out[:100])
    assert np.isfinite(out[:50]).all() and np.isnan(out[50:]).all()
    c.new = [50]  # the first fifty see slots up to 349
    c.lens = [350]
    q, pos = U.f64(c.q[:50]), c.pos[:50]
    K, V = (U.f64(c.cache.rows(x, 0, 350)[1]) for x in (c.cache.k, c.cache.v))
    ref, bar = U.chunk64(q, pos, K, V, U.causal(100, 400, 350)[:50])
    assert (np.abs(out[:50] - ref) <= bar).all()


@pytest.mark.parametrize("scale", [0.0, 30.0, 1000.0])
def test_chunk_logits_of_any_size(scale):
    """Equal logits (a plain mean of the values) and logits so far apart that one slot takes all."""
    for D, new, lens in ((128, [60, 1], [500, 2000]), (64, [9], [300]), (256, [30], [200])):
        c = Chunk(2, 4, D, new, lens, 16, q_scale=scale, seed=8)
        assert c.run().done() == 0
        got = U.f64(c.out[:sum(new)])
        assert np.isfinite(got).all()
        if scale < 100:
            at = 0
            for b, (n, length) in enumerate(zip(new, lens)):
                K, V = (U.f64(c.cache.rows(x, b, length)[1]) for x in (c.cache.k, c.cache.v))
                ref, bar = U.chunk64(U.f64(c.q[at:at + n]), c.pos[at:at + n], K, V, U.causal(n, length, length))
                assert (np.abs(got[at:at + n] - ref) <= bar).all()
                at += n


def test_chunk_rising_maxima():
    """Keys that grow along the sequence: every tile raises the running maximum."""
    for D in (64, 128, 256):
        c = Chunk(1, 4, D, [20], [1500], 16, seed=12)
        grow = torch.linspace(0.1, 12.0, 1500, device=DEV).view(1, 1500, 1, 1)
        w = c.cache.where(0, np.arange(1500))
        c.cache.k[w] = (c.cache.k[w].float() * grow).bfloat16()
        assert c.run().done() == 0
        K, V = (U.f64(c.cache.rows(x, 0, 1500)[1]) for x in (c.cache.k, c.cache.v))
        ref, bar = U.chunk64(U.f64(c.q[:20]), c.pos[:20], K, V, U.causal(20, 1500, 1500))
        assert (np.abs(U.f64(c.out[:20]) - ref) <= bar).all()


def test_chunk_device_errors():
    """Unmapped blocks are left out, lengths beyond the capacity or max_len clamped, malformed offsets refused."""
    c = Chunk(2, 4, 128, [20, 3], [200, 90], 16, unmapped=[(0, 3), (0, 4), (1, 0)])
    assert c.run().done() == prcr.ST_NO_BLOCK
    c.check(drop=lambda b, s: np.isin(s // 16, [3, 4]) if b == 0 else s // 16 == 0)
    c = Chunk(2, 4, 128, [2], [16], 16, unmapped=[(0, 0)], caps=[16])  # no readable slot at all
    assert c.run().done() == prcr.ST_NO_BLOCK and bool((c.out[:2] == 0).all())
    # a length above max_len: queries see slots by their place behind the length, those past max_len are left out
    c = Chunk(2, 4, 64, [20, 3], [200, 90], 0)
    assert c.run(max_len=150).done() == prcr.ST_CAPACITY
    c.check(top=150)
    c = Chunk(2, 4, 64, [20, 3], [200, 90], 0)
    c.lens[0] = 260  # capacity 203
    assert c.run(max_len=203, seq_len=i32(c.lens)).done() == prcr.ST_CAPACITY
    c.check(top=203)
    c = Chunk(2, 4, 64, [20, 3], [200, 90], 0)
    assert c.run(seq_len=i32([-5, 90])).done() == prcr.ST_CAPACITY
    assert bool((c.out[:20] == 0).all())
    c.check(seqs=[1])
    for off in ([1, 20, 23], [0, 23, 20], [0, 20, 27], [0, -1, 23], [0, 2 ** 31 - 1, 23]):
        c = Chunk(2, 4, 64, [20, 3], [200, 90], 16)
        assert c.run(q_off=i32(off)).done() == prcr.ST_CSR
        assert bool((c.out_all == torch.tensor(U.CANARY, dtype=torch.bfloat16)).all())


def test_chunk_far_positions():
    """Angles of positions near the ends of int32."""
    c = Chunk(2, 4, 128, [12], [60], 16, seed=3)
    c.pos = np.random.default_rng(1).integers(-2 ** 31, 2 ** 31, c.pos.shape).astype(np.int32)
    c.args = (i32(c.pos),) + c.args[1:]
    assert c.run().done() == 0
    c.check()


def test_chunk_many_sequences():
    rng = np.random.default_rng(4)
    new = rng.integers(0, 4, 300)
    lens = new + rng.integers(0, 60, 300)
    c = Chunk(2, 2, 64, [int(x) for x in new], [int(x) for x in lens], 8, seed=6)
    assert c.run().done() == 0
    c.check()


def test_chunk_agrees_with_decode_attention():
    """A single new token per sequence is decode_attention's step (its output is float32)."""
    H, g, D = 8, 4, 128
    c = Chunk(H, g, D, [1, 1, 1], [500, 33, 1200], 16, L=1, layer=0, pad=0)
    c.pos[:] = c.pos[:, :1]
    c.args = (i32(c.pos),) + c.args[1:]
    assert c.run().done() == 0
    q = c.q.contiguous().view(3, 1, H * g, D)
    out = torch.empty(q.shape, dtype=torch.float32, device=DEV)
    ws = torch.empty(max(16, prcr.decode_workspace_size(c.cfg, 3, H * g, 1200)), dtype=torch.uint8, device=DEV)
    prcr.decode_attention(c.cfg, c.cache.desc(), q, torch.from_numpy(c.pos[:, 0].astype(np.int64)).to(DEV), c.args[2], 1200, out,
                          c.status, ws)
    assert c.done() == 0
    c.check()
    d = (c.out.float() - out[:, 0]).norm() / out.norm()
    assert float(d) <= NORM


def test_chunk_streams_and_graphs():
    """Two calls at once on two streams with a workspace each; one call captured and replayed with new contents."""
    a = Chunk(4, 4, 128, [3, 200], [3000, 900], 16, seed=1)
    b = Chunk(4, 4, 128, [3, 200], [2500, 1100], 16, seed=2)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        a.run(stream=s1)
        b.run(stream=s2)
    assert a.done() == 0 and b.done() == 0
    a.check(rows=20)
    b.check(rows=20)
    g, want = torch.cuda.CUDAGraph(), a.out.clone()
    with torch.cuda.graph(g):
        a.run()
    a.out.fill_(U.CANARY)
    a.ws.fill_(0xff)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, want)
    a.q.copy_(b.q)
    g.replay()
    torch.cuda.synchronize()
    a.check(rows=20)


def test_chunk_is_repeatable():
    c = Chunk(2, 7, 128, [5, 300], [9000, 700], 16, seed=1)
    c.run().done()
    want = c.out.clone()
    for _ in range(3):
        c.run()
    c.done()
    assert torch.equal(c.out, want)


# ----------------------------------------------------------------------------
# accumulated weights
# ----------------------------------------------------------------------------
def weights64(q, p, K, D, layout):
    """sum over the group of softmax weights [H, S] and a bound on their error: float32 dots and rotations move a logit by at
    most e = 2^-24 (D + 8) sum |q k| / sqrt(D), exp and the sums add 2^-20."""
    Hq, H = q.shape[0], K.shape[1]
    g = Hq // H
    qr = U.rope64(q[None], np.full((1, 3), float(p)), D, layout)[0]
    w, bar = np.zeros((H, K.shape[0])), np.zeros((H, K.shape[0]))
    for h in range(Hq):
        k = K[:, h // g]
        x = U.softmax64(k @ qr[h] / np.sqrt(D))
        e = 2.0 ** -24 * (D + 8) * (np.abs(k) @ np.abs(qr[h])).max() / np.sqrt(D)
        w[h // g] += x
        bar[h // g] += x * (np.expm1(2 * e) + 2.0 ** -20)
    return w, bar


class Weights:
    def __init__(self, H, g, D, L, lens, block, seed=0, layout=prcr.LAYOUT_SECTIONED, caps=None, extra=5, **cache):
        self.H, self.g, self.D, self.L, self.lens, self.layout = H, g, D, L, list(lens), layout
        B, rng = len(lens), np.random.default_rng(seed)
        self.cache = Cache(L, H, D, caps or [n + 3 for n in lens], block, seed=seed, **cache)
        self.cfg = U.cfg_of(L, H, D, layout)
        self.q = normal((B, L, H * g, D), seed + 3)
        self.pos = rng.integers(0, 60000, B)
        self.max_len = max(lens)
        self.score = torch.rand((B, L, H, self.max_len + extra), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
        self.before = self.score.cpu().numpy().astype(np.float64)
        self.status = status_word()

    def run(self, decay=1.0, max_len=None, seq_len=None, pos=None):
        m = self.max_len if max_len is None else max_len
        n = prcr.weights_workspace_size(self.cfg, len(self.lens), self.H * self.g, m)
        ws = torch.full((max(n, 16),), 0xff, dtype=torch.uint8, device=DEV)
        prcr.accumulate_weights(self.cfg, self.cache.desc(), self.q, torch.as_tensor(self.pos if pos is None else pos).to(DEV),
                                i32(self.lens) if seq_len is None else seq_len, m, self.score, self.status, decay, ws)
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, decay=1.0, drop=None, top=None, steps=1):
        got = self.score.cpu().numpy().astype(np.float64)
        for b, n in enumerate(self.lens):
            n = n if top is None else min(n, top)
            assert np.array_equal(got[b, :, :, n:], self.before[b, :, :, n:], equal_nan=True)
            for l in range(self.L):
                if not n:
                    continue
                K = U.f64(self.cache.rows(self.cache.k, b, n)[l])
                keep = np.ones(n, bool) if drop is None else ~drop(b, np.arange(n))
                w, bar = np.zeros((self.H, n)), np.zeros((self.H, n))
                if keep.any():
                    w[:, keep], bar[:, keep] = weights64(U.f64(self.q[b, l]), self.pos[b], K[keep], self.D, self.layout)
                old = 0.0 if decay == 0 else decay * self.before[b, l, :, :n]
                ref = old + w
                assert (np.abs(got[b, l, :, :n] - ref) <= bar + 2.0 ** -22 * (np.abs(old) + w) + 1e-37).all(), (b, l)


@pytest.mark.parametrize("H,g,D,L,lens,block", [
    (8, 4, 128, 2, [1, 0, 300], 16), (4, 7, 128, 1, [933, 17], 0), (2, 1, 64, 3, [129, 128], 7), (1, 8, 128, 2, [2500], 64),
    (2, 4, 256, 2, [65, 700], 16), (3, 8, 64, 1, [5000, 3], 0), (1, 1, 256, 1, [16, 15, 17, 1], 1), (2, 4, 128, 1, [40000], 16),
    (8, 4, 128, 36, [200], 16), (2, 3, 128, 1, [20000, 9], 16), (1, 8, 256, 1, [17000], 16),
    (1, 8, 64, 1, [60000, 31], 16),  # beyond a cluster's shared memory: through the workspace
    (1, 1, 64, 1, [2000, 100, 1], 0), (1, 2, 256, 1, [300, 1000], 7),  # few: a cluster of eight
], ids=lambda v: str(v))
def test_weights(H, g, D, L, lens, block):
    w = Weights(H, g, D, L, lens, block, seed=H + g, gap=8 if block == 7 else 0,
                layout=prcr.LAYOUT_INTERLEAVED if L == 3 else prcr.LAYOUT_SECTIONED)
    assert w.run() == 0
    w.check()


def test_weights_decay():
    w = Weights(2, 4, 128, 1, [300, 20], 16)
    w.score[0, :, :, :300] = float("nan")  # not read at decay 0
    w.before = w.score.cpu().numpy().astype(np.float64)
    assert w.run(decay=0.0) == 0
    w.check(decay=0.0)
    w = Weights(2, 4, 64, 2, [300, 20], 0)
    assert w.run(decay=0.75) == 0
    w.check(decay=0.75)


def test_weights_errors():
    w = Weights(2, 4, 128, 2, [100, 64], 16, unmapped=[(0, 2), (1, 0), (1, 1), (1, 2), (1, 3)], caps=[112, 64])
    assert w.run() == prcr.ST_NO_BLOCK
    w.check(drop=lambda b, s: s // 16 == 2 if b == 0 else s >= 0)
    w = Weights(2, 4, 128, 1, [100, 64], 16)
    assert w.run(max_len=70) == prcr.ST_CAPACITY
    w.check(top=70)
    w = Weights(2, 4, 64, 1, [100, 64], 0)
    assert w.run(seq_len=i32([-1, 64])) == prcr.ST_CAPACITY
    w.lens[0] = 0
    w.check()
    for p in (2 ** 31, -2 ** 31):
        w = Weights(2, 4, 256, 1, [100, 64], 16)
        assert w.run(pos=np.array([p, w.pos[1]])) == prcr.ST_POS_RANGE
        w.lens[0] = 0
        w.check()


def test_weights_hidden_slots_do_not_matter():
    w = Weights(2, 4, 128, 1, [100, 33], 16)
    for b, n in enumerate(w.lens):
        w.cache.k[w.cache.where(b, [n, n + 1])] = float("nan")
    w.cache.v[:] = float("nan")
    assert w.run() == 0
    w.check()


# ----------------------------------------------------------------------------
# eviction
# ----------------------------------------------------------------------------
class Evict:
    def __init__(self, H, D, L, lens, block, budget, sink, recent, in_place, seed=0, dst_block=None, caps=None, dst_caps=None, **cache):
        self.H, self.D, self.L, self.lens = H, D, L, list(lens)
        self.budget, self.sink, self.recent = budget, sink, recent
        B = len(lens)
        self.cfg = U.cfg_of(L, H, D)
        self.src = Cache(L, H, D, caps or [n + 2 for n in lens], block, seed=seed, **cache)
        self.dst = self.src if in_place else Cache(L, H, D, dst_caps or [budget] * B, block if dst_block is None else dst_block, fill=U.CANARY)
        self.in_place, self.max_len = in_place, max(lens)
        self.score = torch.rand((B, L, H, self.max_len + 4), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
        self.status = status_word()

    def run(self, max_len=None, seq_len=None, score_in_place=False):
        B = len(self.lens)
        self.k0, self.v0, self.s0 = self.src.k.clone(), self.src.v.clone(), self.score.cpu().numpy()
        self.dk0, self.dv0 = self.dst.k_all.clone(), self.dst.v_all.clone()
        self.keep = torch.full((B, self.L, self.H, self.budget), -99, dtype=torch.int32, device=DEV)
        self.len_out = torch.full((B,), -99, dtype=torch.int32, device=DEV)
        self.out = self.score if score_in_place else torch.full_like(self.score, U.CANARY)
        prcr.evict(self.cfg, self.src.desc(), i32(self.lens) if seq_len is None else seq_len, self.max_len if max_len is None else max_len,
                   self.budget, self.sink, self.recent, self.score, self.keep, self.len_out, self.status,
                   dst=None if self.in_place else self.dst.desc(), score_out=self.out)
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, broken=()):
        keep, out = self.keep.cpu().numpy(), self.out.cpu().numpy()
        want_k, want_v = self.dk0.clone(), self.dv0.clone()
        row = self.H * self.D
        wk, wv = (x[..., :row].unflatten(-1, (self.H, self.D)) for x in (want_k, want_v))
        for b, n in enumerate(self.lens):
            if b in broken:
                assert (keep[b] == -1).all() and int(self.len_out[b]) == (n if self.in_place else 0)
                assert np.array_equal(out[b], self.s0[b] if self.out is self.score else np.full_like(out[b], U.CANARY))
                continue
            m = min(n, self.budget)
            assert int(self.len_out[b]) == m
            for l in range(self.L):
                for h in range(self.H):
                    ref = U.evict64(self.s0[b, l, h], n, self.budget, self.sink, self.recent)
                    assert list(keep[b, l, h]) == ref + [-1] * (self.budget - m), (b, l, h)
                    s = np.zeros_like(out[b, l, h])
                    s[:m] = self.s0[b, l, h][ref]
                    assert np.array_equal(out[b, l, h], s, equal_nan=True)
            if m:
                idx = self.keep[b, :, :, :m].long()  # [L, H, m]
                for x0, w in ((self.k0, wk), (self.v0, wv)):
                    rows = x0[self.src.where(b, np.arange(n))]  # [L, n, H, D]
                    rows = rows.gather(1, idx.transpose(1, 2).unsqueeze(-1).expand(-1, -1, -1, self.D))
                    w[self.dst.where(b, np.arange(m))] = rows
        assert torch.equal(self.dst.k_all, want_k) and torch.equal(self.dst.v_all, want_v)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("H,D,L,lens,block,budget,sink,recent", [
    (8, 128, 2, [300, 64, 0, 65], 16, 64, 4, 16), (2, 64, 3, [700, 1], 0, 100, 0, 0), (1, 256, 1, [50], 7, 1, 0, 0),
    (3, 128, 2, [513, 512, 511], 1, 200, 100, 100), (2, 48, 1, [1000, 90], 32, 333, 7, 50), (1, 16, 1, [5000], 0, 4999, 2, 9),
    (4, 128, 28, [130, 40], 16, 33, 1, 0), (1, 128, 1, [40000], 16, 3001, 5, 700), (2, 128, 1, [2000], 16, 1, 0, 1),
], ids=lambda v: str(v))
def test_evict(H, D, L, lens, block, budget, sink, recent, in_place):
    e = Evict(H, D, L, lens, block, budget, sink, recent, in_place, seed=H + D, gap=8 if block == 32 else 0)
    assert e.run(score_in_place=in_place) == 0
    e.check()


@pytest.mark.parametrize("in_place", [True, False])
def test_evict_ties_and_odd_scores(in_place):
    """Equal scores, zeros of both signs, infinities and NaN."""
    e = Evict(2, 64, 2, [400, 300], 16, 120, 3, 10, in_place, seed=2)
    rng = np.random.default_rng(0)
    s = rng.choice([0.0, -0.0, 0.25, 0.5, np.inf, -np.inf, np.nan, -1.0, 1e-40, -1e-40], size=tuple(e.score.shape)).astype(np.float32)
    s[1] = 0.25  # all equal
    s[0, 1] = np.nan
    e.score.copy_(torch.from_numpy(s))
    assert e.run() == 0
    e.check()


def test_evict_into_another_kind_of_cache():
    e = Evict(2, 128, 2, [400, 90], 16, 120, 3, 10, False, dst_block=0)
    assert e.run() == 0
    e.check()
    e = Evict(2, 128, 2, [400, 90], 0, 120, 3, 10, False, dst_block=5)
    assert e.run() == 0
    e.check()


def test_evict_errors():
    """A sequence with a fault is left as it was, the others are cut."""
    for in_place in (True, False):
        e = Evict(2, 64, 2, [200, 150, 90], 16, 60, 2, 8, in_place, unmapped=[(1, 3)])
        assert e.run(score_in_place=in_place) == prcr.ST_NO_BLOCK
        e.check(broken=[1])
        e = Evict(2, 64, 2, [200, 150, 90], 0, 60, 2, 8, in_place)
        assert e.run(max_len=180, score_in_place=in_place) == prcr.ST_CAPACITY
        e.check(broken=[0])
        e = Evict(2, 64, 2, [200, 150, 90], 0, 60, 2, 8, in_place)
        e.lens[2] = -4
        assert e.run(seq_len=i32(e.lens)) == prcr.ST_CAPACITY
        e.check(broken=[2])
    e = Evict(2, 64, 2, [200, 150], 16, 60, 2, 8, False, dst_caps=[64, 48])  # the second's table has a fourth block unmapped
    assert e.run() == prcr.ST_NO_BLOCK
    e.check(broken=[1])
    e = Evict(2, 64, 2, [200, 150], 0, 60, 2, 8, False, dst_caps=[59, 59])
    assert e.run() == prcr.ST_CAPACITY
    e.check(broken=[0, 1])


# ----------------------------------------------------------------------------
# together
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("H,g,D,block", [(4, 4, 128, 16), (2, 7, 64, 0), (1, 8, 256, 7)])
def test_a_dialogue(H, g, D, block):
    """Prompts appended and attended over, decode steps with weights added up, an eviction, and more tokens over what is
    left: every attention against the 64-bit formula on rows that the test follows by itself."""
    L, prompts, steps, budget = 2, [90, 41], 3, 48
    B, Hq = len(prompts), H * g
    c = U.cfg_of(L, H, D)
    cache = Cache(L, H, D, [120, 120], block, fill=0.0)
    st = status_word()
    length, nxt = i32([0, 0]), [0, 0]
    rows = [[[[] for _ in range(H)] for _ in range(L)] for _ in range(B)]  # (key, value) of each slot, 64 bits
    score = torch.zeros((B, L, H, 120), device=DEV)
    ref_score = [[[[] for _ in range(H)] for _ in range(L)] for _ in range(B)]
    sizes = [prompts] + [[1, 1]] * steps + ["evict", [5, 1]]
    for turn, new in enumerate(sizes):
        if new == "evict":
            keep = torch.zeros((B, L, H, budget), dtype=torch.int32, device=DEV)
            out = torch.zeros_like(length)
            top = int(length.max())
            prcr.evict(c, cache.desc(), length, top, budget, 2, 6, score, keep, out, st)
            for b in range(B):
                n = int(length[b])
                for l in range(L):
                    for h in range(H):
                        got = [int(i) for i in keep[b, l, h] if i >= 0]
                        s = score_before = np.array(ref_score[b][l][h])
                        assert len(got) == min(n, budget) and got == sorted(set(got))
                        if n > budget:  # the kept ones are the best but for scores closer than float32 tells apart
                            free = [i for i in got if 2 <= i < n - 6]
                            lost = [i for i in range(2, n - 6) if i not in got]
                            assert set(range(2)) <= set(got) and set(range(n - 6, n)) <= set(got)
                            assert s[free].min() >= s[lost].max() * (1 - 1e-4)
                        rows[b][l][h] = [rows[b][l][h][i] for i in got]
                        ref_score[b][l][h] = [score_before[i] for i in got]
            length = out
            continue
        T, off = sum(new), U.offsets(new)
        pos = np.concatenate([positions(n, nxt[b], None) if n > 1 else np.full((1, 3), nxt[b]) for b, n in enumerate(new)]).astype(np.int32)
        for b, n in enumerate(new):
            nxt[b] += n + 12
        ks, vs = normal((L, T, H, D), 50 + turn), normal((L, T, H, D), 70 + turn)
        out_len = torch.zeros_like(length)
        prcr.append_kv(c, cache.desc(), 0, ks, vs, i32(pos), off, length, out_len, st)
        length = out_len
        kr = U.rope64(U.f64(ks), pos, D)
        at = 0
        for b, n in enumerate(new):
            for l in range(L):
                for h in range(H):
                    rows[b][l][h] += [(kr[l, at + i, h], U.f64(vs[l, at + i, h])) for i in range(n)]
                    ref_score[b][l][h] += [0.0] * n
            at += n
        top = int(length.max())
        q = normal((L, T, Hq, D), 90 + turn)
        out = torch.zeros((L, T, Hq, D), dtype=torch.bfloat16, device=DEV)
        for l in range(L):
            ws = torch.empty(max(16, prcr.chunk_workspace_size(c, B, Hq, T, top)), dtype=torch.uint8, device=DEV)
            prcr.chunk_attention(c, cache.desc(), l, q[l], i32(pos), off, length, top, out[l], st, ws)
        if turn:  # a decode step: its weights too
            ql = torch.stack([q[:, int(off[b + 1]) - 1] for b in range(B)])
            p = torch.tensor([int(pos[int(off[b + 1]) - 1, 0]) for b in range(B)], device=DEV)
            ws = torch.empty(prcr.weights_workspace_size(c, B, Hq, top), dtype=torch.uint8, device=DEV)
            prcr.accumulate_weights(c, cache.desc(), ql.contiguous(), p, length, top, score, st, 1.0, ws)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        at = 0
        for b, n in enumerate(new):
            for l in range(L):
                # the cache's keys are the rotated ones rounded to bf16
                K = np.stack([np.stack([r[0] for r in rows[b][l][h]]) for h in range(H)], 1)
                K = U.f64(torch.from_numpy(K).float().bfloat16())
                V = np.stack([np.stack([r[1] for r in rows[b][l][h]]) for h in range(H)], 1)
                S = K.shape[0]
                assert S == int(length[b])
                ref, bar = U.chunk64(U.f64(q[l, at:at + n]), pos[at:at + n], K, V, U.causal(n, S, S))
                d = np.abs(U.f64(out[l, at:at + n]) - ref)
                assert (d <= bar).all(), (turn, b, l, (d / bar).max())
                if turn:
                    w, _ = weights64(U.f64(ql[b, l]), int(p[b]), K, D, prcr.LAYOUT_SECTIONED)
                    for h in range(H):
                        ref_score[b][l][h] = list(np.array(ref_score[b][l][h]) + w[h])
            at += n


def test_the_calls_in_one_graph_and_on_two_streams():
    """Append, attention, weights and eviction of one step, captured together and replayed over a cache set back, beside a
    second batch's on another stream: the results of the same calls made one after the other."""
    L, H, g, D, B, block, budget = 2, 4, 4, 128, 3, 16, 70
    c = U.cfg_of(L, H, D)

    class Step:
        def __init__(self, seed):
            self.cache, self.lens, self.new = Cache(L, H, D, [400, 90, 130], block, seed=seed), i32([390, 60, 70]), [1, 5, 30]
            self.T, self.top = sum(self.new), 400
            self.ks, self.vs = normal((L, self.T, H, D), seed + 1), normal((L, self.T, H, D), seed + 2)
            self.q, self.qw = normal((L, self.T, H * g, D), seed + 3), normal((B, L, H * g, D), seed + 4)
            self.pos, self.off = i32(positions(self.T, 9, None)), U.offsets(self.new)
            self.p = torch.tensor([500, 600, 700], device=DEV)
            self.k0, self.v0 = self.cache.k_all.clone(), self.cache.v_all.clone()
            self.len1, self.len2, self.status = i32([0] * B), i32([0] * B), status_word()
            self.out, self.score = torch.zeros_like(self.q), torch.zeros((B, L, H, 400), device=DEV)
            self.keep = i32(np.zeros((B, L, H, budget)))
            n = max(prcr.chunk_workspace_size(c, B, H * g, self.T, self.top), prcr.weights_workspace_size(c, B, H * g, self.top))
            self.ws = torch.zeros(n + 16, dtype=torch.uint8, device=DEV)

        def reset(self):
            for x, x0 in ((self.cache.k_all, self.k0), (self.cache.v_all, self.v0)):
                x.copy_(x0)
            for x in (self.out, self.score, self.keep, self.len1, self.len2):
                x.zero_()
            self.ws.fill_(0xff)

        def calls(self, stream=None):
            d = self.cache.desc()
            prcr.append_kv(c, d, 0, self.ks, self.vs, self.pos, self.off, self.lens, self.len1, self.status, stream=stream)
            for l in range(L):
                prcr.chunk_attention(c, d, l, self.q[l], self.pos, self.off, self.len1, self.top, self.out[l], self.status, self.ws, stream=stream)
            prcr.accumulate_weights(c, d, self.qw, self.p, self.len1, self.top, self.score, self.status, 1.0, self.ws, stream=stream)
            prcr.evict(c, d, self.len1, self.top, budget, 4, 16, self.score, self.keep, self.len2, self.status, stream=stream)

        def results(self):
            torch.cuda.synchronize()
            assert int(self.status.item()) == 0
            return [x.clone() for x in (self.out, self.score, self.keep, self.len1, self.len2, self.cache.k_all, self.cache.v_all)]

    a, b = Step(10), Step(30)
    want = []
    for x in (a, b):
        x.calls()
        want.append(x.results())
        assert list(x.len1) == [391, 65, 100] and list(x.len2) == [70, 65, 70]
        assert bool((x.out != 0).any()) and not torch.equal(x.cache.k_all, x.k0)
    graphs = []
    for x in (a, b):
        x.reset()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.calls()
    side = torch.cuda.Stream()
    for how in ("graph", "stream"):
        for x in (a, b):
            x.reset()
        torch.cuda.synchronize()
        if how == "graph":
            graphs[0].replay()
            with torch.cuda.stream(side):
                graphs[1].replay()
        else:
            a.calls()
            b.calls(stream=side)
        for x, w in zip((a, b), want):
            for got, ref in zip(x.results(), w):
                assert torch.equal(got, ref), how


def test_evict_of_more_scores_than_shared_memory_holds():
    for in_place in (True, False):
        e = Evict(1, 16, 1, [60000, 49153], 16, 20000, 5, 700, in_place, seed=4)
        assert e.run(score_in_place=in_place) == 0
        e.check()


def test_one_token_of_any_stride():
    """A dimension of one entry is read as packed, whatever its stride says."""
    x = Chunk(4, 2, 64, [1], [50], 16, seed=3, pad=0)
    x.run()
    assert x.done() == 0
    x.check()
    want = x.out.clone()
    x.q = x.q.transpose(0, 1).contiguous().transpose(0, 1)  # strides (D, D, 1)
    x.out = torch.zeros((8, 1, 64), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    x.run()
    assert x.done() == 0 and torch.equal(x.out, want)


def test_a_workspace_for_the_largest_call_serves_the_others():
    """One workspace for the longest and fullest call, dirty from the others, in calls of fewer sequences, tokens and slots."""
    H, g, D, B, T, longest = 2, 4, 128, 3, 600, 9000
    c = U.cfg_of(2, H, D)
    most = prcr.chunk_workspace_size(c, B, H * g, T, longest)
    assert most > 0
    sizes = [prcr.chunk_workspace_size(c, b, H * g, t, n) for b, t, n in ((1, 1, 1), (1, 1, 300), (1, 60, 300), (3, 60, 300), (3, 60, 9000), (3, 599, 9000))]
    assert sizes == sorted(sizes) and sizes[-1] <= most and sizes[0] == 0
    ws = torch.full((most,), 0xff, dtype=torch.uint8, device=DEV)
    for new, lens in (([9, 500, 1], [9000, 4000, 77]), ([1, 0, 2], [300, 5, 129]), ([64], [9000]), ([30, 5, 5], [128, 2000, 5]),
                      ([1, 1, 1], [1, 1, 1]), ([1], [9000]), ([590], [7000]), ([3, 40], [8999, 60])):
        x = Chunk(H, g, D, new, lens, 16, seed=sum(new))
        x.ws = ws
        x.run()
        assert x.done() == 0
        x.check(rows=40)


@pytest.mark.parametrize("H,g,D,new,lens", [(8, 4, 128, [6] * 16, [8198 - 300 * i for i in range(16)]), (2, 8, 64, [1], [2000]),
                                            (4, 2, 64, [3] * 40, [700] * 40), (4, 8, 256, [90, 200], [2500, 3000])], ids=str)
def test_chunk_calls_in_a_row_beside_copies(H, g, D, new, lens):
    """The kernels with two S buffers, whose warps run a tile ahead of the products, hundreds of times while another stream
    keeps the memory busy: no wait runs out, and every call gives the same."""
    c = Chunk(H, g, D, new, lens, 16, seed=7)
    assert c.run().done() == 0
    c.check(rows=9)
    want, side = c.out.clone(), torch.cuda.Stream()
    a, b = (torch.empty(1 << 28, dtype=torch.uint8, device=DEV) for _ in range(2))
    for turn in range(10):
        c.out.fill_(U.CANARY)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(8):
                b.copy_(a)
        for _ in range(40):
            c.run()
        assert c.done() == 0
        assert torch.equal(c.out[:sum(new)], want[:sum(new)])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H,g,D,block,new,lens,slot", [
    (2, 4, 128, 16, [9, 3], [4, 3], 2), (1, 8, 64, 0, [50, 30], [37, 30], 20), (2, 2, 256, 7, [70, 1], [60, 1], 59),
    (2, 4, 128, 0, [300, 20], [230, 20], 100), (4, 2, 64, 16, [700, 3], [650, 3], 0),
    (1, 1, 128, 16, [1710], [1700], 1600),  # the slots in parts
], ids=str)
def test_chunk_rows_that_see_nothing_beside_bad_values(H, g, D, block, new, lens, slot, bad):
    """More new tokens than slots, and a value that is not finite in one of these: zeros for the queries that see no slot,
    the formula's for those that do not see this one."""
    c = Chunk(H, g, D, new, lens, block, seed=13)
    c.cache.v[c.cache.where(0, [slot])] = bad
    assert c.run().done() == 0
    out, none = U.f64(c.out[:new[0]]), new[0] - lens[0]
    assert (out[:none] == 0).all()
    i = np.unique(np.linspace(none, none + slot - 1, 20).astype(int)) if slot else np.arange(0)
    K, V = (U.f64(c.cache.rows(x, 0, lens[0])[1]) for x in (c.cache.k, c.cache.v))
    V[slot] = 0.0
    ref, bar = U.chunk64(U.f64(c.q)[i], c.pos[i], K, V, U.causal(new[0], lens[0], lens[0])[i])
    assert (np.abs(out[i] - ref) <= bar).all()
    assert not np.isfinite(out[none + slot:]).any()
    c.check(seqs=[1])


@pytest.mark.parametrize("H,g,D,lens,block", [(2, 4, 128, [300, 40], 16), (1, 8, 64, [60000], 16), (1, 1, 256, [700, 9], 0), (3, 2, 64, [129], 7)], ids=str)
@pytest.mark.parametrize("moved", [False, True])
def test_weights_infinite_keys(H, g, D, lens, block, moved):
    """A key whose logit is minus infinity gets weight 0 and the others theirs as without it, in a cluster and through the
    workspace (60,000 slots); one of plus infinity or NaN makes that KV head's weights NaN, as the formula does."""
    w = Weights(H, g, D, 2, lens, block, seed=g)
    at, d = 7, 5
    if moved:  # heads of one sign in that dim, at positions that rotate
        w.q[:] = w.q[:, :, ::g].repeat_interleave(g, 2)
        qr = np.stack([U.rope64(U.f64(w.q[b])[:, ::g], np.full((2, 3), float(w.pos[b])), D, w.layout) for b in range(len(lens))])
        sign = np.sign(qr[..., d])
    else:
        w.pos[:] = 0
        w.q[..., d] = w.q[..., d].abs() + 0.01
        sign = np.ones((len(lens), 2, H))
    for b in range(len(lens)):
        where = w.cache.where(b, [at])
        rows = w.cache.k[where]
        rows[:, 0, :, d] = torch.from_numpy(-np.inf * sign[b]).to(DEV).bfloat16()
        w.cache.k[where] = rows
    assert w.run() == 0
    finite = w.cache.k.clone()
    for b in range(len(lens)):
        w.cache.k[w.cache.where(b, [at])] = 0.0
    w.check(drop=lambda b, s: s == at)
    w.cache.k.copy_(finite)
    for bad in (float("inf"), float("nan")):  # in head 0 alone
        where = w.cache.where(0, [at])
        rows = w.cache.k[where]
        for l in range(2):
            rows[l, 0, 0, d] = bad * sign[0, l, 0]
        w.cache.k[where] = rows
        w.score.copy_(torch.from_numpy(w.before))
        assert w.run() == 0
        got = w.score.cpu().numpy()
        assert np.isnan(got[0, :, 0, :lens[0]]).all() and np.isfinite(got[0, :, 1:]).all() and np.isfinite(got[1:]).all()


# ----------------------------------------------------------------------------
# chunk attention at position 0, where the queries are exact (cache_ops_util.chunk64_exact)
# ----------------------------------------------------------------------------
EXACT = [  # H, g, D, block, new, lens: few rows, many, in parts, head_dim 64 and 256
    (2, 4, 128, 16, [40, 1], [500, 2000]), (2, 4, 128, 0, [350, 20], [700, 300]), (1, 8, 64, 0, [9, 3], [300, 1500]), (4, 2, 64, 16, [600], [640]),
    (2, 4, 256, 7, [30, 1], [200, 900]), (2, 4, 256, 0, [300], [420]), (2, 7, 128, 16, [5], [9000]), (1, 4, 128, 16, [600], [4000]),
]


class Exact(Chunk):
    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.pos[:] = 0
        self.args = (i32(self.pos),) + self.args[1:]

    def check(self, rows=24, upto=None, slots=None):
        """Queries of each sequence (those below upto[b], over slots[b] slots) against the reference, over the finite rows."""
        at = 0
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            free = n if upto is None else upto[b]
            i = np.unique(np.linspace(0, max(free - 1, 0), min(rows, max(free, 1))).astype(int))
            S = length if slots is None else slots[b]
            if free > 0:
                K, V = (U.f64(self.cache.rows(x, b, S)[self.layer]) for x in (self.cache.k, self.cache.v))
                U.assert_close(U.f64(self.out)[at + i], *U.chunk64_exact(U.f64(self.q)[at + i], K, V, U.causal(n, length, S)[i]))
            at += n


@pytest.mark.parametrize("scale", [0.0, 1.0, 30.0, 1000.0])
@pytest.mark.parametrize("H,g,D,block,new,lens", EXACT, ids=str)
def test_chunk_exact_logits_of_any_size(H, g, D, block, new, lens, scale):
    """From equal logits to some so far apart that one slot takes all."""
    c = Exact(H, g, D, new, lens, block, q_scale=scale, seed=8)
    assert c.run().done() == 0
    c.check()


@pytest.mark.parametrize("H,g,D,block,new,lens", EXACT, ids=str)
@pytest.mark.parametrize("how", ["rising", "falling", "one tile"])
def test_chunk_exact_maxima(H, g, D, block, new, lens, how):
    """Keys that grow along the sequence (every tile raises the running maximum), that shrink (none does), and that are large in
    one late tile alone."""
    c = Exact(H, g, D, new, lens, block, seed=12)
    for b, n in enumerate(lens):
        f = torch.linspace(0.1, 12.0, n, device=DEV)
        f = f.flip(0) if how == "falling" else f
        if how == "one tile":
            f = torch.where((torch.arange(n, device=DEV) // 128) == (n * 2 // 3) // 128, 20.0, 0.5)
        w = c.cache.where(b, np.arange(n))
        x = c.cache.k[w].float()
        c.cache.k[w] = (x * f.view((1, n, 1, 1) if x.dim() == 4 else (n, 1, 1))).bfloat16()
    assert c.run().done() == 0
    c.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H,g,D,block,new,lens", EXACT, ids=str)
def test_chunk_exact_beside_bad_slots(H, g, D, block, new, lens, bad):
    """Values that are not finite behind the lengths and in a slot that only later queries see: those before it get what the
    formula gives without it."""
    c = Exact(H, g, D, new, lens, block, seed=2)
    upto, slots = [], []
    for b, (n, length) in enumerate(zip(new, lens)):
        w = c.cache.where(b, np.arange(length, length + 3))
        c.cache.k[w], c.cache.v[w] = bad, bad
        s = length - (n + 1) // 2
        c.cache.v[c.cache.where(b, [s])] = bad
        upto.append(n - (length - s))
        slots.append(s)
    assert c.run().done() == 0
    c.check(upto=upto, slots=slots)
    at = 0
    for n, free in zip(new, upto):
        assert not np.isfinite(U.f64(c.out)[at + free:at + n]).any()
        at += n


@pytest.mark.parametrize("H,g,D,block,new,lens", EXACT, ids=str)
def test_chunk_exact_beside_nan_keys(H, g, D, block, new, lens):
    c = Exact(H, g, D, new, lens, block, seed=4)
    upto, slots = [], []
    for b, (n, length) in enumerate(zip(new, lens)):
        s = length - (n + 1) // 2
        c.cache.k[c.cache.where(b, [s])] = float("nan")
        upto.append(n - (length - s))
        slots.append(s)
    assert c.run().done() == 0
    c.check(upto=upto, slots=slots)
    at = 0
    for n, free in zip(new, upto):
        assert np.isnan(U.f64(c.out)[at + free:at + n]).all()
        at += n


def test_layer_by_layer_as_a_decoder_runs():
    """Each layer's rows appended and attended over before the next layer's exist, through two prompts, tokens, an eviction in
    place and tokens behind it: each attention against the 64-bit formula on the rows that the cache holds."""
    L, H, g, D, block, budget = 3, 4, 4, 128, 16, 60
    c, st = U.cfg_of(L, H, D), status_word()
    cache = Cache(L, H, D, [160, 160], block, fill=0.0)
    length = i32([0, 0])
    top, turn = 160, 0
    ws = torch.empty(max(16, prcr.chunk_workspace_size(c, 2, H * g, 140, top)), dtype=torch.uint8, device=DEV)
    for new in ([90, 50], [1, 1], [6, 3], "evict", [1, 1], [5, 40]):
        if new == "evict":
            score = torch.rand((2, L, H, top), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
            keep, cut = i32(np.zeros((2, L, H, budget))), i32([0, 0])
            prcr.evict(c, cache.desc(), length, top, budget, 4, 16, score, keep, cut, st)
            length = cut
            continue
        turn += 1
        T, off, after = sum(new), U.offsets(new), i32([0, 0])
        pos = np.concatenate([positions(n, 200 * turn, None) for n in new]).astype(np.int32)
        for l in range(L):
            k, v, q = normal((1, T, H, D), 10 * turn + l), normal((1, T, H, D), 100 * turn + l), normal((T, H * g, D), 1000 * turn + l)
            out = torch.empty_like(q)
            prcr.append_kv(c, cache.desc(), l, k, v, i32(pos), off, length, after, st)
            prcr.chunk_attention(c, cache.desc(), l, q, i32(pos), off, after, top, out, st, ws)
            torch.cuda.synchronize()
            assert int(st.item()) == 0
            at = 0
            for b, n in enumerate(new):
                S = int(after[b])
                K, V = (U.f64(cache.rows(x, b, S)[l]) for x in (cache.k, cache.v))
                assert torch.equal(cache.rows(cache.v, b, S)[l, S - n:], v[0, at:at + n])
                ref, bar = U.chunk64(U.f64(q[at:at + n]), pos[at:at + n], K, V, U.causal(n, S, S))
                d = np.abs(U.f64(out[at:at + n]) - ref)
                assert (d <= bar).all() and np.sqrt((d ** 2).sum() / (ref ** 2).sum()) <= NORM
                at += n
        assert [int(x) for x in after] == [int(x) + n for x, n in zip(length, new)]
        length = after


@pytest.mark.parametrize("H,g,D,block,new,lens", [
    (8, 4, 128, 16, [2600], [2600]), (8, 4, 128, 64, [300, 2300], [5000, 2300]), (4, 7, 128, 0, [900, 0, 1, 333], [900, 5, 4000, 1333]),
    (2, 8, 256, 16, [1000, 400], [1300, 400]), (8, 2, 64, 7, [1500, 20], [1500, 3000]), (8, 4, 128, 16, [6, 1, 0, 5] * 4, [8198, 2193, 20, 4100] * 4),
    (4, 4, 64, 0, [40, 3], [9000, 4100]), (2, 1, 256, 16, [7], [20000]),
], ids=str)
def test_chunk_every_row_of_long_calls(H, g, D, block, new, lens):
    """Every element of long calls, at position 0, against chunk64_exact's formula and bound (in float64 on the GPU)."""
    c = Exact(H, g, D, new, lens, block, seed=21)
    assert c.run().done() == 0
    at = 0
    for b, (n, S) in enumerate(zip(new, lens)):
        sees = torch.from_numpy(U.causal(n, S, S)).to(DEV)
        for h in range(H * g if n else 0):
            K, V = (c.cache.rows(x, b, S)[c.layer, :, h // g].double() for x in (c.cache.k, c.cache.v))
            q, got = c.q[at:at + n, h].double(), c.out[at:at + n, h].double()
            w = torch.softmax((q @ K.T / D ** 0.5).masked_fill(~sees, float("-inf")), 1)
            e = (D * 2.0 ** -23 * (q.abs() @ K.abs().T) / D ** 0.5).masked_fill(~sees, 0.0).amax(1, keepdim=True)
            ref = w @ V
            bar = (2.0 ** -8 * ref.abs() + (2.0 ** -8 * w + torch.expm1(2 * e) * torch.minimum(w, 1 - w)) @ V.abs()) * 1.001 + 1e-30
            d = (got - ref).abs()
            assert bool((d <= bar).all()), (b, h, float((d / bar).max()))
            assert float(d.norm()) <= 2 * U.EXACT_NORM * float(ref.norm())  # (few elements in a short one: less of a mean)
        at += n

"""CPU checks of append_kv, chunk_attention, accumulate_weights and evict: what the
host refuses, before any CUDA call (the addresses below are never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

import cache_ops_util as U
import paper_2606_26631_gb300 as prcr
from paper_2606_26631_gb300 import _binding as B

FAKE = 1 << 40


def _cfg(D=64, H=2, L=2):
    return prcr.rope_cfg(L, H, D, (D // 2, 0, 0))


def _flat(**o):
    return B.CacheDesc(**{**dict(kind=0, block_size=1, k=FAKE, v=FAKE + 2 ** 20, seq_stride=2 * 256 * 128, layer_stride=256 * 128, block_stride=0,
                                 slot_stride=128, block_table=None, bt_stride=0, n_blocks=0, max_slots=256, n_seqs=3), **o})


def _paged(**o):
    return B.CacheDesc(**{**dict(kind=1, block_size=16, k=FAKE, v=FAKE + 2 ** 20, seq_stride=0, layer_stride=2048 * 64, block_stride=2048,
                                 slot_stride=128, block_table=FAKE, bt_stride=16, n_blocks=64, max_slots=0, n_seqs=3), **o})


APPEND = dict(cfg=_cfg(), cache=_flat(), n_seqs=3, l0=0, nl=2, k=FAKE, v=FAKE, ls=40 * 128, ts=128, coords=FAKE, off=FAKE, total=40,
              len_in=FAKE, len_out=FAKE + 64, status=FAKE)
CHUNK = dict(cfg=_cfg(), cache=_flat(), n_seqs=3, layer=0, hq=8, q=FAKE, qs=512, coords=FAKE, off=FAKE, total=40, len=FAKE, max_len=200,
             out=FAKE + 2 ** 20, os=512, status=FAKE, ws=FAKE, ws_bytes=1 << 40)
WEIGHTS = dict(cfg=_cfg(), cache=_flat(), n_seqs=3, hq=8, q=FAKE, pos=FAKE, len=FAKE, max_len=200, score=FAKE, ss=200, decay=1.0, status=FAKE,
               ws=FAKE, ws_bytes=1 << 40)
EVICT = dict(cfg=_cfg(), cache=_flat(), dst=None, n_seqs=3, len=FAKE, max_len=200, budget=50, sink=4, recent=10, score=FAKE, score_out=FAKE,
             ss=200, keep=FAKE, len_out=FAKE + 64, status=FAKE)
ENTRY = {"prcr_append_kv": APPEND, "prcr_chunk_attention": CHUNK, "prcr_accumulate_weights": WEIGHTS, "prcr_evict": EVICT}


def call(name, **over):
    a = {**ENTRY[name], **over}
    args = [C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()]
    return getattr(prcr.lib(), name)(*args, None)


COMMON = [
    (dict(cfg=_cfg(D=40)), B.EINVAL), (dict(cfg=None), B.EINVAL), (dict(cache=None), B.EINVAL), (dict(n_seqs=-1), B.EINVAL),
    (dict(n_seqs=4), B.EINVAL), (dict(cache=_flat(k=None)), B.EINVAL), (dict(cache=_flat(v=FAKE + 8)), B.EALIGN),
    (dict(cache=_flat(slot_stride=64)), B.EINVAL), (dict(cache=_paged(block_table=None)), B.EINVAL),
    (dict(cache=_paged(block_size=0)), B.EINVAL), (dict(status=None), B.EINVAL), (dict(status=FAKE + 2), B.EALIGN),
]
BAD = {
    "prcr_append_kv": [
        (dict(l0=-1), B.EINVAL), (dict(l0=1), B.EINVAL), (dict(nl=0), B.EINVAL), (dict(total=-1), B.EINVAL), (dict(k=None), B.EINVAL),
        (dict(v=None), B.EINVAL), (dict(ts=64), B.EINVAL), (dict(ls=-8), B.EINVAL), (dict(coords=None), B.EINVAL), (dict(off=None), B.EINVAL),
        (dict(len_in=None), B.EINVAL), (dict(len_out=None), B.EINVAL), (dict(len_out=FAKE), B.EINVAL), (dict(len_out=FAKE + 8), B.EINVAL), (dict(len_in=FAKE + 72), B.EINVAL), (dict(k=FAKE + 8), B.EALIGN),
        (dict(ts=132), B.EALIGN), (dict(ls=4), B.EALIGN), (dict(off=FAKE + 2), B.EALIGN), (dict(coords=FAKE + 1), B.EALIGN)],
    "prcr_chunk_attention": [
        (dict(cfg=_cfg(D=96)), B.EINVAL), (dict(hq=9), B.EINVAL), (dict(hq=1), B.EINVAL), (dict(hq=18), B.EINVAL), (dict(layer=-1), B.EINVAL),
        (dict(layer=2), B.EINVAL), (dict(total=-1), B.EINVAL), (dict(max_len=-1), B.EINVAL), (dict(max_len=257), B.EINVAL),
        (dict(cache=_paged(bt_stride=2 ** 30), max_len=2 ** 30 + 1), B.EINVAL), (dict(q=None), B.EINVAL), (dict(out=None), B.EINVAL),
        (dict(qs=504), B.EINVAL), (dict(os=504), B.EINVAL), (dict(coords=None), B.EINVAL), (dict(off=None), B.EINVAL), (dict(len=None), B.EINVAL),
        (dict(q=FAKE + 8), B.EALIGN), (dict(out=FAKE + 8), B.EALIGN), (dict(qs=516), B.EALIGN), (dict(os=516), B.EALIGN),
        (dict(out=FAKE, q=FAKE), B.EINVAL), (dict(len=FAKE + 2), B.EALIGN), (dict(cfg=_cfg(D=256, H=8), cache=_flat(slot_stride=2048), hq=64), B.EINVAL)],
    "prcr_accumulate_weights": [
        (dict(cfg=_cfg(D=96)), B.EINVAL), (dict(hq=9), B.EINVAL), (dict(max_len=257), B.EINVAL), (dict(ss=199), B.EINVAL),
        (dict(decay=float("nan")), B.EINVAL), (dict(decay=float("inf")), B.EINVAL), (dict(q=None), B.EINVAL), (dict(pos=None), B.EINVAL),
        (dict(score=None), B.EINVAL), (dict(q=FAKE + 4), B.EALIGN), (dict(pos=FAKE + 4), B.EALIGN), (dict(score=FAKE + 2), B.EALIGN)],
    "prcr_evict": [
        (dict(max_len=257), B.EINVAL), (dict(ss=199), B.EINVAL), (dict(budget=0), B.EINVAL), (dict(sink=-1), B.EINVAL),
        (dict(recent=-1), B.EINVAL), (dict(sink=41), B.EINVAL), (dict(score=None), B.EINVAL), (dict(score_out=None), B.EINVAL),
        (dict(keep=None), B.EINVAL), (dict(len=None), B.EINVAL), (dict(len_out=FAKE), B.EINVAL), (dict(len_out=FAKE + 4), B.EINVAL), (dict(keep=FAKE + 2), B.EALIGN),
        (dict(dst=_flat()), B.EINVAL), (dict(cache=_paged(), dst=_paged()), B.EINVAL), (dict(cache=_paged(), dst=_paged(k=FAKE + 2 ** 22)), B.EINVAL), (dict(dst=_flat(k=FAKE + 2 ** 22, v=FAKE + 2 ** 23, n_seqs=2)), B.EINVAL),
        (dict(dst=_flat(k=FAKE + 8)), B.EALIGN), (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), B.EINVAL)],
}


@pytest.mark.parametrize("name,over,code", [(n, o, c) for n in ENTRY for o, c in COMMON + BAD[n]],
                         ids=lambda v: ",".join(v) if isinstance(v, dict) else str(v))
def test_refusals(name, over, code):
    assert call(name, **over) == code


def test_empty_calls():
    for name in ENTRY:
        assert call(name, n_seqs=0) == B.OK
    assert call("prcr_chunk_attention", total=0) == B.OK
    assert call("prcr_accumulate_weights", max_len=0) == B.OK


def test_workspaces():
    c = _cfg(D=128, H=8, L=36)
    assert prcr.weights_workspace_size(_cfg(D=96), 1, 8, 100) == 0
    assert prcr.chunk_workspace_size(_cfg(D=96), 1, 8, 100, 100) == 0
    need = prcr.weights_workspace_size(c, 3, 32, 1000)
    cache = _flat(slot_stride=1024, layer_stride=256 * 1024, max_slots=1000)
    if need:
        assert call("prcr_accumulate_weights", cfg=c, cache=cache, hq=32, max_len=1000, ss=1000, ws_bytes=need - 1) == B.EWORKSPACE
        assert call("prcr_accumulate_weights", cfg=c, cache=cache, hq=32, max_len=1000, ss=1000, ws=None) == B.EWORKSPACE
        assert call("prcr_accumulate_weights", cfg=c, cache=cache, hq=32, max_len=1000, ss=1000, ws=FAKE + 8) == B.EALIGN


def _t(shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses():
    """Wrong types, shapes and layouts raise before the library is called; so do tensors that are not on the current GPU."""
    c, i32 = _cfg(), torch.int32
    cache = prcr.cache_contiguous(_t((3, 2, 9, 2, 64)), _t((3, 2, 9, 2, 64)))
    off, ln, st = _t(4, i32), _t(3, i32), _t(1, i32)
    rows = _t((2, 5, 2, 64))
    q, out, pos = _t((5, 8, 64)), _t((5, 8, 64)), _t((5, 3), i32)
    score, keep = _t((3, 2, 2, 9), torch.float32), _t((3, 2, 2, 4), i32)
    qw, p = _t((3, 2, 8, 64)), _t(3, torch.int64)
    good = {
        "append_kv": [c, cache, 0, rows, rows, pos, off, ln, ln.clone(), st],
        "chunk_attention": [c, cache, 0, q, pos, off, ln, 9, out, st],
        "accumulate_weights": [c, cache, qw, p, ln, 9, score, st],
        "evict": [c, cache, ln, 9, 4, 1, 1, score, keep, ln.clone(), st],
    }
    for name, args in good.items():
        with pytest.raises(ValueError, match="CUDA device"):
            getattr(prcr, name)(*args)
    wrong = {
        "append_kv": {3: [rows.float(), rows[:, :, :1], rows.transpose(2, 3)], 4: [rows[:, :4]], 5: [pos.long(), pos[:4]], 6: [off[:3], off.long()],
                      8: [ln[:2]]},
        "chunk_attention": {3: [q.float(), q[:, :, :32], q.transpose(0, 1)], 4: [pos[:2], pos.float()], 5: [off[:2]], 8: [out[:4], out.float()]},
        "accumulate_weights": {2: [qw.float(), qw[:, :1], qw.transpose(1, 2)], 3: [p.int(), p[:2]], 6: [score.double(), score[:2], score[..., :5]]},
        "evict": {7: [score.half(), score[:, :1]], 8: [keep[:2], keep.float()], 9: [ln[:1]], 2: [ln.long()]},
    }
    for name, at in wrong.items():
        for i, values in at.items():
            for v in values:
                with pytest.raises((TypeError, ValueError)) as e:
                    getattr(prcr, name)(*good[name][:i], v, *good[name][i + 1:])
                assert "CUDA device" not in str(e.value), (name, i)
    # a cache of fewer layers, or of other rows, than the call's
    for other in ((3, 1, 9, 2, 64), (3, 2, 9, 1, 128), (3, 2, 9, 4, 64)):
        small = prcr.cache_contiguous(_t(other), _t(other))
        paged = prcr.cache_paged(_t(other[1:]).unsqueeze(1), _t(other[1:]).unsqueeze(1), _t((3, 1), i32))
        for name, args in good.items():
            for bad in (small, paged):
                late = {"append_kv": [], "chunk_attention": [1]}.get(name)  # (the second layer)
                a = args[:2] + late + args[3:] if late else list(args)
                a[1] = bad
                with pytest.raises(ValueError, match="the cache holds"):
                    getattr(prcr, name)(*a)
    with pytest.raises(ValueError, match="the cache holds"):
        prcr.evict(*good["evict"], dst=small)
    with pytest.raises(ValueError, match="keep_out"):
        prcr.evict(*good["evict"][:8], _t((3, 2, 2, 9), i32), *good["evict"][9:])


def test_strides_of_single_entries():
    """A dimension of one entry may have any stride: it is read as packed."""
    assert B._strides(torch.as_strided(_t(4096), (1, 8, 64), (0, 64, 1)), 3, "q")[0] == 512
    assert B._strides(_t((8, 1, 64)).transpose(0, 1), 3, "q")[0] == 512
    assert B._strides(_t((2, 5, 2, 64)), 4, "k") == (640, 128, 64, 1)
    assert B._strides(torch.as_strided(_t(4096), (2, 1, 2, 64), (256, 8, 64, 1)), 4, "k") == (256, 128, 64, 1)
    assert B._strides(torch.as_strided(_t(4096), (1, 2, 2, 64), (0, 128, 64, 1)), 4, "k") == (256, 128, 64, 1)


def test_weights_workspace_refusals():
    """A call of lengths that need a workspace: none, one a byte short, and one that is not aligned."""
    c, n = _cfg(D=128, H=8, L=36), 120000
    need = prcr.weights_workspace_size(c, 3, 32, n)
    assert need == 3 * 36 * 32 * n * 4
    a = dict(cfg=c, cache=_flat(slot_stride=1024, layer_stride=n * 1024, seq_stride=36 * n * 1024, max_slots=n), hq=32, max_len=n, ss=n)
    assert call("prcr_accumulate_weights", **a, ws_bytes=need - 1) == B.EWORKSPACE
    assert call("prcr_accumulate_weights", **a, ws=None, ws_bytes=need) == B.EWORKSPACE
    assert call("prcr_accumulate_weights", **a, ws=FAKE + 8, ws_bytes=need) == B.EALIGN


def _wrong(ref, V, sees, g):
    """Results as mistakes would make them: nothing, the sign, a slot too many or too few, a lost part of the slots."""
    yield np.zeros_like(ref)
    yield -ref
    yield ref * (1 + 2.0 ** -6)
    yield np.roll(ref, 1, axis=0)
    yield np.repeat(V[:1].mean(0)[None], ref.shape[0], 0).repeat(g, 1)


@pytest.mark.parametrize("scale", [1.0, 30.0, 1000.0])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_the_bars_of_large_logits_see_wrong_results(D, scale):
    """What chunk_attention is held to at large logits is not wider than the results: wrong ones fail, and the right one
    rounded to bf16 passes."""
    rng = np.random.default_rng(D)
    bf16 = lambda x: torch.from_numpy(x).bfloat16().double().numpy()
    q, K, V = (bf16(rng.standard_normal(s) * f) for s, f in (((20, 4, D), scale), ((300, 2, D), 1.0), ((300, 2, D), 1.0)))
    sees = U.causal(20, 300, 300)
    ref, bar = U.chunk64_exact(q, K, V, sees)
    U.assert_close(bf16(ref), ref, bar)
    for bad in _wrong(ref, V, sees, 2):
        with pytest.raises(AssertionError):
            U.assert_close(bad, ref, bar)
    fewer, _ = U.chunk64_exact(q, K[:256], V[:256], U.causal(20, 300, 256))
    with pytest.raises(AssertionError):
        U.assert_close(fewer, ref, bar)


def test_documented_limits():
    """The largest numbers of layers, sequences and rows that a launch holds, and one more."""
    wide = dict(seq_stride=1 << 40, slot_stride=128)
    layers = lambda n: dict(cfg=_cfg(H=2, L=n), cache=_flat(**wide))
    assert call("prcr_accumulate_weights", **layers(32768)) == B.EINVAL  # 65536 layers by KV heads
    assert call("prcr_evict", **layers(65536)) == B.EINVAL
    many = _flat(n_seqs=70000)
    assert call("prcr_accumulate_weights", cache=many, n_seqs=65536) == B.EINVAL
    assert call("prcr_evict", cache=many, n_seqs=65536, len_out=FAKE + 2 ** 20) == B.EINVAL
    for name in ("prcr_chunk_attention", "prcr_accumulate_weights", "prcr_evict"):  # max_len at most the capacity, and 2^30
        assert call(name, max_len=257, **({} if name == "prcr_chunk_attention" else dict(ss=300))) == B.EINVAL
        big = dict(cache=_paged(bt_stride=2 ** 30, n_blocks=2 ** 30), max_len=2 ** 30 + 1)
        assert call(name, **big, **({} if name == "prcr_chunk_attention" else dict(ss=2 ** 31))) == B.EINVAL

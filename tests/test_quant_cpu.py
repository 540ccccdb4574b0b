"""CPU checks of append_kv_quant, quantize_cache, dequantize_cache and decode_attention_quant:
what the host refuses, before any CUDA call (the addresses below are never read), what it launches
(against a CUDA runtime that only keeps the launches), and the tests' own formats."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

import fake_gpu as F
import paper_2606_26631_gb300 as prcr
import quant_util as Q
from paper_2606_26631_gb300 import _binding as B

FAKE = 1 << 40


def _cfg(D=64, H=2, L=2):
    return prcr.rope_cfg(L, H, D, (D // 2, 0, 0))


def _wide(**o):
    return B.CacheDesc(**{**dict(kind=0, block_size=1, k=FAKE, v=FAKE + 2 ** 20, seq_stride=2 * 256 * 128, layer_stride=256 * 128, block_stride=0,
                                 slot_stride=128, block_table=None, bt_stride=0, n_blocks=0, max_slots=256, n_seqs=3), **o})


def _few(fmt=0, H=2, D=64, L=2, S=256, B_=3, **o):
    w, n = (D, 1) if fmt == 0 else (D // 2, D // 32)
    return B.QCacheDesc(**{**dict(format=fmt, kind=0, k=FAKE, v=FAKE + 2 ** 20, k_scale=FAKE, v_scale=FAKE + 2 ** 20, seq_stride=L * S * H * w,
                                  layer_stride=S * H * w, block_stride=0, slot_stride=H * w, scale_seq_stride=L * S * H * n, scale_layer_stride=S * H * n,
                                  scale_block_stride=0, scale_slot_stride=H * n, block_table=None, bt_stride=0, block_size=1, n_blocks=0,
                                  max_slots=S, n_seqs=B_, reserved=0), **o})


def _paged(fmt=0, H=2, D=64, bt=16, block=16, n_blocks=64, B_=3, **o):
    w, n = (D, 1) if fmt == 0 else (D // 2, D // 32)
    return _few(fmt, H, D, **{**dict(kind=1, seq_stride=0, scale_seq_stride=0, layer_stride=n_blocks * block * H * w, block_stride=block * H * w,
                                     scale_layer_stride=n_blocks * block * H * n, scale_block_stride=block * H * n, block_table=FAKE,
                                     bt_stride=bt, block_size=block, n_blocks=n_blocks, max_slots=0, n_seqs=B_), **o})


APPEND = dict(cfg=_cfg(), cache=_few(), n_seqs=3, l0=0, nl=2, k=FAKE, v=FAKE, ls=40 * 128, ts=128, coords=FAKE, off=FAKE, total=40,
              len_in=FAKE, len_out=FAKE + 64, status=FAKE)
QUANT = dict(cfg=_cfg(), src=_wide(), sl=0, cache=_few(), dl=0, nl=2, n_seqs=3, sb=FAKE, db=FAKE, count=FAKE, top=100, status=FAKE)
READ = dict(cfg=_cfg(), cache=_few(), sl=0, dst=_wide(), dl=0, nl=2, n_seqs=3, sb=FAKE, db=FAKE, count=FAKE, top=100, status=FAKE)
DECODE = dict(cfg=_cfg(), cache=_few(), n_seqs=3, l0=0, nl=2, hq=8, q=FAKE, pos=FAKE, len=FAKE, max_len=200, out=FAKE + 2 ** 24, status=FAKE,
              ws=FAKE, ws_bytes=1 << 40)
ENTRY = {"prcr_append_kv_quant": APPEND, "prcr_quantize_cache": QUANT, "prcr_dequantize_cache": READ, "prcr_decode_attention_quant": DECODE}


def call(name, lib=None, **over):
    a = {**ENTRY[name], **over}
    args = [C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()]
    return getattr(lib or prcr.lib(), name)(*args, None)


COMMON = [
    (dict(cfg=_cfg(D=40)), B.EINVAL), (dict(cfg=None), B.EINVAL), (dict(cache=None), B.EINVAL), (dict(n_seqs=-1), B.EINVAL), (dict(n_seqs=4), B.EINVAL),
    (dict(cache=_few(k=None)), B.EINVAL), (dict(cache=_few(v=None)), B.EINVAL), (dict(cache=_few(k_scale=None)), B.EINVAL),
    (dict(cache=_few(v_scale=None)), B.EINVAL), (dict(cache=_few(format=2)), B.EINVAL), (dict(cache=_few(reserved=1)), B.EINVAL),
    (dict(cache=_few(kind=2)), B.EINVAL), (dict(cache=_few(slot_stride=64)), B.EINVAL), (dict(cache=_few(scale_slot_stride=1)), B.EINVAL),
    (dict(cache=_few(layer_stride=-16)), B.EINVAL), (dict(cache=_few(seq_stride=-16)), B.EINVAL), (dict(cache=_few(scale_seq_stride=-1)), B.EINVAL),
    (dict(cache=_few(max_slots=-1)), B.EINVAL), (dict(cache=_few(k=FAKE + 8)), B.EALIGN), (dict(cache=_few(slot_stride=136)), B.EALIGN),
    (dict(cache=_few(1, scale_slot_stride=5)), B.EALIGN), (dict(cache=_few(1, k_scale=FAKE + 1)), B.EALIGN),
    (dict(cache=_few(1, scale_layer_stride=513)), B.EALIGN), (dict(cache=_paged(block_table=None)), B.EINVAL), (dict(cache=_paged(block_size=0)), B.EINVAL),
    (dict(cache=_paged(scale_block_stride=-1)), B.EINVAL), (dict(cache=_paged(block_table=FAKE + 2)), B.EALIGN), (dict(cache=_paged(block_stride=8)), B.EALIGN),
    (dict(cfg=_cfg(D=96), cache=_few(1, D=96)), B.EINVAL), (dict(status=None), B.EINVAL), (dict(status=FAKE + 2), B.EALIGN), (dict(nl=0), B.EINVAL)]
CAST = [(dict(sl=-1), B.EINVAL), (dict(sl=1), B.EINVAL), (dict(dl=-1), B.EINVAL), (dict(dl=1), B.EINVAL), (dict(top=-1), B.EINVAL),
        (dict(top=2 ** 30 + 1), B.EINVAL), (dict(sb=None), B.EINVAL), (dict(db=None), B.EINVAL), (dict(count=None), B.EINVAL), (dict(count=FAKE + 1), B.EALIGN)]
BAD = {
    "prcr_append_kv_quant": [
        (dict(l0=-1), B.EINVAL), (dict(l0=1), B.EINVAL), (dict(total=-1), B.EINVAL), (dict(k=None), B.EINVAL), (dict(v=None), B.EINVAL),
        (dict(ts=64), B.EINVAL), (dict(ls=-8), B.EINVAL), (dict(coords=None), B.EINVAL), (dict(off=None), B.EINVAL), (dict(len_in=None), B.EINVAL),
        (dict(len_out=None), B.EINVAL), (dict(len_out=FAKE + 8), B.EINVAL), (dict(k=FAKE + 8), B.EALIGN), (dict(ts=132), B.EALIGN), (dict(ls=4), B.EALIGN),
        (dict(off=FAKE + 2), B.EALIGN), (dict(coords=FAKE + 1), B.EALIGN)],
    "prcr_quantize_cache": CAST + [(dict(src=None), B.EINVAL), (dict(src=_wide(v=FAKE + 8)), B.EALIGN), (dict(src=_wide(n_seqs=2)), B.EINVAL)],
    "prcr_dequantize_cache": CAST + [(dict(dst=None), B.EINVAL), (dict(dst=_wide(slot_stride=132)), B.EALIGN), (dict(dst=_wide(n_seqs=2)), B.EINVAL)],
    "prcr_decode_attention_quant": [
        (dict(cfg=_cfg(D=96), cache=_few(D=96)), B.EINVAL), (dict(hq=9), B.EINVAL), (dict(hq=1), B.EINVAL), (dict(hq=18), B.EINVAL), (dict(l0=-1), B.EINVAL),
        (dict(l0=1), B.EINVAL), (dict(max_len=-1), B.EINVAL), (dict(max_len=257), B.EINVAL), (dict(cache=_paged(bt=2 ** 30), max_len=2 ** 30 + 1), B.EINVAL),
        (dict(q=None), B.EINVAL), (dict(pos=None), B.EINVAL), (dict(len=None), B.EINVAL), (dict(out=None), B.EINVAL), (dict(out=FAKE), B.EINVAL),
        (dict(q=FAKE + 2), B.EALIGN), (dict(pos=FAKE + 4), B.EALIGN), (dict(len=FAKE + 2), B.EALIGN), (dict(out=FAKE + 2 ** 24 + 8), B.EALIGN),
        (dict(cfg=_cfg(D=256, H=8), cache=_few(D=256, H=8), hq=64), B.EINVAL)],
}


@pytest.mark.parametrize("name,over,code", [(n, o, c) for n in ENTRY for o, c in COMMON + BAD[n]],
                         ids=lambda v: ",".join(v) if isinstance(v, dict) else str(v))
def test_refusals(name, over, code):
    assert call(name, **over) == code


def test_empty_calls():
    for name in ENTRY:
        assert call(name, n_seqs=0) == B.OK


def test_struct_layout():
    assert C.sizeof(B.QCacheDesc) == 136
    assert (prcr.QFMT_E4M3, prcr.QFMT_E2M1) == (0, 1)


def _decode(fmt, H, g, D, L, seqs, top, ws_bytes, lib):
    c = _cfg(D, H, L)
    return call("prcr_decode_attention_quant", lib, cfg=c, cache=_few(fmt, H, D, L, max(1, top), seqs), n_seqs=seqs, nl=L, hq=H * g, max_len=top, ws_bytes=ws_bytes)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("fmt", [0, 1])
def test_a_workspace_holds_every_smaller_call(fmt, D):
    """Sized once it is enough for every call of fewer sequences, layers and slots; a byte less than a call's is refused."""
    lib, rng = F.lib(), random.Random(D)
    for H, g in ((1, 1), (1, 8), (2, 4), (4, 7), (8, 4), (5, 3), (16, 1), (3, 2)):
        if H * g * D > 8192:
            continue
        for L, seqs, top in ((1, 1, 900), (36, 16, 8198), (1, 64, 32768), (2, 300, 40), (4, 3, 1 << 20)):
            size = lib.prcr_decode_quant_workspace_size(C.byref(_cfg(D, H, L)), fmt, seqs, L, H * g, top)
            for _ in range(20):
                l, b, n = (max(1, int(round(x ** rng.random()))) for x in (L, seqs, top))
                assert _decode(fmt, H, g, D, l, b, n, size, lib) == B.OK
                assert lib.prcr_decode_quant_workspace_size(C.byref(_cfg(D, H, L)), fmt, b, l, H * g, n) <= size
            assert _decode(fmt, H, g, D, L, seqs, top, size, lib) == B.OK
            assert _decode(fmt, H, g, D, L, seqs, top, size - 1, lib) == B.EWORKSPACE
    c = _cfg(D, 2, 2)
    assert call("prcr_decode_attention_quant", lib, cfg=c, cache=_few(fmt, 2, D), ws=None) == B.EWORKSPACE
    assert call("prcr_decode_attention_quant", lib, cfg=c, cache=_few(fmt, 2, D), ws=FAKE + 8) == B.EALIGN
    for bad in (dict(fmt=2), dict(n=-1), dict(n=2 ** 30 + 1), dict(hq=3), dict(L=0), dict(seqs=0)):
        a = {**dict(fmt=fmt, seqs=1, L=1, hq=8, n=100), **bad}
        assert lib.prcr_decode_quant_workspace_size(C.byref(c), a["fmt"], a["seqs"], a["L"], a["hq"], a["n"]) == 0
    F.launches()
    assert lib.fake_lowered() == 0


def test_launches():
    """One kernel to write or read rows, two for a decode step; sizes at the launch's limits."""
    lib = F.lib()
    F.launches()
    for name, n in (("prcr_append_kv_quant", 1), ("prcr_quantize_cache", 1), ("prcr_dequantize_cache", 1), ("prcr_decode_attention_quant", 2)):
        for fmt in (0, 1):
            assert call(name, lib, cache=_few(fmt)) == B.OK
            assert len(F.launches()) == n
    # many heads, layers and tokens; nothing at all
    for H, D in ((512, 16), (102, 80), (170, 48), (32, 256), (1, 16)):
        c, few, wide = _cfg(D, H, 2), _few(0, H, D), _wide(slot_stride=H * D, layer_stride=256 * H * D, seq_stride=512 * H * D)
        for total in (0, 1, 2 ** 31 - 1):
            assert call("prcr_append_kv_quant", lib, cfg=c, cache=few, ts=H * D, ls=0, total=total) == B.OK
        for top in (0, 1, 2 ** 30):
            assert call("prcr_quantize_cache", lib, cfg=c, src=wide, cache=few, top=top) == B.OK
            assert call("prcr_dequantize_cache", lib, cfg=c, dst=wide, cache=few, top=top) == B.OK
    many = _cfg(64, 2, 100000)
    wide, few = _wide(n_seqs=70000, layer_stride=0, seq_stride=0), _few(layer_stride=0, scale_layer_stride=0, n_seqs=70000)
    assert call("prcr_append_kv_quant", lib, cfg=many, cache=few, nl=100000) == B.OK
    assert call("prcr_quantize_cache", lib, cfg=many, src=wide, cache=few, nl=100000) == B.OK
    assert call("prcr_quantize_cache", lib, src=wide, cache=few, n_seqs=65536) == B.EINVAL
    assert call("prcr_dequantize_cache", lib, dst=wide, cache=few, n_seqs=65536) == B.EINVAL
    assert call("prcr_decode_attention_quant", lib, cfg=many, cache=few, n_seqs=70000, nl=100000, ws_bytes=1 << 60) == B.EINVAL  # rows: grid x
    F.launches()


def _t(shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses():
    """Wrong types, shapes and layouts raise before the library is called; so do tensors that are not on the current GPU."""
    c, i32, u8, e4 = _cfg(), torch.int32, torch.uint8, torch.float8_e4m3fn
    wide = prcr.cache_contiguous(_t((3, 2, 9, 2, 64)), _t((3, 2, 9, 2, 64)))
    k4, s4 = _t((3, 2, 9, 2, 64), e4), _t((3, 2, 9, 2, 1), u8)
    k2, s2 = _t((3, 2, 9, 2, 32), u8), _t((3, 2, 9, 2, 2), u8)
    few = prcr.qcache_contiguous(k4, k4, s4, s4)
    assert (few.format, few.slot_stride, few.scale_slot_stride, few.seq_stride) == (0, 128, 2, 2 * 9 * 128)
    four = prcr.qcache_contiguous(k2, k2, s2, s2)
    assert (four.format, four.slot_stride, four.scale_slot_stride, four._rows) == (1, 64, 4, (2, 2, 64))
    table = _t((3, 4), i32)
    paged = prcr.qcache_paged(k2, k2, s2, s2, table)
    assert (paged.block_size, paged.n_blocks, paged.bt_stride, paged._rows) == (9, 2, 4, (3, 2, 64))
    for bad in ((k4.view(u8).float(), k4, s4, s4), (k4, k2, s4, s4), (k4, k4, s2, s2), (k2, k2, s4, s4), (k4[:, :1], k4, s4, s4), (k4, k4, s4[:, :1], s4),
                (k4, k4, s4.int(), s4), (k4[..., :32], k4[..., :32], s4, s4), (k4[0], k4[0], s4[0], s4[0]), (k4, k4, s4, s4.transpose(0, 1))):
        with pytest.raises((TypeError, ValueError)):
            prcr.qcache_contiguous(*bad)
    for bad in (table.long(), table.t()):
        with pytest.raises(ValueError):
            prcr.qcache_paged(k2, k2, s2, s2, bad)
    off, ln, st, rows, pos = _t(4, i32), _t(3, i32), _t(1, i32), _t((2, 5, 2, 64)), _t((5, 3), i32)
    q, p, out = _t((3, 2, 8, 64)), _t(3, torch.int64), _t((3, 2, 8, 64), torch.float32)
    good = {
        "append_kv_quant": [c, few, 0, rows, rows, pos, off, ln, ln.clone(), st],
        "quantize_cache": [c, wide, 0, few, 0, 2, ln, ln, ln, 9, st],
        "dequantize_cache": [c, four, 0, wide, 0, 2, ln, ln, ln, 9, st],
        "decode_attention_quant": [c, four, 0, q, p, ln, 9, out, st],
    }
    for name, args in good.items():
        with pytest.raises(ValueError, match="CUDA device"):
            getattr(prcr, name)(*args)
    wrong = {
        "append_kv_quant": {2: [1], 3: [rows.float(), rows[:, :, :1], rows.transpose(2, 3)], 4: [rows[:, :4]], 5: [pos.long(), pos[:4]], 6: [off[:3]], 8: [ln[:2]]},
        "quantize_cache": {1: [few], 3: [wide], 5: [3], 2: [1], 4: [1], 6: [ln[:2], ln.long()], 7: [ln[:2]], 8: [ln.long()]},
        "dequantize_cache": {1: [wide], 3: [four], 5: [3], 6: [ln.float()], 8: [ln.long()]},
        "decode_attention_quant": {2: [1], 3: [q.float(), q[:, :1], q[0], q[..., :32], q.transpose(1, 2)], 4: [p.int(), p[:2]], 5: [ln.long(), ln[:2]],
                                   7: [out.double(), out[:2]]},
    }
    for name, at in wrong.items():
        for i, values in at.items():
            for v in values:
                with pytest.raises((TypeError, ValueError)) as e:
                    getattr(prcr, name)(*good[name][:i], v, *good[name][i + 1:])
                assert "CUDA device" not in str(e.value), (name, i)
    other = prcr.qcache_contiguous(_t((3, 2, 9, 1, 64), e4), _t((3, 2, 9, 1, 64), e4), _t((3, 2, 9, 1, 1), u8), _t((3, 2, 9, 1, 1), u8))
    for name, at in (("append_kv_quant", 1), ("quantize_cache", 3), ("dequantize_cache", 1), ("decode_attention_quant", 1)):
        with pytest.raises(ValueError, match="the cache holds"):
            getattr(prcr, name)(*good[name][:at], other, *good[name][at + 1:])


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_the_tests_formats(fmt):
    """The reference's rounding against torch's own conversion (E4M3), and by hand (E2M1); scales, ties, what a group holds."""
    rng = np.random.default_rng(1)
    D = 64
    x = torch.from_numpy(rng.standard_normal((50, D))).bfloat16().double().numpy()
    codes, byte = Q.quantize(fmt, x)
    val = Q.stand_for(fmt, codes, byte)
    g = Q.groups(fmt, D)
    for j in range(byte.shape[-1]):
        top = np.abs(x[:, g == j]).max(-1) / Q.scale64(byte[:, j])
        assert (top <= Q.VALUES[fmt][-1]).all() and (top > Q.VALUES[fmt][-1] / 2).all()
    s = Q.scale64(byte)[:, g]
    if fmt == "e4m3":
        want = torch.from_numpy(x / s).float().to(torch.float8_e4m3fn)
        assert np.array_equal(want.view(torch.uint8).numpy(), codes)
        assert np.array_equal(np.unique(Q.E4M3), torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    else:
        ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
        assert Q.E2M1[Q.nearest("e2m1", ties, np.full(7, 127))].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert np.abs(val - x).max() <= 0.51 * np.abs(x).max()
    again = Q.quantize(fmt, val)
    assert np.array_equal(Q.stand_for(fmt, *again), val)
    assert np.array_equal(Q.unpack(fmt, Q.pack(fmt, codes)), codes)
    for bad in (np.inf, np.nan):
        y = x[:1].copy()
        y[0, 5] = bad
        codes, byte = Q.quantize(fmt, y)
        hit = g == g[5]
        assert np.isnan(Q.stand_for(fmt, codes, byte)[0][hit]).all() and (codes[0][hit] == 0).all()
        assert not np.isnan(Q.stand_for(fmt, codes, byte)[0][~hit]).any()


def test_the_bar_of_decode_sees_wrong_results():
    """What decode_attention_quant is held to is far narrower than its results: a slot too few, a weight or a scale off fail it."""
    rng = np.random.default_rng(3)
    q, K, V = rng.standard_normal((4, 128)), rng.standard_normal((300, 1, 128)), rng.standard_normal((300, 1, 128))
    ref, bar = Q.decode64(q, 5, K, V)
    assert (bar < 1e-3 * np.abs(ref).max()).all()
    for wrong in (Q.decode64(q, 5, K[:299], V[:299])[0], Q.decode64(q, 6, K, V)[0], Q.decode64(q, 5, K * 1.01, V)[0], ref * 1.002,
                  Q.decode64(q, 5, K, np.concatenate([V[:299], 2 * V[299:]]))[0]):
        assert (np.abs(wrong - ref) > bar).any()

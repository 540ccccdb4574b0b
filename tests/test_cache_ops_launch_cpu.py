"""CPU checks of what append_kv, chunk_attention, accumulate_weights and evict
launch, against a CUDA runtime that only keeps the launches (fake_gpu)."""
import ctypes as C
import random

import pytest

import fake_gpu as F
from paper_2606_26631_gb300 import _binding as B


def chunk(c, seqs, group, total, max_len, ws_bytes):
    cache, Hq = F.contiguous(c, seqs, max(1, max_len)), c.n_kv_heads * group
    row = Hq * c.head_dim
    return F.lib().prcr_chunk_attention(C.byref(c), C.byref(cache), seqs, 0, Hq, F.FAKE, row, F.FAKE, F.FAKE, total, F.FAKE, max_len,
                                        F.WORK, row, F.FAKE, F.WORK, ws_bytes, None)


def weights(c, seqs, group, max_len, ws_bytes):
    cache, Hq = F.contiguous(c, seqs, max(1, max_len)), c.n_kv_heads * group
    return F.lib().prcr_accumulate_weights(C.byref(c), C.byref(cache), seqs, Hq, F.FAKE, F.FAKE, F.FAKE, max_len, F.FAKE, max_len, 1.0,
                                           F.FAKE, F.WORK, ws_bytes, None)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_workspaces_hold_every_smaller_call(D):
    """A workspace sized once is enough for every call of fewer sequences, tokens and slots."""
    rng = random.Random(D)
    for H, g in ((1, 1), (1, 8), (2, 4), (4, 7), (8, 4), (5, 3), (100 if D == 64 else 20, 1)):
        if H * g * D > 16384:
            continue
        c = F.cfg(2, H, D)
        for seqs, total, top in ((1, 1, 900), (1, 500, 8192), (16, 96, 8198), (4, 4096, 16384), (300, 300, 40000), (2, 30000, 1 << 20)):
            size = F.lib().prcr_chunk_workspace_size(C.byref(c), seqs, H * g, total, top)
            for _ in range(60):
                b, t, n = (int(round(x ** rng.random())) for x in (seqs, total, top))
                assert chunk(c, b, g, t, n, size) == B.OK, (H, g, seqs, total, top, b, t, n)
                assert F.lib().prcr_chunk_workspace_size(C.byref(c), b, H * g, t, n) <= size
            assert chunk(c, seqs, g, total, top, size) == B.OK
        for seqs, top in ((1, 900), (16, 8198), (3, 60000), (2, 500000)):
            size = F.lib().prcr_weights_workspace_size(C.byref(c), seqs, H * g, top)
            for _ in range(60):
                b, n = (int(round(x ** rng.random())) for x in (seqs, top))
                assert weights(c, b, g, n, size) == B.OK, (H, g, seqs, top, b, n)
            assert weights(c, seqs, g, top, size) == B.OK
    F.launches()


def test_a_chunk_call_short_of_workspace_is_refused():
    c = F.cfg(2, 8, 128)
    splits_of = lambda seqs, total, n: sum("merge" in k for k, _ in F.launches()) if chunk(c, seqs, 4, total, n, 1 << 40) == B.OK else None
    F.launches()
    assert splits_of(1, 1, 933) == 1  # split: a second kernel joins the parts
    assert chunk(c, 1, 4, 1, 933, 32 * 8 * 130 * 4) == B.OK  # 8 tiles of 128 slots, a split each
    assert chunk(c, 1, 4, 1, 933, 32 * 8 * 130 * 4 - 1) == B.EWORKSPACE
    F.launches()
    assert splits_of(1, 8192, 8192) == 0  # 1024 units: none
    assert chunk(c, 1, 4, 8192, 8192, 0) == B.OK


def test_shared_memory_and_limits():
    """Weights over every length that a cluster holds: within an SM's shared memory, and the limit of a kernel only rises."""
    F.lib()
    for D in (64, 128, 256):
        for g in (1, 4, 8):
            c = F.cfg(2, 2, D)
            for n in (1, 15, 16, 128, 129, 933, 4096, 12000, 30000, 49000, 50000, 51000, 120000, 399000, 400000, 410000):
                size = F.lib().prcr_weights_workspace_size(C.byref(c), 2, 2 * g, n)
                assert n * g > 380000 if size else n * g < 420000, (D, g, n)
                assert weights(c, 2, g, n, size) == B.OK
    names = {k for k, _ in F.launches()}
    assert any("weights_kernel" in k for k in names) and any("weights_sum" in k for k in names)
    assert F.lib().fake_lowered() == 0


@pytest.mark.parametrize("D", [64, 128, 256])
def test_weights_need_no_workspace_up_to_the_documented_length(D):
    """399,000 / query heads per KV head slots, and every length below: no bytes are asked for, and none is a call's."""
    for g in range(1, 9):
        c, most = F.cfg(1, 1, D), 399000 // g
        rng = random.Random(g)
        for n in [most, most - 1, most - 15, most // 2, most // 8 + 1] + [rng.randint(1, most) for _ in range(40)]:
            for seqs in (1, 16):
                assert F.lib().prcr_weights_workspace_size(C.byref(c), seqs, g, n) == 0, (D, g, n)
                assert weights(c, seqs, g, n, 0) == B.OK, (D, g, n)
    F.launches()

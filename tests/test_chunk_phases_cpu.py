"""The order of the steps inside a CTA of the chunk attention kernel, over every way that its
warps and the tensor cores can come to run: no wait is ever left behind, and none ends early.

The model has the kernel's actors: softmax warps, the warp that issues matrix instructions, and the
tensor cores, which work through what was issued in order. A barrier is what the hardware's is:
a count of completed phases of which a wait sees the parity alone. Which barrier and parity a
step uses comes from the kernel's own header (csrc/prcr_chunk_phases.h)."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

import pytest

from paper_2606_26631_gb300 import _build

SOURCE = """
#include "prcr_chunk_phases.h"
extern "C" void scores(int nq, int q, int j, int* out) { auto p = prcr::chunk_scores(nq, q, j); out[0] = p.bar; out[1] = int(p.parity); }
extern "C" void products(int nq, int q, int j, int* out) { auto p = prcr::chunk_products(nq, q, j); out[0] = p.bar; out[1] = int(p.parity); }
"""


@functools.lru_cache(None)
def header():
    where = tempfile.mkdtemp()
    src, lib = os.path.join(where, "phases.cpp"), os.path.join(where, "phases.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", "-I", _build.CSRC, src, "-o", lib], check=True)
    return C.CDLL(lib)


def phases(nq):
    def of(name):
        def step(q, j):
            out = (C.c_int * 2)()
            getattr(header(), name)(nq, q, j, out)
            return out[0], out[1]
        return functools.lru_cache(None)(step)
    return of("scores"), of("products")


def issuer(nq, tiles, scores, products):
    """What the issuing warp does: waits for both halves of P of (half, tile), commits of a step's barrier."""
    steps = [("commit", "s", scores(q, 0)[0], ("s", q, 0)) for q in range(nq) if tiles[q]]
    for j in range(max(tiles)):
        if nq == 1 and j + 1 < tiles[0]:
            steps.append(("commit", "s", scores(0, j + 1)[0], ("s", 0, j + 1)))
        for q in range(nq):
            if j >= tiles[q]:
                continue
            steps += [("wait", "p%d" % half, *scores(q, j), ("p%d" % half, q, j)) for half in (0, 1)]
            if nq == 2 and j + 1 < tiles[q]:
                steps.append(("commit", "s", scores(q, j + 1)[0], ("s", q, j + 1)))
            else:
                steps.append(("commit", "o", products(q, j)[0], ("o", q, j)))
    return steps


def explore(nq, tiles, warps, scores, products):
    """Every state that is reached; the first fault found, or None. A warp's tile: stage 0 waits for S; the ways from there
    are raise (1 waits for the last tile's products, then 2) or not (2); 2 and 3 hand over P's halves; 4 waits for the last
    tile's products where the tile did not raise; behind the last tile a wait for its own."""
    steps = issuer(nq, tiles, scores, products)
    commits = [s for s in steps if s[0] == "commit"]
    owners = [q for q in range(nq) for _ in range(warps)]

    def completed(state, kind, bar):  # phases of a barrier that are over
        if kind in ("s", "o"):
            return sum(1 for c in commits[:state[1]] if c[1] == kind and c[2] == bar)
        half, count = int(kind[1]), {}
        for q, (j, stage, _) in zip(owners, state[2:]):
            for t in range(tiles[q]):
                if t < j or (t == j and stage > 2 + half):
                    if scores(q, t)[0] == bar:
                        count[(q, t)] = count.get((q, t), 0) + 1
        return sum(1 for n in count.values() if n == warps)

    def happened(state, what):
        kind, q, j = what
        if kind in ("s", "o"):
            return any(c[3] == what for c in commits[:state[1]])
        return all(t > j or (t == j and stage > 2 + int(kind[1])) for o, (t, stage, _) in zip(owners, state[2:]) if o == q)

    def waits(state, kind, bar, parity, what):
        """Whether the wait is over; a fault if it is, and what it waits for did not happen."""
        over = (completed(state, kind, bar) & 1) != parity
        if over and not happened(state, what):
            raise AssertionError(f"a wait for {what} ended early in {state}")
        return over

    start = (0, 0) + tuple((0, 0, 0) for _ in owners)
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        pos, done = state[:2]
        after = []
        if pos < len(steps):
            s = steps[pos]
            if s[0] == "commit" or waits(state, *s[1:]):
                after.append((pos + 1, done) + state[2:])
        if done < sum(1 for s in steps[:pos] if s[0] == "commit"):  # the tensor cores finish the next step
            after.append((pos, done + 1) + state[2:])
        for w, (q, (j, stage, raised)) in enumerate(zip(owners, state[2:])):
            def go(*to):
                after.append(state[:2 + w] + (to,) + state[3 + w:])
            n = tiles[q]
            if j > n or n == 0:
                continue  # done
            if j == n:  # behind the last tile: its products
                if waits(state, "o", *products(q, n - 1), ("o", q, n - 1)):
                    go(n + 1, 0, 0)
            elif stage == 0:
                if waits(state, "s", *scores(q, j), ("s", q, j)):
                    go(j, 2, 0)
                    if j and nq == 1:
                        go(j, 1, 1)
            elif stage == 1:
                if waits(state, "o", *products(q, j - 1), ("o", q, j - 1)):
                    go(j, 2, 1)
            elif stage in (2, 3):
                go(j, stage + 1, raised)
            elif nq == 2 or j == 0 or raised or waits(state, "o", *products(q, j - 1), ("o", q, j - 1)):
                go(j + 1, 0, 0)
        if not after and (pos < len(steps) or any(j <= tiles[q] and tiles[q] for q, (j, _, _) in zip(owners, state[2:]))):
            raise AssertionError(f"nothing can go on in {state}")
        for x in after:
            if x not in seen:
                seen.add(x)
                todo.append(x)
    return len(seen)


@pytest.mark.parametrize("nq,tiles,warps", [(1, (1,), 2), (1, (2,), 2), (1, (3,), 2), (1, (5,), 2), (1, (9,), 1),
                                            (2, (1, 1), 1), (2, (4, 5), 1), (2, (5, 2), 1), (2, (3, 0), 2)], ids=str)
def test_every_wait_ends_and_none_early(nq, tiles, warps):
    assert explore(nq, tiles, warps, *phases(nq)) > 10 * max(tiles)


def test_the_model_sees_a_barrier_that_laps_a_warp():
    """Every tile's products on one barrier: a warp that hands over P before it looks at the barrier waits for good."""
    scores, _ = phases(1)
    with pytest.raises(AssertionError, match="nothing can go on"):
        explore(1, (3,), 2, scores, lambda q, j: (0, j & 1))

// Which of the chunk attention kernel's barriers stands for a step of tile j, and the
// parity of its phase (host and device: the order of the steps is tested on a CPU).
//
// A wait by parity tells a phase from the next one only, so a barrier must not complete
// two phases while a warp waits for the first. Every step has such a barrier: the phase
// behind the one that a warp waits for needs an arrival that this warp makes later.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define PRCR_HOST_DEVICE __host__ __device__
#else
#define PRCR_HOST_DEVICE
#endif

namespace prcr {

struct ChunkPhase {
    int bar;
    uint32_t parity;
};

// S of a tile, and P of it: with two halves of 128 rows (nq = 2) half q's, else the
// buffers of even and of odd tiles in turn.
PRCR_HOST_DEVICE constexpr ChunkPhase chunk_scores(int nq, int q, int j) {
    return nq == 2 ? ChunkPhase{q, uint32_t(j & 1)} : ChunkPhase{j & 1, uint32_t((j >> 1) & 1)};
}

// The products of a tile added to O: with two halves the last tile's alone, else every
// tile's, on barriers in turn. (A warp hands over tile j's P before it waits for tile
// j - 1's products, so tile j's may be done by then: on one barrier both phases would have
// gone by. Tile j + 1's, next on the barrier of j - 1, need this warp's next P.)
PRCR_HOST_DEVICE constexpr ChunkPhase chunk_products(int nq, int q, int j) {
    return nq == 2 ? ChunkPhase{q, 0} : ChunkPhase{j & 1, uint32_t((j >> 1) & 1)};
}

}  // namespace prcr

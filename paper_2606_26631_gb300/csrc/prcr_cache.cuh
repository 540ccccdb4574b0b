// Device helpers of the kernels that append to, attend over, weigh and evict
// the decoder cache.
#pragma once

#include "prcr_device.cuh"

namespace prcr {

// The block of a sequence's table that holds a slot (below 2^31).
__device__ __forceinline__ uint32_t block_index(const CacheView& c, uint32_t slot) {
    return uint32_t((uint64_t(slot) * c.div_mul) >> c.div_shift);
}

// Element offset of a slot's row (layer and head terms excluded) given its block
// (paged), or -1 where that is not mapped.
__device__ __forceinline__ int64_t row_in_block(const CacheView& c, int b, uint32_t slot, int32_t blk) {
    if (c.kind == PRCR_CACHE_CONTIGUOUS) return int64_t(b) * c.seq_stride + int64_t(slot) * c.slot_stride;
    if (blk < 0 || blk >= c.n_blocks) return -1;
    const uint32_t o = slot - block_index(c, slot) * uint32_t(c.block_size);
    return int64_t(blk) * c.block_stride + int64_t(o) * c.slot_stride;
}

// Element offset of a slot's row (layer and head terms excluded), or -1 with the
// reason in err: beyond the capacity, or in a block that is not mapped.
__device__ __forceinline__ int64_t slot_row(const CacheView& c, int b, int64_t slot, uint32_t& err) {
    if (slot < 0 || slot >= c.capacity) {
        err |= PRCR_ST_CAPACITY;
        return -1;
    }
    if (slot >= (int64_t(1) << 31)) {  // (a sequence's slots are counted in an int32)
        err |= PRCR_ST_CAPACITY;
        return -1;
    }
    const uint32_t s = uint32_t(slot);
    const int32_t blk = c.kind == PRCR_CACHE_CONTIGUOUS ? 0 : c.block_table[int64_t(b) * c.bt_stride + block_index(c, s)];
    const int64_t row = row_in_block(c, b, s, blk);
    if (row < 0) err |= PRCR_ST_NO_BLOCK;
    return row;
}

// Whether this thread sees a fault in the offsets of n packed sequences: off[0]
// = 0, none below the one before, the last at most `total`. The block's
// threads take the entries in turn.
__device__ __forceinline__ bool bad_offsets(const int32_t* off, int n, int total) {
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int x = off[i], y = off[i + 1];
        bad |= (i == 0 && x != 0) || y < x || y > total;
    }
    return bad;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

}  // namespace prcr

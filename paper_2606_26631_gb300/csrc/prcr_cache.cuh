// Device helpers of the kernels that append to, attend over, weigh and evict
// the decoder cache.
#pragma once

#include "prcr_device.cuh"

namespace prcr {

// Element offset of a slot's row (layer and head terms excluded), or -1 with the
// reason in err: beyond the capacity, or in a block that is not mapped.
__device__ __forceinline__ int64_t slot_row(const CacheView& c, int b, int64_t slot, uint32_t& err) {
    if (slot < 0 || slot >= c.capacity) {
        err |= PRCR_ST_CAPACITY;
        return -1;
    }
    if (c.kind == PRCR_CACHE_CONTIGUOUS) return int64_t(b) * c.seq_stride + slot * c.slot_stride;
    const uint32_t s = uint32_t(slot), lb = s / uint32_t(c.block_size);  // a slot is below 2^31
    const int32_t blk = c.block_table[int64_t(b) * c.bt_stride + lb];
    if (blk < 0 || blk >= c.n_blocks) {
        err |= PRCR_ST_NO_BLOCK;
        return -1;
    }
    return int64_t(blk) * c.block_stride + int64_t(s - lb * uint32_t(c.block_size)) * c.slot_stride;
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

}  // namespace prcr

// Eviction from the decoder cache: of every sequence longer than the budget,
// each (layer, KV head) keeps its first n_sink and last n_recent slots and,
// of the others, those of the highest score; the kept rows move to slots
// 0 .. budget - 1 in their order, in place or into another cache.
//
// One CTA per (KV head, layer, sequence):
//  1. the score at the cut by a radix selection, 8 bits a pass, over the
//     scores mapped to integers of the same order;
//  2. one pass over the slots in order, tile by tile, that gives every kept
//     slot its place by prefix sums (equal scores at the cut: the lower slots
//     first), writes the indices and moves the scores;
//  3. the rows, in order, tile by tile. In place a tile's destinations are
//     slots below those that later tiles read (slot keep[j] >= j), so reading
//     a whole tile before writing it is all the order that is needed.
// Memory-bound: the kept rows are read once and written once.
#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"

namespace prcr {
namespace {

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr unsigned kFull = 0xffffffffu;

// An integer of the score's order, NaN below everything (equal zeros, whatever
// their sign).
__device__ __forceinline__ uint32_t score_key(float f) {
    const uint32_t u = __float_as_uint(f + 0.0f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(const __grid_constant__ EvictArgs a) {
    __shared__ uint32_t s_hist[256];
    __shared__ int s_scan[2][kEvictWarps];
    __shared__ uint32_t s_pick[2];
    const int h = blockIdx.x, l = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t col = (int64_t(b) * a.n_layers + l) * a.n_kv_heads + h;
    int32_t* keep = a.keep + col * a.budget;
    const float* score = a.score + col * a.score_stride;
    float* score_out = a.score_out + col * a.score_stride;
    pdl_allow();
    pdl_wait();

    const int n = a.seq_len[b];
    const int m = min(n, a.budget);
    // a sequence with a fault is left as it was
    uint32_t err = 0;
    if (n < 0 || n > a.max_len || n > a.src.capacity || m > a.dst.capacity) {
        err = PRCR_ST_CAPACITY;
    } else if (a.src.kind == PRCR_CACHE_PAGED) {
        for (int i = tid; i < int((int64_t(n) + a.src.block_size - 1) / a.src.block_size); i += kEvictThreads) {
            const int32_t blk = a.src.block_table[int64_t(b) * a.src.bt_stride + i];
            if (blk < 0 || blk >= a.src.n_blocks) err = PRCR_ST_NO_BLOCK;
        }
    }
    if (err == 0 && !a.in_place && a.dst.kind == PRCR_CACHE_PAGED) {
        for (int i = tid; i < int((int64_t(m) + a.dst.block_size - 1) / a.dst.block_size); i += kEvictThreads) {
            const int32_t blk = a.dst.block_table[int64_t(b) * a.dst.bt_stride + i];
            if (blk < 0 || blk >= a.dst.n_blocks) err = PRCR_ST_NO_BLOCK;
        }
    }
    const bool lead = h == 0 && l == 0;
    if (err && lead) atomicOr(a.status, err);
    if (__syncthreads_or(err != 0)) {
        for (int j = tid; j < a.budget; j += kEvictThreads) keep[j] = -1;
        if (lead && tid == 0) a.len_out[b] = a.in_place ? n : 0;
        return;
    }
    if (lead && tid == 0) a.len_out[b] = m;

    // 1. the cut among the slots between the first and the last ones
    const int lo = n > a.budget ? a.n_sink : n, hi = n > a.budget ? n - a.n_recent : n;
    int need = a.budget - a.n_sink - a.n_recent;  // of those
    uint32_t cut = 0xffffffffu;                   // keys above it stay
    int ties = 0;                                 // and so many, the first ones, of those equal to it
    if (n > a.budget && need > 0) {
        uint32_t prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kEvictThreads) s_hist[i] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += kEvictThreads) {
                const uint32_t k = score_key(score[i]);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
                    atomicAdd(&s_hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (warp == 0) {  // the bin, from the top, where the count reaches `need`
                uint32_t own[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += own[i] = s_hist[255 - (lane * 8 + i)];
                uint32_t upto = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_up_sync(kFull, upto, d);
                    if (lane >= d) upto += o;
                }
                uint32_t before = upto - sum;
                if (before < uint32_t(need) && upto >= uint32_t(need)) {
                    int i = 0;
                    while (before + own[i] < uint32_t(need)) before += own[i++];
                    s_pick[0] = uint32_t(255 - (lane * 8 + i));
                    s_pick[1] = before;
                }
            }
            __syncthreads();
            prefix |= s_pick[0] << shift;
            need -= int(s_pick[1]);
        }
        cut = prefix;
        ties = need;
    }

    // 2. places: kept slots before a slot = those above the cut + the ties taken
    int base_above = 0, base_tie = 0;
    for (int i0 = 0; i0 < n; i0 += kEvictThreads) {
        const int i = i0 + tid;
        bool above = false, tie = false;
        float x = 0.0f;
        if (i < n) {
            x = score[i];
            if (i < lo || i >= hi) {
                above = true;
            } else {
                const uint32_t k = score_key(x);
                above = k > cut;
                tie = k == cut && ties > 0;
            }
        }
        const uint32_t ma = __ballot_sync(kFull, above), mt = __ballot_sync(kFull, tie);
        if (lane == 0) {
            s_scan[0][warp] = __popc(ma);
            s_scan[1][warp] = __popc(mt);
        }
        __syncthreads();  // also: the tile's scores are read before any is written
        int wa = 0, wt = 0, ta = 0, tt = 0;
#pragma unroll
        for (int w = 0; w < kEvictWarps; ++w) {
            const int ca = s_scan[0][w], ct = s_scan[1][w];
            if (w < warp) wa += ca, wt += ct;
            ta += ca;
            tt += ct;
        }
        const uint32_t below = (1u << lane) - 1;
        const int pa = base_above + wa + __popc(ma & below), pt = base_tie + wt + __popc(mt & below);
        if (above || (tie && pt < ties)) {
            const int j = pa + min(pt, ties);
            keep[j] = i;
            score_out[j] = x;
        }
        base_above += ta;
        base_tie += tt;
        __syncthreads();
    }
    for (int j = m + tid; j < a.budget; j += kEvictThreads) keep[j] = -1;
    for (int64_t j = m + tid; j < a.score_stride; j += kEvictThreads) score_out[j] = 0.0f;
    __syncthreads();

    // 3. rows: a thread moves one 16-byte vector of K and of V of kRows rows a tile
    constexpr int kRows = 4;
    const int lanes = a.head_dim / 8, per = kEvictThreads / lanes;
    const int r0 = tid / lanes, v = tid - r0 * lanes;
    const int64_t col_src = int64_t(l) * a.src.layer_stride + int64_t(h) * a.head_dim + v * 8;
    const int64_t col_dst = int64_t(l) * a.dst.layer_stride + int64_t(h) * a.head_dim + v * 8;
    for (int j0 = 0; j0 < m; j0 += per * kRows) {
        uint4 k[kRows], w[kRows];
        int64_t to[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int j = j0 + r * per + r0;
            to[r] = -1;
            if (r0 < per && j < m) {
                const int i = keep[j];
                uint32_t e = 0;
                if (!a.in_place || i != j) {
                    const int64_t from = slot_row(a.src, b, i, e) + col_src;
                    to[r] = slot_row(a.dst, b, j, e) + col_dst;
                    k[r] = *reinterpret_cast<const uint4*>(a.src.k + from);
                    w[r] = *reinterpret_cast<const uint4*>(a.src.v + from);
                }
            }
        }
        if (a.in_place) __syncthreads();
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (to[r] >= 0) {
                st_row(a.dst.k + to[r], k[r]);
                st_row(a.dst.v + to[r], w[r]);
            }
        }
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, int n_seqs, cudaStream_t stream) {
    const dim3 grid(unsigned(a.n_kv_heads), unsigned(a.n_layers), unsigned(n_seqs));
    return launch_pdl(evict_kernel, grid, dim3(kEvictThreads), 0, stream, a);
}

}  // namespace prcr

// Eviction from the decoder cache: of every sequence longer than the budget,
// each (layer, KV head) keeps its first n_sink and last n_recent slots and,
// of the others, those of the highest score; the kept rows move to slots
// 0 .. budget - 1 in their order, in place or into another cache.
//
// One CTA per (KV head, layer, sequence), or where that leaves SMs idle a cluster of
// up to 8: its first CTA does steps 1 and 2, and in step 3 each takes some of the rows'
// dims, which move independently of the others also in place.
//  1. the score at the cut by a radix selection, 11 bits a pass, over the
//     scores mapped to integers of the same order (held in shared memory where they
//     fit); it ends at the pass whose bin stays whole, the second for most scores;
//  2. one pass over the slots in order, in tiles of 4096, that gives every kept
//     slot its place by prefix sums (equal scores at the cut: the lower slots
//     first), writes the indices and moves the scores;
//  3. the rows, in order, tile by tile: a thread copies one 16-byte vector of K and
//     one of V of a tile asynchronously into its own part of a ring in shared memory,
//     several tiles ahead, and writes them out when they have landed. In place a
//     tile's destinations are slots below those that later tiles read (slot
//     keep[j] >= j), so a barrier between a tile's arrival at all threads and its
//     writes is all the order that is needed.
// Memory-bound: the kept rows are read once and written once; two CTAs per SM keep
// up to 192 KB in flight, and where there are more CTAs than that one's selection
// runs during the other's copies. Measured with head_dim 128: 8 sequences of up to
// 8192 slots to 2048, 28 layers of 4 heads, 326 us (5.9 TB/s of rows and scores); one of
// 4096 to 1024, 36 layers of 8 heads, 65 us (4.8 TB/s): there all CTAs select at once,
// 15 us before the first row moves. (With a barrier pair per 512 slots in step 2 and always
// three passes, 20 us; 256 threads, or tiles held in registers instead of the ring, are slower.)
#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"
#include "prcr_tc.cuh"

namespace prcr {
namespace {

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr unsigned kFull = 0xffffffffu;
constexpr int kRing = 6;                                     // tiles
constexpr int kRingBytes = kRing * kEvictThreads * 32;       // 32 bytes a thread and tile
constexpr int kBins = 2048;
constexpr size_t kEvictSmem = kRingBytes + 2 * kEvictThreads * 16;
constexpr int kHeldScores = kRingBytes / 4;                  // the ring holds the scores first

// An integer of the score's order, NaN below everything (equal zeros, whatever
// their sign).
__device__ __forceinline__ uint32_t score_key(float f) {
    const uint32_t u = __float_as_uint(f + 0.0f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kEvictThreads, 2) evict_kernel(const __grid_constant__ EvictArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_scan[2][2][kEvictWarps];
    __shared__ uint32_t s_pick[3];
    // the ring, before that the scores; the rows' places, before that the bins
    float* const s_score = reinterpret_cast<float*>(smem);
    longlong2* const s_row = reinterpret_cast<longlong2*>(smem + kRingBytes);  // [2][kEvictThreads] (from, to)
    uint32_t* const s_hist = reinterpret_cast<uint32_t*>(smem + kRingBytes);
    static_assert(kBins * 4 <= 2 * kEvictThreads * 16, "bins in the rows' place");
    const int C = a.cluster, rank = int(blockIdx.x) % C;
    const int h = int(blockIdx.x) / C, l = blockIdx.y, b = blockIdx.z;
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
    const bool lead = h == 0 && l == 0 && rank == 0;
    if (err && lead) atomicOr(a.status, err);
    if (__syncthreads_or(err != 0)) {
        if (rank == 0)
            for (int j = tid; j < a.budget; j += kEvictThreads) keep[j] = -1;
        if (lead && tid == 0) a.len_out[b] = a.in_place ? n : 0;
        return;
    }
    if (lead && tid == 0) a.len_out[b] = m;

    if (rank == 0) {
        const bool held = n <= kHeldScores;
        if (held) {
#pragma unroll 8
            for (int i = tid; i < n; i += kEvictThreads) s_score[i] = score[i];
        }
        for (int i = tid; i < kBins; i += kEvictThreads) s_hist[i] = 0;
        __syncthreads();
        auto score_at = [&](int i) { return held ? s_score[i] : score[i]; };

        // 1. the cut among the slots between the first and the last ones
        const int lo = n > a.budget ? a.n_sink : n, hi = n > a.budget ? n - a.n_recent : n;
        int need = a.budget - a.n_sink - a.n_recent;  // of those
        uint32_t from = 0xffffffffu;                  // keys from here on stay (no score's is that large)
        uint32_t cut = 0;                             // and of those equal to this one
        int ties = 0;                                 // so many, the first ones
        if (n > a.budget && need > 0) {
            uint32_t prefix = 0;
            for (int shift = 21;; shift -= 11) {  // bits 31..21, 20..10, 9..0
                const int at = max(shift, 0), bits = shift < 0 ? 10 : 11;
                for (int i = lo + tid; i < hi; i += kEvictThreads) {
                    const uint32_t k = score_key(score_at(i));
                    if (shift == 21 || (k >> (at + bits)) == (prefix >> (at + bits)))
                        atomicAdd(&s_hist[(k >> at) & ((1u << bits) - 1)], 1u);
                }
                __syncthreads();
                // the bin, from the top, where the count reaches `need`: four bins a thread
                constexpr int kPer = kBins / kEvictThreads;
                uint32_t own[kPer], sum = 0;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    uint32_t& bin = s_hist[kBins - 1 - (tid * kPer + i)];
                    sum += own[i] = bin;
                    bin = 0;  // for the next pass
                }
                uint32_t upto = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_up_sync(kFull, upto, d);
                    if (lane >= d) upto += o;
                }
                if (lane == 31) s_scan[0][0][warp] = int(upto);
                __syncthreads();
                uint32_t before = upto - sum;
#pragma unroll
                for (int w = 0; w < kEvictWarps; ++w)
                    if (w < warp) before += uint32_t(s_scan[0][0][w]);
                if (before < uint32_t(need) && before + sum >= uint32_t(need)) {
                    int i = 0;
                    uint32_t count = own[0];
#pragma unroll
                    for (int x = 0; x < kPer - 1; ++x)
                        if (i == x && before + own[x] < uint32_t(need)) before += own[x], count = own[x + 1], ++i;
                    s_pick[0] = uint32_t(kBins - 1 - (tid * kPer + i));
                    s_pick[1] = before;
                    s_pick[2] = count;
                }
                __syncthreads();
                prefix |= s_pick[0] << at;
                need -= int(s_pick[1]);
                if (s_pick[2] == uint32_t(need)) {  // all of the bin stays: its lower bits do not matter
                    from = prefix;
                    break;
                }
                if (shift < 0) {
                    from = prefix + 1;
                    cut = prefix;
                    ties = need;
                    break;
                }
            }
        }

        // 2. places: kept slots before a slot = those above the cut + the ties taken. A warp
        // takes 32 kRun slots in a row of each tile, so that one barrier serves them all
        constexpr int kRun = 8;
        int base_above = 0, base_tie = 0;
        for (int i0 = 0, turn = 0; i0 < n; i0 += kRun * kEvictThreads, turn ^= 1) {
            const int first = i0 + warp * (32 * kRun) + lane;
            uint32_t ma[kRun], mt[kRun];
            float x[kRun];
            int ca = 0, ct = 0;
#pragma unroll
            for (int u = 0; u < kRun; ++u) {
                const int i = first + u * 32;
                bool above = false, tie = false;
                x[u] = 0.0f;
                if (i < n) {
                    x[u] = score_at(i);
                    if (i < lo || i >= hi) {
                        above = true;
                    } else {
                        const uint32_t k = score_key(x[u]);
                        above = k >= from;
                        tie = k == cut && ties > 0;
                    }
                }
                ma[u] = __ballot_sync(kFull, above);
                mt[u] = __ballot_sync(kFull, tie);
                ca += __popc(ma[u]);
                ct += __popc(mt[u]);
            }
            if (lane == 0) {
                s_scan[turn][0][warp] = ca;
                s_scan[turn][1][warp] = ct;
            }
            __syncthreads();  // also: the tile's scores are read before any is written
            int pa = base_above, pt = base_tie;
#pragma unroll
            for (int w = 0; w < kEvictWarps; ++w) {
                const int wa = s_scan[turn][0][w], wt = s_scan[turn][1][w];
                if (w < warp) pa += wa, pt += wt;
                base_above += wa;
                base_tie += wt;
            }
            const uint32_t below = (1u << lane) - 1;
#pragma unroll
            for (int u = 0; u < kRun; ++u) {
                const int t = pt + __popc(mt[u] & below);
                if (((ma[u] >> lane) & 1u) || (((mt[u] >> lane) & 1u) && t < ties)) {
                    const int j = pa + __popc(ma[u] & below) + min(t, ties);
                    keep[j] = first + u * 32;
                    score_out[j] = x[u];
                }
                pa += __popc(ma[u]);
                pt += __popc(mt[u]);
            }
        }
        for (int j = m + tid; j < a.budget; j += kEvictThreads) keep[j] = -1;
        for (int64_t j = m + tid; j < a.score_stride; j += kEvictThreads) score_out[j] = 0.0f;
    }
    if (C > 1) {
        cluster_arrive();
        cluster_wait();
    }
    __syncthreads();

    // 3. rows. Their places are looked up by a thread each, for so many tiles at a time
    const int lanes = a.head_dim / 8 / C, per = kEvictThreads / lanes;  // threads a row, rows a tile
    const int group = kEvictThreads / per;                          // tiles whose rows a lookup covers
    const int my = tid / lanes, v = tid - my * lanes;
    const int64_t part = int64_t(h) * a.head_dim + (rank * lanes + v) * 8;
    const uint16_t* const sk = a.src.k + int64_t(l) * a.src.layer_stride + part;
    const uint16_t* const sv = a.src.v + (sk - a.src.k);
    uint16_t* const dk = a.dst.k + int64_t(l) * a.dst.layer_stride + part;
    uint16_t* const dv = a.dst.v + (dk - a.dst.k);
    const uint32_t ring = smem_u32(smem) + uint32_t(tid) * 16;  // a tile: the threads' vectors of K, then of V
    auto look_up = [&](int c) {
        const int j = c * group * per + tid;
        longlong2 r = make_longlong2(-1, -1);
        if (tid < group * per && j < m) {
            const int i = keep[j];
            uint32_t e = 0;
            if (!a.in_place || i != j) r = make_longlong2(slot_row(a.src, b, i, e), slot_row(a.dst, b, j, e));
        }
        s_row[(c & 1) * kEvictThreads + tid] = r;
    };
    const int n_tiles = (m + per - 1) / per;
    look_up(0);
    int64_t to[kRing];
    int c = 0, in = 0;  // the lookup in use, and the next tile's place in it
    for (int t0 = 0; t0 < n_tiles + kRing - 1; t0 += kRing) {
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            const int t = t0 + u;
            if (t < n_tiles) {
                if (in == 0) {
                    __syncthreads();  // lookup c is there, and c - 1 no longer needed
                    look_up(c + 1);
                }
                to[u] = -1;
                if (my < per) {
                    const longlong2 r = s_row[(c & 1) * kEvictThreads + in * per + my];
                    to[u] = r.y;
                    if (r.x >= 0) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + uint32_t(u) * (kEvictThreads * 32)),
                                     "l"(sk + r.x)
                                     : "memory");
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + uint32_t(u) * (kEvictThreads * 32) + kEvictThreads * 16),
                                     "l"(sv + r.x)
                                     : "memory");
                    }
                }
                if (++in == group) in = 0, ++c;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            constexpr int kBack = kRing - 1;
            if (t >= kBack && t - kBack < n_tiles) {  // the tile kBack before has landed
                const int o = (u + 1) % kRing;
                asm volatile("cp.async.wait_group %0;" ::"n"(kBack) : "memory");
                if (a.in_place) __syncthreads();
                if (to[o] >= 0) {
                    uint4 x, y;
                    const uint32_t p = ring + uint32_t(o) * (kEvictThreads * 32);
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(p) : "memory");
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w) : "r"(p + kEvictThreads * 16) : "memory");
                    st_row(dk + to[o], x);
                    st_row(dv + to[o], y);
                }
            }
        }
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, int n_seqs, cudaStream_t stream) {
    const dim3 grid(unsigned(a.n_kv_heads * a.cluster), unsigned(a.n_layers), unsigned(n_seqs));
    const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(evict_kernel), kEvictSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl_clusters(evict_kernel, a.cluster, grid, dim3(kEvictThreads), kEvictSmem, stream, a);
}

}  // namespace prcr

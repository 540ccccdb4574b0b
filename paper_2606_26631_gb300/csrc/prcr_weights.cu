// Attention weight of one decode step's queries added to each slot's score:
//   score[b][l][h][s] = decay score[b][l][h][s] + sum over the query heads g of
//   KV head h of softmax_s(RoPE(q[b][l][g], (p, p, p)) . K[b][l][s][h] / sqrt(D)).
//
// A cluster of 1 to 8 CTAs takes one (sequence, layer, KV head) and reads its keys
// once (weights_kernel):
//  1. Warps stream tiles of 16 slots from global memory straight into the A
//     fragments of mma.sync m16n8k16 (the dot product does not depend on the
//     order of the dims, so a lane's 16-byte chunks of its two slots' rows are
//     fragments as they are), the next tile's loads in flight during this one's
//     products; columns are the group's query heads. bf16 operands hold 8
//     bits, so the float32 query is split into three of them: products with
//     the bf16 keys are exact to float32's accuracy. The logits stay in shared memory, [head][slot].
//  2. Maxima, then exp and sums, of each head over all slots; a cluster's CTAs write theirs into
//     one another's shared memory.
//  3. The slot's weights, normalised, are added to its score.
// Memory-bound: keys and scores are touched once. A warp has a tile (4 KB at
// head_dim 128) in flight behind the one in use; two CTAs of 8 warps fit an SM (6
// warps with three tiles each in flight were slower, and so was an L2 prefetch of the first
// slots beside the queries' angles). Measured with 8 heads of 128 in groups of 4, 36 layers:
// 16 sequences of up to 4096 slots 515 us, 5.6 TB/s; one of 933 slots 18.5 us,
// 3.9 TB/s: one wave, whose first rows wait for the queries and whose last for the sums.
// Where the logits of a sequence do not fit a cluster's shared memory (above 399,360 / group
// slots at head_dim 256, 417,792 at 64), they go through the workspace instead
// (weights_logits_kernel, weights_sum_kernel).
#include <algorithm>

#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"
#include "prcr_tc.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kWeightsThreads = 256;
constexpr int kSlotsPerCta = 128;

// The length that a sequence's weights cover, with what is wrong in err.
__device__ __forceinline__ int64_t weights_len(const WeightsArgs& a, int b, uint32_t& err) {
    int64_t len = a.seq_len[b];
    const int64_t p = a.q_pos[b];
    if (len < 0 || len > a.cache.capacity || len > a.max_len) {
        err |= PRCR_ST_CAPACITY;
        len = len < 0 ? 0 : min(a.cache.capacity, a.max_len);
    }
    if (p <= -2147483648LL || p >= 2147483648LL) {
        err |= PRCR_ST_POS_RANGE;
        len = 0;
    }
    return len;
}

__global__ void __launch_bounds__(kWeightsThreads) weights_logits_kernel(const __grid_constant__ WeightsArgs a) {
    extern __shared__ __align__(16) float q_s[];  // [group][D] rotated, scaled
    const int D = a.head_dim, P = D / 2, g = a.group;
    const int b = blockIdx.z, l = blockIdx.y / a.n_kv_heads, h = blockIdx.y % a.n_kv_heads;
    pdl_allow();
    pdl_wait();
    uint32_t err = 0;
    const int64_t len = weights_len(a, b, err), s0 = int64_t(blockIdx.x) * kSlotsPerCta;
    if (err && threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(a.status, err);
    if (s0 >= len) return;
    const int Hq = a.n_kv_heads * g;
    const uint16_t* q = a.q + ((int64_t(b) * a.n_layers + l) * Hq + h * g) * D;
    for (int i = threadIdx.x; i < P; i += kWeightsThreads) {
        float c, s;
        sincos_turns(double(a.q_pos[b]), a.turn_freq[i], &s, &c);
        for (int j = 0; j < g; ++j) {
            const float x = lo_f32(q[j * D + i]), y = lo_f32(q[j * D + i + P]);
            q_s[j * D + i] = fmaf(x, c, -y * s) * a.scale_log2;
            q_s[j * D + i + P] = fmaf(y, c, x * s) * a.scale_log2;
        }
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* out = a.logits + ((int64_t(b) * a.n_layers + l) * Hq + h * g) * a.max_len;
    err = 0;
    for (int64_t s = s0 + warp; s < min(len, s0 + kSlotsPerCta); s += kWeightsThreads / 32) {
        const int64_t row = slot_row(a.cache, b, s, err);
        const uint16_t* k = a.cache.k + row + int64_t(l) * a.cache.layer_stride + int64_t(h) * D;
        for (int j = 0; j < g; ++j) {
            float x = 0.0f;
            if (row >= 0)
                for (int i = lane; i < D; i += 32) x = fmaf(q_s[j * D + i], lo_f32(k[i]), x);
#pragma unroll
            for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(kFull, x, d);
            if (lane == 0) out[j * a.max_len + s] = row >= 0 ? x : -INFINITY;
        }
    }
    if (err && lane == 0) atomicOr(a.status, err);
}

__device__ __forceinline__ float block_max(float x, float* s) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, d));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    for (int w = 0; w < kWeightsThreads / 32; ++w) x = fmaxf(x, s[w]);
    return x;
}
__device__ __forceinline__ float block_sum(float x, float* s) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(kFull, x, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0f;
    for (int w = 0; w < kWeightsThreads / 32; ++w) x += s[w];
    return x;
}

__global__ void __launch_bounds__(kWeightsThreads) weights_sum_kernel(const __grid_constant__ WeightsArgs a) {
    __shared__ float s_red[kWeightsThreads / 32];
    const int h = blockIdx.x, l = blockIdx.y, b = blockIdx.z, g = a.group;
    pdl_allow();
    pdl_wait();
    uint32_t err = 0;
    const int64_t len = weights_len(a, b, err);
    const float* x = a.logits + ((int64_t(b) * a.n_layers + l) * a.n_kv_heads + h) * g * a.max_len;
    float* score = a.score + ((int64_t(b) * a.n_layers + l) * a.n_kv_heads + h) * a.score_stride;
    float mx[8], inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        mx[j] = 0.0f;
        inv[j] = 0.0f;
        if (j < g) {
            float m = -INFINITY, sum = 0.0f;
            for (int64_t s = threadIdx.x; s < len; s += kWeightsThreads) m = fmaxf(m, x[j * a.max_len + s]);
            m = block_max(m, s_red);
            if (m == -INFINITY) m = 0.0f;  // no readable slot: weights of zero
            for (int64_t s = threadIdx.x; s < len; s += kWeightsThreads) sum += exp2f(x[j * a.max_len + s] - m);
            sum = block_sum(sum, s_red);
            mx[j] = m;
            inv[j] = sum == 0.0f ? 0.0f : 1.0f / sum;
        }
    }
    for (int64_t s = threadIdx.x; s < len; s += kWeightsThreads) {
        float w = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < g) w += exp2f(x[j * a.max_len + s] - mx[j]) * inv[j];
        score[s] = a.decay == 0.0f ? w : fmaf(a.decay, score[s], w);
    }
}

// ---- one cluster per (sequence, layer, KV head) ----------------------------------------

constexpr int kWarps = 8;
constexpr int kMaxRanks = 8;

// floats between the logits of two heads: 4 mod 32, so that a fragment's lanes
// (8 slots x 4 pairs of heads) write to different banks
__host__ __device__ inline int logit_stride(int slots) { return (slots + 31) / 32 * 32 + 4; }

template <int D>
struct WeightsShape {
    static constexpr int kDims = D < 128 ? D : 128;  // dims of a load stage
    static constexpr int kParts = D / kDims;
    static constexpr int kLoads = kDims / 32;        // 16-byte chunks a lane reads of each of its two rows
    static constexpr int kSteps = D / 16;
    static constexpr size_t kFragBytes = size_t(3) * kSteps * 32 * sizeof(uint2);
};

__device__ __forceinline__ void st_peer(const float* p, int rank, float x) {
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}" ::"r"(smem_u32(p)),
                 "r"(rank), "f"(x)
                 : "memory");
}

// The NaN among a CTA's exponentials again, from float32 FMAs, and the heads' sums over the
// cluster: an infinite key times a later term of the query, of the other sign or 0, makes a
// NaN where the product with the whole query is an infinity (and a logit of -inf a weight of
// 0). A call, for the rare sum that is a NaN: a test of each logit in the kernel took 3 %
// longer. smem: the query's fragments, no longer needed, and the exponentials; s0, n: the
// CTA's slots; head: in, the maxima, out, the sums; peer: the cluster's CTAs' sums.
template <int D>
__device__ __noinline__ void exact_nans(const WeightsArgs& a, unsigned char* smem, int s0, int n, float* head, float (*peer)[8]) {
    const int C = a.cluster, H = a.n_kv_heads, unit = int(blockIdx.x) / C, h = unit % H, l = unit / H % a.n_layers, b = unit / (H * a.n_layers);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, stride = logit_stride(a.slots_per_cta);
    float* const q_s = reinterpret_cast<float*>(smem);  // [group][D]
    float* const e = reinterpret_cast<float*>(smem + WeightsShape<D>::kFragBytes);
    const uint16_t* const q = a.q + int64_t(unit) * a.group * D;
    for (int i = tid; i < a.group * (D / 2); i += kWarps * 32) {
        const int j = i / (D / 2), d = i % (D / 2);
        float s, c;
        sincos_turns(double(a.q_pos[b]), a.turn_freq[d], &s, &c);
        const float u = lo_f32(q[j * D + d]), v = lo_f32(q[j * D + d + D / 2]);
        q_s[j * D + d] = fmaf(u, c, -v * s) * a.scale_log2;
        q_s[j * D + d + D / 2] = fmaf(v, c, u * s) * a.scale_log2;
    }
    __syncthreads();
    const uint16_t* const k = a.cache.k + int64_t(l) * a.cache.layer_stride + int64_t(h) * D;
    for (int s = tid; s < n; s += kWarps * 32)
        for (int j = 0; j < a.group; ++j) {
            if (e[j * stride + s] == e[j * stride + s]) continue;
            uint32_t err = 0;
            const int64_t row = slot_row(a.cache, b, s0 + s, err);
            float x = row < 0 ? -INFINITY : 0.0f;
            for (int d = 0; d < D && row >= 0; ++d) x = fmaf(q_s[j * D + d], lo_f32(k[row + d]), x);
            // (plus infinity was not among the maxima: less itself it would be the NaN that it is here)
            e[j * stride + s] = x == INFINITY ? NAN : exp2_fast(x - head[j]);
        }
    __syncthreads();
    static_assert(kWarps == 8, "a warp a head");
    float sum = 0.0f;
    for (int s = lane; warp < a.group && s < n; s += 32) sum += e[warp * stride + s];
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
    if (C == 1) {
        if (lane == 0) head[warp] = sum;
    } else {
        if (lane < C) st_peer(&peer[int(blockIdx.x) % C][warp], lane, sum);
        cluster_arrive();
        cluster_wait();
        if (tid < 8) {
            float x = 0.0f;
            for (int r = 0; r < C; ++r) x += peer[r][tid];
            head[tid] = x;
        }
    }
    __syncthreads();
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 2) weights_kernel(const __grid_constant__ WeightsArgs a) {
    using Sh = WeightsShape<D>;
    constexpr int P = D / 2, KS = Sh::kSteps, LV = Sh::kLoads, PARTS = Sh::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float s_part[kWarps][8], s_peer[3][kMaxRanks][8];
    uint4* const frag = reinterpret_cast<uint4*>(smem);  // [3][KS / 2][32]: the query's B fragments of two k-steps
    float* const logit = reinterpret_cast<float*>(smem + Sh::kFragBytes);
    const int C = a.cluster, rank = int(blockIdx.x) % C;
    const int unit = int(blockIdx.x) / C;
    const int h = unit % a.n_kv_heads, l = unit / a.n_kv_heads % a.n_layers, b = unit / (a.n_kv_heads * a.n_layers);
    const int g = a.group, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, t = lane & 3;
    const int stride = logit_stride(a.slots_per_cta);
    if (C > 1) cluster_arrive();
    pdl_allow();
    pdl_wait();
    uint32_t err = 0;
    const int len = int(weights_len(a, b, err));
    const int64_t pos = a.q_pos[b];
    const int per = ((len + 15) / 16 + C - 1) / C * 16;  // slots of a CTA, at most slots_per_cta
    const int s0 = min(len, rank * per), n = min(len, s0 + per) - s0;
    const int n_pairs = (n + 31) / 32;  // a warp's turn is two tiles of 16 slots

    // keys: a lane looks up the row of one of the 32 slots, a turn ahead, its block
    // two; it reads 16-byte chunks of rows gid and gid + 8 of each tile
    const uint16_t* const kbase = a.cache.k + int64_t(l) * a.cache.layer_stride + int64_t(h) * D + t * 8;
    const int32_t* const bt = a.cache.block_table + int64_t(b) * a.cache.bt_stride;
    const bool paged = a.cache.kind == PRCR_CACHE_PAGED;
    auto block_of = [&](int i) -> int32_t {
        const int s = i * 32 + lane;
        return paged && s < n ? bt[block_index(a.cache, uint32_t(s0 + s))] : 0;
    };
    auto row_of = [&](int i, int32_t blk) -> int64_t {
        const int s = i * 32 + lane;
        if (s >= n) return -1;
        const int64_t row = row_in_block(a.cache, b, uint32_t(s0 + s), blk);
        if (row < 0) err |= PRCR_ST_NO_BLOCK;
        return row;
    };
    struct Stage {
        uint4 w0[LV], w1[LV];
    };
    auto load = [&](Stage& s, int64_t row, int half, int part) {
        const int64_t r0 = __shfl_sync(kFull, row, half * 16 + gid), r1 = __shfl_sync(kFull, row, half * 16 + 8 + gid);
        const uint16_t* const p0 = kbase + r0 + part * Sh::kDims;
        const uint16_t* const p1 = kbase + r1 + part * Sh::kDims;
#pragma unroll
        for (int u = 0; u < LV; ++u) {
            s.w0[u] = s.w1[u] = make_uint4(0, 0, 0, 0);
            if (r0 >= 0) s.w0[u] = ld_stream(p0 + 32 * u);
            if (r1 >= 0) s.w1[u] = ld_stream(p1 + 32 * u);
        }
    };
    int pair = warp;
    int64_t row = row_of(pair, block_of(pair));
    int32_t blk = block_of(pair + kWarps);
    Stage st[2];
    if (pair < n_pairs) load(st[0], row, 0, 0);

    // the group's queries, rotated and scaled, as fragments of three bf16 terms:
    // k-step j of lane group t covers dims 8 (t + 4 (j / 2)) + 4 (j % 2) + 0..3, as
    // the key chunks that the lane reads
    const uint16_t* q = a.q + ((int64_t(b) * a.n_layers + l) * a.n_kv_heads + h) * g * D;
    float* const q_s = logit;  // [8][D] until the fragments are made
    for (int i = tid; i < 8 * P; i += kWarps * 32) {
        const int j = i / P, d = i % P;
        float x = 0.0f, y = 0.0f;
        if (j < g) {
            float s, c;
            sincos_turns(double(pos), a.turn_freq[d], &s, &c);
            const float u = lo_f32(q[j * D + d]), v = lo_f32(q[j * D + d + P]);
            x = fmaf(u, c, -v * s) * a.scale_log2;
            y = fmaf(v, c, u * s) * a.scale_log2;
        }
        q_s[j * D + d] = x;
        q_s[j * D + d + P] = y;
    }
    __syncthreads();
    for (int i = tid; i < KS * 32; i += kWarps * 32) {
        const int j = i / 32, ln = i % 32;
        const float* x = q_s + (ln >> 2) * D + 8 * ((ln & 3) + 4 * (j >> 1)) + 4 * (j & 1);
        float v[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int term = 0; term < 3; ++term) {
            const uint2 f = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            reinterpret_cast<uint2*>(frag)[((term * KS + (j & ~1)) * 32 + 2 * ln) + (j & 1)] = f;
            v[0] -= lo_f32(f.x);
            v[1] -= hi_f32(f.x);
            v[2] -= lo_f32(f.y);
            v[3] -= hi_f32(f.y);
        }
    }
    __syncthreads();

    float mx[2] = {-INFINITY, -INFINITY};  // of heads 2t, 2t + 1
    float acc[3][4];
    auto products = [&](const Stage& s, int part) {
        if (part == 0) {
#pragma unroll
            for (int i = 0; i < 12; ++i) acc[i / 4][i % 4] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < LV; ++u) {
            const int j = (part * Sh::kDims / 16) + 2 * u;
#pragma unroll
            for (int term = 0; term < 3; ++term) {
                const uint4 f = frag[(term * (KS / 2) + (j >> 1)) * 32 + lane];
                mma_16816(acc[term], s.w0[u].x, s.w1[u].x, s.w0[u].y, s.w1[u].y, f.x, f.y);
                mma_16816(acc[term], s.w0[u].z, s.w1[u].z, s.w0[u].w, s.w1[u].w, f.z, f.w);
            }
        }
    };
    // the next stage is asked for, then this one's products are made; after a
    // tile's last part its logits are kept
    for (; pair < n_pairs; pair += kWarps) {
        const int64_t next = row_of(pair + kWarps, blk);
        blk = block_of(pair + 2 * kWarps);
        const uint32_t there = __ballot_sync(kFull, row >= 0);
#pragma unroll
        for (int i = 0; i < 2 * PARTS; ++i) {
            const int half = i / PARTS, part = i % PARTS;
            if (i + 1 < 2 * PARTS) load(st[(i + 1) & 1], row, (i + 1) / PARTS, (i + 1) % PARTS);
            else if (pair + kWarps < n_pairs) load(st[0], next, 0, 0);
            products(st[i & 1], part);
            if (part == PARTS - 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int head = 2 * t + (e & 1), s = half * 16 + (e >> 1) * 8 + gid;
                    const float x = (there >> s) & 1u ? acc[0][e] + (acc[1][e] + acc[2][e]) : -INFINITY;
                    if (head < g) logit[head * stride + pair * 32 + s] = x;
                    mx[e & 1] = fmaxf(mx[e & 1], x);
                }
            }
        }
        row = next;
    }

    // each head's maximum over the cluster
    auto join = [&](float v0, float v1, int which, auto op, float init, float (&out)[8]) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            v0 = op(v0, __shfl_xor_sync(kFull, v0, d));
            v1 = op(v1, __shfl_xor_sync(kFull, v1, d));
        }
        if (gid == 0) {
            s_part[warp][2 * t] = v0;
            s_part[warp][2 * t + 1] = v1;
        }
        __syncthreads();
        if (C > 1) {
            if (which == 0) cluster_wait();  // every CTA has begun
            if (tid < 8 * C) {
                float x = init;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) x = op(x, s_part[w][tid & 7]);
                st_peer(&s_peer[which][rank][tid & 7], tid >> 3, x);
            }
            cluster_arrive();
            cluster_wait();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = init;
            if (C > 1) {
                for (int r = 0; r < C; ++r) x = op(x, s_peer[which][r][j]);
            } else {
#pragma unroll
                for (int w = 0; w < kWarps; ++w) x = op(x, s_part[w][j]);
            }
            out[j] = x;
        }
        __syncthreads();
    };
    float m[8], inv[8];
    join(mx[0], mx[1], 0, [](float x, float y) { return fmaxf(x, y); }, -INFINITY, m);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (m[j] == -INFINITY) m[j] = 0.0f;  // no readable slot: weights of zero

    // exponentials in place of the logits, and their sums
    float sum[8] = {};
    for (int s = tid; s < n; s += kWarps * 32) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < g) {
                const float e = exp2_fast(logit[j * stride + s] - m[j]);
                logit[j * stride + s] = e;
                sum[j] += e;
            }
    }
    // (a lane ends with the warp's sums of heads 2t, 2t + 1 for `join`)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sum[j] += __shfl_xor_sync(kFull, sum[j], 1);
        sum[j] += __shfl_xor_sync(kFull, sum[j], 2);
    }
    const float v0 = t == 0 ? sum[0] : t == 1 ? sum[2] : t == 2 ? sum[4] : sum[6];
    const float v1 = t == 0 ? sum[1] : t == 1 ? sum[3] : t == 2 ? sum[5] : sum[7];
    join(v0, v1, 1, [](float x, float y) { return x + y; }, 0.0f, inv);
    float all = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) all += inv[j];
    if (all != all) {  // the same in all of the cluster's CTAs
        if (tid == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s_part[0][j] = m[j];
        }
        __syncthreads();
        exact_nans<D>(a, smem, s0, n, s_part[0], s_peer[2]);
#pragma unroll
        for (int j = 0; j < 8; ++j) inv[j] = s_part[0][j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = inv[j] == 0.0f ? 0.0f : 1.0f / inv[j];

    float* const score = a.score + int64_t(unit) * a.score_stride + s0;
#pragma unroll 4
    for (int s = tid; s < n; s += kWarps * 32) {
        float w = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < g) w = fmaf(logit[j * stride + s], inv[j], w);
        score[s] = a.decay == 0.0f ? w : fmaf(a.decay, score[s], w);
    }
    if (err && (rank == 0 || (err & PRCR_ST_NO_BLOCK))) atomicOr(a.status, err);
}

template <int D>
cudaError_t launch_cluster(const WeightsArgs& a, cudaStream_t stream) {
    const size_t smem = weights_smem(D, a.group, a.slots_per_cta);
    const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(weights_kernel<D>), smem);
    if (e != cudaSuccess) return e;
    const dim3 grid(unsigned(int64_t(a.n_seqs) * a.n_layers * a.n_kv_heads * a.cluster));
    return launch_pdl_clusters(weights_kernel<D>, a.cluster, grid, dim3(kWarps * 32), smem, stream, a);
}

}  // namespace

size_t weights_smem(int head_dim, int group, int slots) {
    const size_t frag = size_t(3) * (head_dim / 16) * 32 * sizeof(uint2);
    // (the queries lie in the logits' place first)
    return frag + std::max(size_t(group) * logit_stride(slots), size_t(8) * head_dim) * sizeof(float);
}

cudaError_t launch_weights(const WeightsArgs& a, cudaStream_t stream) {
    if (a.cluster > 0) {
        if (a.head_dim == 64) return launch_cluster<64>(a, stream);
        if (a.head_dim == 128) return launch_cluster<128>(a, stream);
        return launch_cluster<256>(a, stream);
    }
    const int64_t parts = (a.max_len + kSlotsPerCta - 1) / kSlotsPerCta;
    cudaError_t e = launch_pdl(weights_logits_kernel, dim3(unsigned(parts), unsigned(a.n_layers * a.n_kv_heads), unsigned(a.n_seqs)),
                               dim3(kWeightsThreads), size_t(a.group) * a.head_dim * sizeof(float), stream, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(weights_sum_kernel, dim3(unsigned(a.n_kv_heads), unsigned(a.n_layers), unsigned(a.n_seqs)),
                      dim3(kWeightsThreads), 0, stream, a);
}

}  // namespace prcr

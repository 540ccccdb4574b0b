// Attention weight of one decode step's queries added to each slot's score:
//   score[b][l][h][s] = decay score[b][l][h][s] + sum over the query heads g of
//   KV head h of softmax_s(RoPE(q[b][l][g], (p, p, p)) . K[b][l][s][h] / sqrt(D)).
//
// Two kernels: the logits to the workspace, then per (sequence, layer, KV head)
// the normalisers and the sums.
#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"

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

}  // namespace

cudaError_t launch_weights(const WeightsArgs& a, cudaStream_t stream) {
    const int64_t parts = (a.max_len + kSlotsPerCta - 1) / kSlotsPerCta;
    cudaError_t e = launch_pdl(weights_logits_kernel, dim3(unsigned(parts), unsigned(a.n_layers * a.n_kv_heads), unsigned(a.n_seqs)),
                               dim3(kWeightsThreads), size_t(a.group) * a.head_dim * sizeof(float), stream, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(weights_sum_kernel, dim3(unsigned(a.n_kv_heads), unsigned(a.n_layers), unsigned(a.n_seqs)),
                      dim3(kWeightsThreads), 0, stream, a);
}

}  // namespace prcr

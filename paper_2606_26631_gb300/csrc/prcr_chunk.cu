// Attention of a packed batch's new tokens over the decoder cache, one layer:
// query i of the n_b new tokens of sequence b sees the slots up to its own,
//   out = softmax(RoPE(q, (t, h, w)) K^T / sqrt(D)) V over slots [0, len_b - n_b + i].
#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;

// One query row by one warp in float32: online softmax over slots
// [lo, hi), E dims a lane (dims lane * E ..). m is in units of log2.
template <int D>
__device__ __forceinline__ void row_attention(const ChunkArgs& a, int b, int t, int hq, int64_t lo, int64_t hi,
                                              float& m, float& l, float (&o)[D / 32], uint32_t& err) {
    constexpr int E = D / 32, P = D / 2;
    const int lane = threadIdx.x & 31;
    const int kh = hq / a.group;
    const uint16_t* qr = a.q + int64_t(t) * a.q_stride + int64_t(hq) * D + lane * E;
    float q[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = lo_f32(qr[e]), y = __shfl_xor_sync(kFull, x, 16);  // the pair's other half
        const int i = (lane & 15) * E + e;
        float s, c;
        sincos_turns(double(a.coords[3 * int64_t(t) + pair_axis(i, a.layout, a.sec_t, a.sec_h, a.sec_w)]),
                     a.turn_freq[i], &s, &c);
        q[e] = (lane < 16 ? fmaf(x, c, -y * s) : fmaf(x, c, y * s)) * a.scale_log2;
    }
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    for (int64_t s = lo; s < hi; ++s) {
        const int64_t row = slot_row(a.cache, b, s, err);
        if (row < 0) continue;
        const uint16_t* k = a.cache.k + row + int64_t(kh) * D + lane * E;
        const uint16_t* v = a.cache.v + row + int64_t(kh) * D + lane * E;
        float x = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[e], lo_f32(k[e]), x);
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(kFull, x, d);
        const float mn = fmaxf(m, x);
        const float mu = mn == -INFINITY ? 0.0f : mn;
        const float r = exp2f(m - mu), p = exp2f(x - mu);
        m = mn;
        l = fmaf(l, r, p);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], r, p * lo_f32(v[e]));
    }
}

// The slots that token t of sequence b sees (at most the capacity and max_len).
__device__ __forceinline__ int64_t visible(const ChunkArgs& a, int b, int t, uint32_t& err) {
    const int64_t len = a.seq_len[b], top = min(a.cache.capacity, a.max_len);
    if (len < 0 || len > top) err |= PRCR_ST_CAPACITY;
    return max(int64_t(0), min(top, len - (a.q_off[b + 1] - 1 - t)));
}

template <int D>
__global__ void __launch_bounds__(256) chunk_rows_kernel(const __grid_constant__ ChunkArgs a) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const int Hq = a.n_kv_heads * a.group;
    const int64_t row = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
    pdl_allow();
    pdl_wait();
    if (__syncthreads_or(bad_offsets(a.q_off, a.n_seqs, a.total_q))) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, PRCR_ST_CSR);
        return;
    }
    if (row >= int64_t(a.total_q) * Hq) return;
    const int t = int(row / Hq), hq = int(row - int64_t(t) * Hq);
    const int b = sequence_of(a.q_off, a.n_seqs, t);
    if (t >= a.q_off[b + 1]) return;  // behind the last sequence
    uint32_t err = 0;
    float m, l, o[E];
    row_attention<D>(a, b, t, hq, 0, visible(a, b, t, err), m, l, o, err);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t* out = a.out + int64_t(t) * a.out_stride + int64_t(hq) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(out + e) = pack_bf16x2(o[e] * inv, o[e + 1] * inv);
    if (err && lane == 0) atomicOr(a.status, err);
}

}  // namespace

cudaError_t launch_chunk(const ChunkArgs& a, cudaStream_t stream) {
    const int64_t rows = int64_t(a.total_q) * a.n_kv_heads * a.group;
    const dim3 grid(unsigned((rows + 7) / 8));
    if (a.head_dim == 64) return launch_pdl(chunk_rows_kernel<64>, grid, dim3(256), 0, stream, a);
    if (a.head_dim == 128) return launch_pdl(chunk_rows_kernel<128>, grid, dim3(256), 0, stream, a);
    return launch_pdl(chunk_rows_kernel<256>, grid, dim3(256), 0, stream, a);
}

}  // namespace prcr

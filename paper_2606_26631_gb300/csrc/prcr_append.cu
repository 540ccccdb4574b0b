// Rows of new tokens into the decoder cache: for a packed batch of sequences,
// K = RoPE(k_raw, (t, h, w)) and V unchanged to the slots behind each
// sequence's length, every layer of the call.
//
// Memory-bound: each row is read once and written once (4 x head_dim bytes each
// way per K/V pair and head). As in the capture kernel a thread holds one 16-byte vector of a
// token's key, its rotate-half partner and the two vectors of the value, and
// walks its layers with the next one's rows requested before the current
// ones are written; the cos/sin of a token are computed once per CTA for all
// heads and the CTA's layers. Measured: six prompts of up to 2116 tokens, 28 layers of
// 4 heads of 128, 168 us, 6.1 TB/s (a CTA takes up to 8 layers; up to 2, 190 us: each
// computes its tokens' angles again); one token each of 16 sequences, 36 layers of 8
// heads, 4 us in a graph, 9 from Python, all latency.
#include "prcr_cache.cuh"
#include "prcr_pdl.cuh"

namespace prcr {
namespace {

__global__ void __launch_bounds__(512) append_kernel(const __grid_constant__ AppendArgs a) {
    extern __shared__ __align__(16) float smem[];
    const int P = a.head_dim >> 1;
    const int T = a.tok_per_cta;
    float* cos_s = smem;
    float* sin_s = smem + T * P;
    int64_t* dst_s = reinterpret_cast<int64_t*>(sin_s + T * P);
    const int tok0 = blockIdx.x * T;

    const int my_t = threadIdx.x / a.lanes;
    const int lane = threadIdx.x - my_t * a.lanes;
    const int my_j = tok0 + my_t;
    const bool act = my_t < T && my_j < a.total;
    const int vph = a.head_dim >> 4;
    const int h = lane / vph;
    const int v = lane - h * vph;
    const int64_t off = int64_t(h) * a.head_dim + v * 8;
    const int l0 = blockIdx.y * a.layers_per_cta;
    const int l1 = min(l0 + a.layers_per_cta, a.n_layers);
    const int64_t s_off = int64_t(l0) * a.src_layer_stride + int64_t(my_j) * a.src_token_stride + off;
    const uint16_t* sk = a.src_k + s_off;
    const uint16_t* sv = a.src_v + s_off;
    uint4 k0, k1, v0, v1;
    auto load = [&]() {
        k0 = ld_stream(sk);
        k1 = ld_stream(sk + P);
        v0 = ld_stream(sv);
        v1 = ld_stream(sv + P);
    };
    pdl_allow();
    pdl_wait();
    if (act) load();

    // the tokens' rows: a warp finds a token's sequence with 32 probes a round
    uint32_t err = 0;
    // (a block's last warp may not be whole and takes none; a block has 129 threads
    // at least)
    const int warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    for (int t = warp; warp < n_warps && t < T; t += n_warps) {
        const int j = tok0 + t;
        int64_t dst = -1;
        if (j < a.total) {
            const int b = sequence_of(a.tok_off, a.n_seqs, j);
            const int first = a.tok_off[b];
            if (j >= first && j < a.tok_off[b + 1]) {
                const int len = a.len_in[b];
                uint32_t e = 0;
                if (len < 0) e = PRCR_ST_CAPACITY;
                else dst = slot_row(a.cache, b, int64_t(len) + (j - first), e);
                err |= e;
            }
        }
        if ((threadIdx.x & 31) == 0) dst_s[t] = dst;
    }
    for (int q = threadIdx.x; q < T * P; q += blockDim.x) {
        const int t = q / P;
        const int i = q - t * P;
        const int j = tok0 + t;
        float c = 1.0f, s = 0.0f;
        if (j < a.total) {
            const int ax = pair_axis(i, a.layout, a.sec_t, a.sec_h, a.sec_w);
            sincos_turns(double(a.coords[3 * int64_t(j) + ax]), a.turn_freq[i], &s, &c);
        }
        cos_s[q] = c;
        sin_s[q] = s;
    }
    const bool bad = __syncthreads_or(bad_offsets(a.tok_off, a.n_seqs, a.total));
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        if (bad && threadIdx.x == 0) atomicOr(a.status, PRCR_ST_CSR);
        for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
            a.len_out[b] = a.len_in[b] + (bad ? 0 : a.tok_off[b + 1] - a.tok_off[b]);
    }
    if (bad) return;
    if (err && blockIdx.y == 0 && (threadIdx.x & 31) == 0) atomicOr(a.status, err);
    if (!act) return;
    const int64_t dst = dst_s[my_t];
    if (dst < 0) return;
    float c[8], s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float4 c4 = *reinterpret_cast<const float4*>(cos_s + my_t * P + v * 8 + 4 * u);
        const float4 s4 = *reinterpret_cast<const float4*>(sin_s + my_t * P + v * 8 + 4 * u);
        c[4 * u] = c4.x; c[4 * u + 1] = c4.y; c[4 * u + 2] = c4.z; c[4 * u + 3] = c4.w;
        s[4 * u] = s4.x; s[4 * u + 1] = s4.y; s[4 * u + 2] = s4.z; s[4 * u + 3] = s4.w;
    }
    const int64_t c_off = dst + int64_t(l0) * a.cache.layer_stride + off;
    uint16_t* ck = a.cache.k + c_off;
    uint16_t* cv = a.cache.v + c_off;
    for (int l = l0; l < l1; ++l) {
        const uint4 x0 = k0, x1 = k1, y0 = v0, y1 = v1;
        sk += a.src_layer_stride;
        sv += a.src_layer_stride;
        if (l + 1 < l1) load();
        uint4 o0, o1;
        rotate_vec(x0, x1, c, s, o0, o1);
        st_row(ck, o0);
        st_row(ck + P, o1);
        st_row(cv, y0);
        st_row(cv + P, y1);
        ck += a.cache.layer_stride;
        cv += a.cache.layer_stride;
    }
}

}  // namespace

cudaError_t append_blocks_per_sm(int block, size_t smem, int* out) {
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(out, append_kernel, block, smem);
}

cudaError_t launch_append(const AppendArgs& a, dim3 grid, int block, size_t smem, cudaStream_t stream) {
    return launch_pdl(append_kernel, grid, dim3(block), smem, stream, a);
}

}  // namespace prcr

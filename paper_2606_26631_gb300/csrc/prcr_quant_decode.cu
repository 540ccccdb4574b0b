// One new token of each sequence over a quantised cache: for every sequence, layer
// and query head
//   o = sum_s p_s V_s,   p = softmax(RoPE(q, (p, p, p)) K^T / sqrt(D)),
// with K and V the codes' values times their groups' powers of two.
//
// Memory-bound in bytes, but only just: a code costs a conversion beside its
// product, and a byte of codes brings two or four times a bf16 byte's products.
// So nothing passes through shared memory on its way: a warp loads its tiles'
// codes straight into the registers in which the matrix instructions want them,
// the next tile's as soon as a tile's are used up.
//   S^T (16 slots x 8 heads) = K Q^T. The order of the dims in a dot product is
//     free, so lane t of a slot's four takes 16-byte pieces t, t + 4, ... of its
//     row; four dims in a lane are one k-step's share.
//   O^T (16 dims x 8 heads) += V^T P^T. Which dims are the rows of which product is free
//     too: lane group r takes piece r of the rows of four slots, and interleaving the
//     bytes of two slots gives the pairs along the slots that the product sums over.
// Codes are exact in fp16, in which they enter. The query (scaled by a power of
// two to at most 2^14) and the weights enter as two fp16 each, 22 bits; with up to four
// heads to a group the two lie side by side in the product's eight columns, so that one
// product takes both.
// Scales never touch the codes: E4M3's of a key multiplies the slot's logits, E2M1's the
// partial sums of their groups' k-steps; a value's goes into the weight's exponent, per
// group in E2M1 (whose groups take every (D/32)-th quad of dims, so that each
// lane's piece of a row has quads of all groups).
// Weights are therefore kept against two references, both powers of two: p = 2^(x - m)
// for the sum, w = 2^(x + e - r + 11) for the accumulator, e the value's scale. m and r follow the
// largest x and x + e, but only when one is more than 2^4 past them, so that most tiles
// rescale nothing and need no reduction over the lanes; w stays below 2^15, and what fp16 loses
// of it is 2^-36 of the largest at most.
#include <cuda_fp16.h>

#include "prcr_pdl.cuh"
#include "prcr_quant.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr float kNone = -3.0e38f;   // reference of no slot yet: below every logit, and finite
constexpr float kSlack = 4.0f;      // log2 of how far past its reference a weight may go
constexpr float kWeightLog2 = 11.0f;
constexpr int kMaxWarps = 16;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Two floats as fp16 pairs: a head and the rounded remainder.
__device__ __forceinline__ void split_f16x2(float x0, float x1, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16x2(x0, x1);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    lo = pack_f16x2(x0 - h.x, x1 - h.y);
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Transpose of an 8 x 8 matrix of 16-bit values held as mma fragments.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// N words from p, or zeros.
template <int N>
__device__ __forceinline__ void load_codes(uint32_t* w, const uint8_t* p, bool ok) {
    static_assert(N == 1 || N == 2 || N == 4, "4, 8 or 16 bytes");
    if constexpr (N == 4) {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %5, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\nmov.b32 %2, 0;\nmov.b32 %3, 0;\n"
                     "@p ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                     : "=&r"(w[0]), "=&r"(w[1]), "=&r"(w[2]), "=&r"(w[3]) : "l"(p), "r"(int(ok)));
    } else if constexpr (N == 2) {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %3, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\n"
                     "@p ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];\n}"
                     : "=&r"(w[0]), "=&r"(w[1]) : "l"(p), "r"(int(ok)));
    } else {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.nc.L1::no_allocate.u32 %0, [%1];\n}"
                     : "=&r"(w[0]) : "l"(p), "r"(int(ok)));
    }
}

// Sizes of a format's rows: RB bytes of codes; a warp takes SUB x 16 slots at once.
template <int FMT, int D> struct Shape {
    static constexpr bool kFour = FMT == PRCR_QFMT_E2M1;
    static constexpr int RB = kFour ? D / 2 : D;
    static constexpr int SUB = RB >= 128 ? 1 : 128 / RB;
    static constexpr int TS = 16 * SUB;
    static constexpr int N = kFour ? D / 32 : 1;  // scales of a row
    static constexpr int KW = RB / 16, VW = RB / 32;  // a lane's words of a row
    static constexpr int KS = D / 16;  // k-steps of S^T, products of O^T
    static constexpr int SW = (N + 3) / 4;  // words of a row's scales
    static constexpr int OWN = (TS + 31) / 32;  // slots that a lane looks up
    static constexpr int kThreads = D == 256 ? 256 : 512;
    // the dim of word i's first code in lane t of a key's row, and in lane group r of a value's
    static __device__ __forceinline__ int kdim(int t, int i) {
        const int byte = RB >= 64 ? 16 * (t + 4 * (i / 4)) + 4 * (i % 4) : 8 * t + 4 * i;
        return kFour ? 2 * byte : byte;
    }
    static __device__ __forceinline__ int vdim(int r, int i) {
        const int byte = RB == 256 ? 128 * (i / 4) + 16 * r + 4 * (i % 4) : r * (RB / 8) + 4 * i;
        return kFour ? 2 * byte : byte;
    }
};

// What a lane knows of a slot that it looked up.
template <int SW> struct Slot {
    int64_t codes;       // -1: not there
    uint32_t ks[SW], vs[SW];  // scales' bytes
    float bias;          // added to a logit: 0, -inf for a slot that is not there, NaN for a key that reads as NaN
    float kf, ve;        // E4M3: the key's scale; the value's exponent (E2M1: the largest of its groups')
};

template <int FMT, int D, bool PAIR>
__global__ void __launch_bounds__(Shape<FMT, D>::kThreads, 1) decode_quant_kernel(const __grid_constant__ DecodeQuantArgs a) {
    using S = Shape<FMT, D>;
    constexpr bool kFour = S::kFour;
    constexpr int SUB = S::SUB, TS = S::TS, N = S::N, KW = S::KW, VW = S::VW, KS = S::KS, SW = S::SW, OWN = S::OWN;
    constexpr int P = D / 2, PITCH = D + 4, QP = PAIR ? 1 : 2, LS = PAIR ? 1 : 2;  // query pieces in registers, slots of a lane's logits
    extern __shared__ __align__(16) float smem[];
    __shared__ float s_cos[P], s_sin[P], s_qs[8];
    __shared__ float s_m[kMaxWarps][8], s_l[kMaxWarps][8], s_r[kMaxWarps][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, t = lane & 3, W = blockDim.x >> 5;
    const int H = a.n_kv_heads, g = a.group;
    // this CTA's part: of a (sequence, layer) and split, heads fastest
    uint32_t unit = blockIdx.x;
    const int kh = int(unit % uint32_t(H));
    unit /= uint32_t(H);
    const int split = int(unit % uint32_t(a.splits));
    unit /= uint32_t(a.splits);
    const int l = int(unit % uint32_t(a.n_layers)), b = int(unit / uint32_t(a.n_layers));
    const int64_t head0 = ((int64_t(b) * a.n_layers + l) * H + kh) * g;  // this group's first query head
    pdl_wait();
    const int64_t pos = a.q_pos[b];
    int len = a.seq_len[b];
    uint32_t err = 0;
    if (len < 0 || len > a.max_len) {  // (max_len is at most the capacity)
        err |= PRCR_ST_CAPACITY;
        len = len < 0 ? 0 : a.max_len;
    }
    if (pos <= -2147483648LL || pos >= 2147483648LL) {
        err |= PRCR_ST_POS_RANGE;
        len = 0;
    }
    const int s_begin = min(len, split * a.chunk), s_end = min(len, s_begin + a.chunk);
    const int tiles = (s_end - s_begin + TS - 1) / TS;
    if (tiles == 0 && a.splits > 1) {
        for (int h = threadIdx.x; h < g; h += blockDim.x)
            *reinterpret_cast<float2*>(a.partial + ((head0 + h) * a.splits + split) * (D + 2) + D) = make_float2(kNone, 0.0f);
        if (err && threadIdx.x == 0) atomicOr(a.status, err);
        return;
    }
    const int64_t head_codes = int64_t(l) * a.cache.layer_stride + int64_t(kh) * S::RB;
    const int64_t head_scales = int64_t(l) * a.cache.scale_layer_stride + int64_t(kh) * N;
    const uint8_t *kb = a.cache.k + head_codes, *vb = a.cache.v + head_codes;
    const uint8_t *kf = a.cache.k_scale + head_scales, *vf = a.cache.v_scale + head_scales;

    // A lane looks up slots (lane + 32 j) % TS of a tile: its block, then where it lies.
    auto slot_of = [&](int tile, int j) { return s_begin + tile * TS + (TS == 16 ? lane & 15 : lane + 32 * j); };
    auto blocks = [&](int tile, int32_t (&blk)[OWN]) {
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int s = slot_of(tile, j);
            blk[j] = tile < tiles && s < s_end ? qblock(a.cache, b, uint32_t(s)) : -1;
        }
    };
    Slot<SW> own[OWN];
    int64_t scales_at[OWN];
    auto places = [&](int tile, const int32_t (&blk)[OWN]) {
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int s = slot_of(tile, j);
            own[j].codes = -1;
            scales_at[j] = 0;
            if (tile < tiles && s < s_end) {
                const QPlace p = qplace_in_block(a.cache, b, uint32_t(s), blk[j]);
                if (p.codes < 0) err |= PRCR_ST_NO_BLOCK;
                own[j].codes = p.codes;
                scales_at[j] = p.scales;
            }
        }
    };
    auto load_scales = [&]() {
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const bool ok = own[j].codes >= 0;
            const uint8_t *pk = kf + scales_at[j], *pv = vf + scales_at[j];
            if constexpr (N == 8) {
                load_codes<2>(own[j].ks, pk, ok);
                load_codes<2>(own[j].vs, pv, ok);
            } else if constexpr (N == 4) {
                load_codes<1>(own[j].ks, pk, ok);
                load_codes<1>(own[j].vs, pv, ok);
            } else if constexpr (N == 2) {
                own[j].ks[0] = ok ? *reinterpret_cast<const uint16_t*>(pk) : 0u;
                own[j].vs[0] = ok ? *reinterpret_cast<const uint16_t*>(pv) : 0u;
            } else {
                own[j].ks[0] = ok ? *pk : 0u;
                own[j].vs[0] = ok ? *pv : 0u;
            }
        }
    };
    const uint8_t* kl = kb + (S::RB >= 64 ? 16 * t : 8 * t);
    const uint8_t* vl = vb + gid * (S::RB == 256 ? 16 : S::RB / 8);
    uint32_t kw[SUB][2][KW], vw[SUB][4][VW];
    auto load_k = [&]() {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int64_t at = __shfl_sync(kFull, own[u / 2].codes, (16 * u + gid + 8 * i) & 31);
                if constexpr (KW >= 4) {
#pragma unroll
                    for (int c = 0; c < KW / 4; ++c) load_codes<4>(kw[u][i] + 4 * c, kl + at + 64 * c, at >= 0);
                } else {
                    load_codes<KW>(kw[u][i], kl + at, at >= 0);
                }
            }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t at = __shfl_sync(kFull, own[u / 2].codes, (16 * u + 2 * t + (i & 1) + 8 * (i >> 1)) & 31);
                if constexpr (VW >= 4) {
#pragma unroll
                    for (int c = 0; c < VW / 4; ++c) load_codes<4>(vw[u][i] + 4 * c, vl + at + 128 * c, at >= 0);
                } else {
                    load_codes<VW>(vw[u][i], vl + at, at >= 0);
                }
            }
    };

    // the first tile is requested before the query is read
    int32_t blk[OWN];
    blocks(warp, blk);
    places(warp, blk);
    load_k();
    load_scales();
    load_v();
    blocks(warp + W, blk);

    // the group's queries, rotated at (p, p, p): pair i turns by p * rate i whatever its band
    for (int i = threadIdx.x; i < P; i += blockDim.x) sincos_turns(double(pos), a.turn_freq[i], &s_sin[i], &s_cos[i]);
    __syncthreads();
    for (int h = warp; h < g; h += W) {
        const uint16_t* q = a.q + (head0 + h) * D;
        float x[P / 32], y[P / 32];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            const int d = lane + 32 * i;
            const float qx = __uint_as_float(uint32_t(q[d]) << 16), qy = __uint_as_float(uint32_t(q[d + P]) << 16);
            x[i] = fmaf(qx, s_cos[d], -qy * s_sin[d]) * a.scale_log2;
            y[i] = fmaf(qy, s_cos[d], qx * s_sin[d]) * a.scale_log2;
            most = max(most, max(__float_as_uint(x[i]) & 0x7fffffffu, __float_as_uint(y[i]) & 0x7fffffffu));
        }
        most = __reduce_max_sync(kFull, most);
        // times 2^up: below 2^14 (2^40 at most, so that a logit times it stays finite)
        const int up = min(40, 13 - (int(most >> 23) - 127));
        const float f = __uint_as_float(uint32_t(127 + up) << 23);
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            smem[h * PITCH + lane + 32 * i] = x[i] * f;
            smem[h * PITCH + lane + 32 * i + P] = y[i] * f;
        }
        if (lane == 0) s_qs[h] = __uint_as_float(uint32_t(127 - up) << 23);
    }
    __syncthreads();
    // B fragments: column r is head r, or with pairs head r % 4, of its first or second piece
    uint32_t qf[KS][QP][2];
    {
        const int h = PAIR ? gid & 3 : gid;
        const bool hv = h < g;
        const float* qr = smem + (hv ? h : 0) * PITCH;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const float4 x = *reinterpret_cast<const float4*>(qr + (kFour ? S::kdim(t, j >> 1) + 4 * (j & 1) : S::kdim(t, j)));
            uint32_t h0, l0, h1, l1;
            split_f16x2(hv ? x.x : 0.0f, hv ? x.y : 0.0f, h0, l0);
            split_f16x2(hv ? x.z : 0.0f, hv ? x.w : 0.0f, h1, l1);
            if (PAIR) {
                qf[j][0][0] = gid < 4 ? h0 : l0;
                qf[j][0][1] = gid < 4 ? h1 : l1;
            } else {
                qf[j][0][0] = h0;
                qf[j][0][1] = h1;
                qf[j][QP - 1][0] = l0;
                qf[j][QP - 1][1] = l1;
            }
        }
    }
    // this lane's heads are h0 and h0 + 1, in S^T's columns and in O^T's
    const int h0 = PAIR ? 2 * (t & 1) : 2 * t;
    const float qs[2] = {h0 < g ? s_qs[h0] : 0.0f, h0 + 1 < g ? s_qs[h0 + 1] : 0.0f};

    float o[KS][4];
#pragma unroll
    for (int j = 0; j < KS; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
    float m[2] = {kNone, kNone}, r[2] = {kNone, kNone}, sum[2] = {0.0f, 0.0f};

    for (int tile = warp; tile < tiles; tile += W) {
        // what the lanes know of this tile's slots
        bool v_nan = false;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            Slot<SW>& w = own[j];
            if (kFour) {
                bool nan = false;
                int top = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int bk = (w.ks[i / 4] >> (8 * (i % 4))) & 255, bv = (w.vs[i / 4] >> (8 * (i % 4))) & 255;
                    nan |= bk == kScaleNan;
                    v_nan |= bv == kScaleNan;
                    top = max(top, bv == kScaleNan ? 0 : bv);
                }
                w.ve = float(top - 127);
                w.bias = w.codes < 0 ? -INFINITY : nan ? __uint_as_float(0x7fffffffu) : 0.0f;
            } else {
                w.kf = w.codes < 0 ? 0.0f : scale_value(int(w.ks[0]));
                w.ve = w.vs[0] == kScaleNan ? __uint_as_float(0x7fffffffu) : float(int(w.vs[0]) - 127);
                w.bias = w.codes < 0 ? -INFINITY : 0.0f;
            }
        }
        v_nan = kFour && __any_sync(kFull, v_nan);

        float x[SUB][LS][2], ve[SUB][LS];
        uint32_t vs[SUB][LS][SW];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            float c[kFour ? N : 2][4];
#pragma unroll
            for (int j = 0; j < (kFour ? N : 2); ++j) c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.0f;
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                if constexpr (kFour) {
                    uint32_t p[4], q[4];
                    f16_of_e2m1(kw[u][0][i], p);
                    f16_of_e2m1(kw[u][1][i], q);
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int z = 0; z < QP; ++z)
                            mma_f16(c[(2 * i + e) % N], p[2 * e], q[2 * e], p[2 * e + 1], q[2 * e + 1], qf[2 * i + e][z][0], qf[2 * i + e][z][1]);
                } else {
                    uint32_t p[2], q[2];
                    f16_of_e4m3(kw[u][0][i], p);
                    f16_of_e4m3(kw[u][1][i], q);
#pragma unroll
                    for (int z = 0; z < QP; ++z) mma_f16(c[(i + z) & 1], p[0], q[0], p[1], q[1], qf[i][z][0], qf[i][z][1]);
                }
            }
            float d[4];
            if constexpr (kFour) {
                d[0] = d[1] = d[2] = d[3] = 0.0f;
#pragma unroll
                for (int k = 0; k < SW; ++k) {
                    const uint32_t wa = __shfl_sync(kFull, own[u / 2].ks[k], (16 * u + gid) & 31);
                    const uint32_t wb = __shfl_sync(kFull, own[u / 2].ks[k], (16 * u + gid + 8) & 31);
#pragma unroll
                    for (int i = 4 * k; i < min(N, 4 * k + 4); ++i) {
                        // the byte as a float's exponent
                        const float fa = __uint_as_float((i % 4 == 3 ? wa >> 1 : wa << (23 - 8 * (i % 4))) & 0x7f800000u);
                        const float fb = __uint_as_float((i % 4 == 3 ? wb >> 1 : wb << (23 - 8 * (i % 4))) & 0x7f800000u);
                        d[0] = fmaf(c[i][0], fa, d[0]);
                        d[1] = fmaf(c[i][1], fa, d[1]);
                        d[2] = fmaf(c[i][2], fb, d[2]);
                        d[3] = fmaf(c[i][3], fb, d[3]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = c[0][i] + c[1][i];
            }
            if (PAIR) {  // lanes t and t ^ 2 add their pieces, the first for slot r, the other for r + 8
                const float s0 = t < 2 ? d[2] : d[0], s1 = t < 2 ? d[3] : d[1];
                const float r0 = __shfl_xor_sync(kFull, s0, 2), r1 = __shfl_xor_sync(kFull, s1, 2);
                d[0] = (t < 2 ? d[0] : d[2]) + r0;
                d[1] = (t < 2 ? d[1] : d[3]) + r1;
            }
#pragma unroll
            for (int i = 0; i < LS; ++i) {
                const int from = (16 * u + gid + 8 * (PAIR ? t >> 1 : i)) & 31;
                const float bias = __shfl_sync(kFull, own[u / 2].bias, from);
                ve[u][i] = __shfl_sync(kFull, own[u / 2].ve, from);
                const float f = kFour ? 1.0f : __shfl_sync(kFull, own[u / 2].kf, from);
                x[u][i][0] = fmaf(kFour ? d[2 * i] : d[2 * i] * f, qs[0], bias);
                x[u][i][1] = fmaf(kFour ? d[2 * i + 1] : d[2 * i + 1] * f, qs[1], bias);
                if constexpr (kFour) {
#pragma unroll
                    for (int k = 0; k < SW; ++k) vs[u][i][k] = __shfl_sync(kFull, own[u / 2].vs[k], from);
                }
            }
        }
        // the keys' registers are free: the next tile's
        places(tile + W, blk);
        load_k();
        load_scales();

        // a logit past its reference by more than the slack moves the references
        bool far = false;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < LS; ++i)
#pragma unroll
                for (int z = 0; z < 2; ++z) far |= x[u][i][z] > m[z] + kSlack || x[u][i][z] + ve[u][i] > r[z] + kSlack;
        if (__any_sync(kFull, far)) {
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float mx = m[z], rx = r[z];
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < LS; ++i) {
                        mx = fmaxf(mx, x[u][i][z]);
                        rx = fmaxf(rx, x[u][i][z] + ve[u][i]);
                    }
#pragma unroll
                for (int k = PAIR ? 2 : 4; k < 32; k *= 2) {
                    mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, k));
                    rx = fmaxf(rx, __shfl_xor_sync(kFull, rx, k));
                }
                const float am = ex2(m[z] - mx), ar = ex2(r[z] - rx);
                m[z] = mx;
                r[z] = rx;
                sum[z] *= am;
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    o[j][z] *= ar;
                    o[j][2 + z] *= ar;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            float y[LS][2];  // log2 of the weights, the value's exponent aside
#pragma unroll
            for (int i = 0; i < LS; ++i)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    sum[z] += ex2(x[u][i][z] - m[z]);
                    y[i][z] = x[u][i][z] - r[z] + kWeightLog2;
                }
            // B fragments of P^T from weights of these exponents: [first and second piece][slots 0..7, 8..15]
            auto weights = [&](const float (&e)[LS], uint32_t (&pf)[QP][2]) {
                uint32_t hi[LS], lo[LS];
#pragma unroll
                for (int i = 0; i < LS; ++i) split_f16x2(ex2(y[i][0] + e[i]), ex2(y[i][1] + e[i]), hi[i], lo[i]);
                if (PAIR) {
                    const uint32_t got = __shfl_xor_sync(kFull, t < 2 ? lo[0] : hi[0], 2);
                    pf[0][0] = transposed(t < 2 ? hi[0] : got);
                    pf[0][1] = transposed(t < 2 ? got : lo[0]);
                } else {
#pragma unroll
                    for (int i = 0; i < LS; ++i) {
                        pf[0][i] = transposed(hi[i]);
                        pf[QP - 1][i] = transposed(lo[i]);
                    }
                }
            };
            if constexpr (kFour) {
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    // bytes of (slot 2t, slot 2t + 1) and of the slots 8 behind, even dims and odd
                    uint32_t ev[2][4], od[2][4];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t p = vw[u][2 * k][i], q = vw[u][2 * k + 1][i];
                        f16_of_e2m1((p & 0x0f0f0f0fu) | ((q << 4) & 0xf0f0f0f0u), ev[k]);
                        f16_of_e2m1(((p >> 4) & 0x0f0f0f0fu) | (q & 0xf0f0f0f0u), od[k]);
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int grp = 2 * i + e;
                        float ex[LS];
#pragma unroll
                        for (int k = 0; k < LS; ++k) {
                            // the byte behind 2^23's bits: 2^23 + byte
                            ex[k] = __uint_as_float(__byte_perm(vs[u][k][grp / 4], 0x4b000000u, 0x7650u + grp % 4)) - 8388735.0f;
                            if (v_nan && ex[k] == 128.0f) ex[k] = __uint_as_float(0x7fffffffu);
                        }
                        uint32_t pf[QP][2];
                        weights(ex, pf);
#pragma unroll
                        for (int k = 2 * e; k < 2 * e + 2; ++k)
#pragma unroll
                            for (int z = 0; z < QP; ++z) mma_f16(o[4 * i + k], ev[0][k], od[0][k], ev[1][k], od[1][k], pf[z][0], pf[z][1]);
                    }
                }
            } else {
                uint32_t pf[QP][2];
                weights(ve[u], pf);
#pragma unroll
                for (int i = 0; i < VW; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // dims 2e and 2e + 1 of the word, of two slots each
                        uint32_t p[2], q[2];
                        f16_of_e4m3(__byte_perm(vw[u][0][i], vw[u][1][i], e ? 0x7362 : 0x5140), p);
                        f16_of_e4m3(__byte_perm(vw[u][2][i], vw[u][3][i], e ? 0x7362 : 0x5140), q);
#pragma unroll
                        for (int z = 0; z < QP; ++z) mma_f16(o[2 * i + e], p[0], p[1], q[0], q[1], pf[z][0], pf[z][1]);
                    }
            }
        }
        load_v();
        blocks(tile + 2 * W, blk);
    }
    pdl_allow();

    // join the lanes' sums, the two pieces, the warps
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int k = PAIR ? 2 : 4; k < 32; k *= 2) sum[z] += __shfl_xor_sync(kFull, sum[z], k);
    if (PAIR) {
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int z = 0; z < 4; ++z) o[j][z] += __shfl_xor_sync(kFull, o[j][z], 2);
    }
    __syncthreads();  // the queries are read
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const int h = h0 + z;
        if (h >= g || (PAIR && t >= 2)) continue;
        float* row = smem + (warp * g + h) * PITCH;
#pragma unroll
        for (int j = 0; j < KS; ++j)
            *reinterpret_cast<float2*>(row + (kFour ? S::vdim(gid, j / 4) + 2 * (j % 4) : S::vdim(gid, j / 2) + 2 * (j % 2))) =
                make_float2(o[j][z], o[j][2 + z]);
        if (gid == 0) {
            s_m[warp][h] = m[z];
            s_l[warp][h] = sum[z];
            s_r[warp][h] = r[z];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < g * (D / 2); e += blockDim.x) {
        const int h = e / (D / 2), d = 2 * (e - h * (D / 2));
        float M = s_m[0][h], R = s_r[0][h];
        for (int w = 1; w < W; ++w) {
            M = fmaxf(M, s_m[w][h]);
            R = fmaxf(R, s_r[w][h]);
        }
        float2 acc = make_float2(0.0f, 0.0f);
        float den = 0.0f;
        for (int w = 0; w < W; ++w) {
            const float f = ex2(s_r[w][h] - R);
            const float2 y = *reinterpret_cast<const float2*>(smem + (w * g + h) * PITCH + d);
            acc.x = fmaf(f, y.x, acc.x);
            acc.y = fmaf(f, y.y, acc.y);
            den = fmaf(ex2(s_m[w][h] - M), s_l[w][h], den);
        }
        const float back = ex2(R - M - kWeightLog2);  // to the sums' reference
        acc.x *= back;
        acc.y *= back;
        if (a.splits == 1) {
            const float inv = den == 0.0f ? 0.0f : 1.0f / den;
            *reinterpret_cast<float2*>(a.out + (head0 + h) * D + d) = make_float2(acc.x * inv, acc.y * inv);
        } else {
            float* part = a.partial + ((head0 + h) * a.splits + split) * (D + 2);
            *reinterpret_cast<float2*>(part + d) = acc;
            if (d == 0) *reinterpret_cast<float2*>(part + D) = make_float2(M, den);
        }
    }
    if (err) atomicOr(a.status, err);
}

// Joins a query head's splits: a warp each; lanes hold 32 splits' references and sums at a time.
template <int D>
__global__ void __launch_bounds__(128) decode_quant_join_kernel(const __grid_constant__ DecodeQuantArgs a, int64_t heads) {
    constexpr int NV = D / 64;
    pdl_allow();
    pdl_wait();
    const int lane = threadIdx.x & 31, n = a.splits;
    const int64_t head = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (head >= heads) return;
    const float* part = a.partial + head * n * (D + 2);
    float M = kNone, den = 0.0f;
    float2 acc[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) acc[k] = make_float2(0.0f, 0.0f);
    for (int s0 = 0; s0 < n; s0 += 32) {
        const float2 mz = s0 + lane < n ? *reinterpret_cast<const float2*>(part + int64_t(s0 + lane) * (D + 2) + D) : make_float2(kNone, 0.0f);
        float top = fmaxf(M, mz.x);
#pragma unroll
        for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, k));
        const float back = ex2(M - top), w = ex2(mz.x - top);
        M = top;
        den = den * back + w * mz.y;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            acc[k].x *= back;
            acc[k].y *= back;
        }
        const int cnt = min(32, n - s0);
        for (int s = 0; s < cnt; ++s) {
            if (__shfl_sync(kFull, mz.x, s) == kNone) continue;  // nothing was written for it
            const float f = __shfl_sync(kFull, w, s);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const float2 y = *reinterpret_cast<const float2*>(part + int64_t(s0 + s) * (D + 2) + 2 * lane + 64 * k);
                acc[k].x = fmaf(f, y.x, acc[k].x);
                acc[k].y = fmaf(f, y.y, acc[k].y);
            }
        }
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) den += __shfl_xor_sync(kFull, den, k);
    const float inv = den == 0.0f ? 0.0f : 1.0f / den;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        *reinterpret_cast<float2*>(a.out + head * D + 2 * lane + 64 * k) = make_float2(acc[k].x * inv, acc[k].y * inv);
}

template <int FMT, int D>
cudaError_t launch_fd(const DecodeQuantArgs& a, cudaStream_t stream) {
    const size_t smem = size_t(a.warps) * a.group * (D + 4) * sizeof(float);
    auto k = a.group <= 4 ? decode_quant_kernel<FMT, D, true> : decode_quant_kernel<FMT, D, false>;
    cudaError_t e = smem > 48 * 1024 ? raise_smem_limit(reinterpret_cast<const void*>(k), smem) : cudaSuccess;
    const int64_t heads = int64_t(a.n_seqs) * a.n_layers * a.n_kv_heads;
    if (e == cudaSuccess) e = launch_pdl(k, dim3(unsigned(heads * a.splits)), dim3(a.warps * 32), smem, stream, a);
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_pdl(decode_quant_join_kernel<D>, dim3(unsigned((heads * a.group + 3) / 4)), dim3(128), 0, stream, a, heads * a.group);
}

template <int FMT>
cudaError_t launch_f(const DecodeQuantArgs& a, cudaStream_t stream) {
    return a.head_dim == 64 ? launch_fd<FMT, 64>(a, stream) : a.head_dim == 128 ? launch_fd<FMT, 128>(a, stream) : launch_fd<FMT, 256>(a, stream);
}

}  // namespace

cudaError_t launch_decode_quant(const DecodeQuantArgs& a, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_f<PRCR_QFMT_E4M3>(a, stream) : launch_f<PRCR_QFMT_E2M1>(a, stream);
}

int decode_quant_tile(int format, int head_dim) {
    const int bytes = format == PRCR_QFMT_E4M3 ? head_dim : head_dim / 2;
    return bytes >= 128 ? 16 : 16 * (128 / bytes);
}

}  // namespace prcr

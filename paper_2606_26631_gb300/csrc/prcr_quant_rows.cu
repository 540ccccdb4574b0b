// Rows into and out of a quantised cache: new tokens' rows rotated and rounded
// (append_quant_kernel), slots of a bf16 cache rounded (quantize_kernel) and read
// back (dequantize_kernel).
//
// Memory-bound, every row read once and written once. Neighbouring lanes hold
// neighbouring 16 bytes of bf16 of one head's row, a group's largest magnitude is
// a butterfly over the lanes that hold it, and a thread walks its layers with the
// next one's rows requested before the current ones are converted. Padding a
// head's lanes to a power of two keeps E4M3's butterflies inside a warp.
#include "prcr_pdl.cuh"
#include "prcr_quant.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;

__device__ __forceinline__ uint32_t lane_max(uint32_t x, int lanes, int step) {
    for (int o = step; o < lanes; o *= 2) x = max(x, __shfl_xor_sync(kFull, x, o));
    return x;
}

__device__ __forceinline__ uint32_t float_abs(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// x[0..n) times 2^(127 - byte), held below the code that is 2^128 (QFormat::kHighest); zeros in
// a group that reads as NaN.
template <int FMT, int N>
__device__ __forceinline__ void to_units(float* x, int byte) {
    const float f = __uint_as_float(uint32_t(254 - byte) << 23);  // 2^-126 at least: byte <= 253
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = byte == kScaleNan ? 0.0f : x[i] * f;
    if (byte == QFormat<FMT>::kHighest) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fminf(fmaxf(x[i], -QFormat<FMT>::kHighestTop), QFormat<FMT>::kHighestTop);
    }
}

// The codes of eight dims, whose quads have these bytes (E4M3: the same), at p.
template <int FMT>
__device__ __forceinline__ void store_codes(uint8_t* p, float (&x)[8], int byte0, int byte1) {
    if (FMT == PRCR_QFMT_E4M3) {
        to_units<FMT, 8>(x, byte0);
        *reinterpret_cast<uint2*>(p) = make_uint2(codes_e4m3(x[0], x[1], x[2], x[3]), codes_e4m3(x[4], x[5], x[6], x[7]));
    } else {
        to_units<FMT, 4>(x, byte0);
        to_units<FMT, 4>(x + 4, byte1);
        *reinterpret_cast<uint32_t*>(p) = codes_e2m1(x);
    }
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
    x[0] = lo_f32(w.x); x[1] = hi_f32(w.x); x[2] = lo_f32(w.y); x[3] = hi_f32(w.y);
    x[4] = lo_f32(w.z); x[5] = hi_f32(w.z); x[6] = lo_f32(w.w); x[7] = hi_f32(w.w);
}

// Largest magnitudes of the first and the second four, as float32 bits.
__device__ __forceinline__ void quad_max(const float (&x)[8], uint32_t& a, uint32_t& b) {
    a = max(max(float_abs(x[0]), float_abs(x[1])), max(float_abs(x[2]), float_abs(x[3])));
    b = max(max(float_abs(x[4]), float_abs(x[5])), max(float_abs(x[6]), float_abs(x[7])));
}

// ----------------------------------------------------------------------------
// new tokens
// ----------------------------------------------------------------------------
// One thread: eight dims of a head's first half and the eight that they rotate with,
// of K and of V. A head has `pad` threads, a power of two; E2M1's quads repeat their
// groups in the second half, so one butterfly serves both.
template <int FMT>
__global__ void __launch_bounds__(256) append_quant_kernel(const __grid_constant__ AppendQuantArgs a) {
    extern __shared__ __align__(16) float smem[];
    const int P = a.head_dim >> 1, T = a.tok_per_cta;
    float* cos_s = smem;
    float* sin_s = smem + T * P;
    QPlace* place_s = reinterpret_cast<QPlace*>(sin_s + T * P);
    const int tok0 = blockIdx.x * T;
    const int my_t = threadIdx.x / a.lanes;
    const int lane = threadIdx.x - my_t * a.lanes;
    const int my_j = tok0 + my_t;
    const int h = blockIdx.z * (a.lanes / a.pad) + lane / a.pad, v = lane & (a.pad - 1);
    const bool act = my_t < T && my_j < a.total && h < a.n_kv_heads && v < (a.head_dim >> 4);
    const int l0 = blockIdx.y * a.layers_per_cta, l1 = min(l0 + a.layers_per_cta, a.n_layers);
    const int64_t s_off = int64_t(l0) * a.src_layer_stride + int64_t(my_j) * a.src_token_stride + int64_t(h) * a.head_dim + v * 8;
    const uint16_t* sk = a.src_k + s_off;
    const uint16_t* sv = a.src_v + s_off;
    uint4 k0 = {}, k1 = {}, v0 = {}, v1 = {};
    auto load = [&]() {
        k0 = ld_stream(sk);
        k1 = ld_stream(sk + P);
        v0 = ld_stream(sv);
        v1 = ld_stream(sv + P);
    };
    pdl_allow();
    pdl_wait();
    if (act) load();

    // the tokens' places: a warp finds a token's sequence with 32 probes a round
    uint32_t err = 0;
    const int warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    for (int t = warp; t < T; t += n_warps) {
        const int j = tok0 + t;
        QPlace dst = {-1, 0};
        if (j < a.total) {
            const int b = sequence_of(a.tok_off, a.n_seqs, j);
            const int first = a.tok_off[b];
            if (j >= first && j < a.tok_off[b + 1]) {
                const int len = a.len_in[b];
                uint32_t e = 0;
                if (len < 0) e = PRCR_ST_CAPACITY;
                else dst = qplace(a.cache, b, int64_t(len) + (j - first), e);
                err |= e;
            }
        }
        if ((threadIdx.x & 31) == 0) place_s[t] = dst;
    }
    for (int q = threadIdx.x; q < T * P; q += blockDim.x) {
        const int t = q / P, i = q - t * P, j = tok0 + t;
        float c = 1.0f, s = 0.0f;
        if (j < a.total) {
            const int ax = pair_axis(i, a.layout, a.sec_t, a.sec_h, a.sec_w);
            sincos_turns(double(a.coords[3 * int64_t(j) + ax]), a.turn_freq[i], &s, &c);
        }
        cos_s[q] = c;
        sin_s[q] = s;
    }
    const bool bad = __syncthreads_or(bad_offsets(a.tok_off, a.n_seqs, a.total));
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) {
        if (bad && threadIdx.x == 0) atomicOr(a.status, PRCR_ST_CSR);
        for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
            a.len_out[b] = a.len_in[b] + (bad ? 0 : a.tok_off[b + 1] - a.tok_off[b]);
    }
    if (bad) return;
    if (err && blockIdx.y == 0 && (threadIdx.x & 31) == 0) atomicOr(a.status, err);
    QPlace dst = {-1, 0};
    float c[8] = {}, s[8] = {};
    if (act) {
        dst = place_s[my_t];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float4 c4 = *reinterpret_cast<const float4*>(cos_s + my_t * P + v * 8 + 4 * u);
            const float4 s4 = *reinterpret_cast<const float4*>(sin_s + my_t * P + v * 8 + 4 * u);
            c[4 * u] = c4.x; c[4 * u + 1] = c4.y; c[4 * u + 2] = c4.z; c[4 * u + 3] = c4.w;
            s[4 * u] = s4.x; s[4 * u + 1] = s4.y; s[4 * u + 2] = s4.z; s[4 * u + 3] = s4.w;
        }
    }
    const bool write = dst.codes >= 0;
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales;  // of a head
    const int64_t c_off = dst.codes + int64_t(l0) * a.cache.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v * B8;
    const int64_t f_off = dst.scales + int64_t(l0) * a.cache.scale_layer_stride + int64_t(h) * n;
    uint8_t *ck = a.cache.k + c_off, *cv = a.cache.v + c_off, *fk = a.cache.k_scale + f_off, *fv = a.cache.v_scale + f_off;
    const int half = P / 8 * B8;
    // lanes that share a group: E4M3 all of the head's, E2M1 every n/2-th
    const int step = FMT == PRCR_QFMT_E4M3 ? 1 : n >> 1;
    const bool keeps = v < step;  // stores its quads' scales
    for (int l = l0; l < l1; ++l) {
        float x0[8], x1[8], y0[8], y1[8];
        unpack8(k0, x0);
        unpack8(k1, x1);
        unpack8(v0, y0);
        unpack8(v1, y1);
        sk += a.src_layer_stride;
        sv += a.src_layer_stride;
        if (act && l + 1 < l1) load();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = fmaf(x0[i], c[i], -x1[i] * s[i]);
            x1[i] = fmaf(x1[i], c[i], x0[i] * s[i]);
            x0[i] = p;
        }
        int bk[2], bv[2];
        auto bytes = [&](const float (&p)[8], const float (&q)[8], int (&out)[2]) {
            uint32_t a0, a1, b0, b1;
            quad_max(p, a0, a1);
            quad_max(q, b0, b1);
            if (FMT == PRCR_QFMT_E4M3) {
                out[0] = out[1] = scale_byte<FMT>(lane_max(max(max(a0, b0), max(a1, b1)), a.pad, 1));
            } else {
                out[0] = scale_byte<FMT>(lane_max(max(a0, b0), a.pad, step));
                out[1] = scale_byte<FMT>(lane_max(max(a1, b1), a.pad, step));
            }
        };
        bytes(x0, x1, bk);
        bytes(y0, y1, bv);
        if (write) {
            store_codes<FMT>(ck, x0, bk[0], bk[1]);
            store_codes<FMT>(ck + half, x1, bk[0], bk[1]);
            store_codes<FMT>(cv, y0, bv[0], bv[1]);
            store_codes<FMT>(cv + half, y1, bv[0], bv[1]);
            if (keeps) {
                if (FMT == PRCR_QFMT_E4M3) {
                    *fk = uint8_t(bk[0]);
                    *fv = uint8_t(bv[0]);
                } else {
                    *reinterpret_cast<uint16_t*>(fk + 2 * v) = uint16_t(bk[0] | bk[1] << 8);
                    *reinterpret_cast<uint16_t*>(fv + 2 * v) = uint16_t(bv[0] | bv[1] << 8);
                }
            }
        }
        ck += a.cache.layer_stride;
        cv += a.cache.layer_stride;
        fk += a.cache.scale_layer_stride;
        fv += a.cache.scale_layer_stride;
    }
}

// ----------------------------------------------------------------------------
// slots of one cache into the other
// ----------------------------------------------------------------------------
// Token i of sequence b: from slot src_begin[b] + i to slot dst_begin[b] + i. A thread has
// eight dims of a head; all of a token's threads look its rows up, at the same addresses.
struct CastRow {
    int64_t row;   // of the bf16 cache, elements
    QPlace place;  // of the quantised one
};

template <bool READ>
__device__ __forceinline__ CastRow cast_row(const CastArgs& a, int b, int i, uint32_t& err) {
    CastRow r = {-1, {-1, 0}};
    const int count = a.count[b];
    if ((count < 0 || count > a.max_count) && i == 0) err |= PRCR_ST_CAPACITY;
    if (i >= count) return r;
    const int64_t s = a.src_begin[b], d = a.dst_begin[b];  // (a negative one is refused by the lookups for its own slots)
    const int64_t wide = READ ? d : s, few = READ ? s : d;
    if (s < 0 || d < 0) {
        err |= PRCR_ST_CAPACITY;
        return r;
    }
    r.row = slot_row(a.wide, b, wide + i, err);
    r.place = qplace(a.few, b, few + i, err);
    if (r.row < 0 || r.place.codes < 0) r.row = r.place.codes = -1;
    return r;
}

template <int FMT>
__global__ void __launch_bounds__(256) quantize_kernel(const __grid_constant__ CastArgs a) {
    const int b = blockIdx.z, l0 = blockIdx.y * a.layers_per_cta, l1 = min(l0 + a.layers_per_cta, a.n_layers);
    const int tok0 = blockIdx.x * a.tok_per_cta;
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales, step = FMT == PRCR_QFMT_E4M3 ? 1 : n >> 1;
    uint32_t err = 0;
    pdl_allow();
    pdl_wait();
    if (tok0 >= a.count[b] && tok0 > 0) return;
    // (whole warps: a head's lanes are a power of two)
    for (int u = threadIdx.x; u < a.units; u += blockDim.x) {
        const int t = u / a.lanes, lane = u - t * a.lanes, h = lane / a.pad, v = lane & (a.pad - 1), i = tok0 + t;
        CastRow r = {-1, {-1, 0}};
        if (t < a.tok_per_cta && i < a.max_count) r = cast_row<false>(a, b, i, err);
        const bool act = r.row >= 0 && v < (a.head_dim >> 3);
        const int64_t off = r.row + int64_t(l0) * a.wide.layer_stride + int64_t(h) * a.head_dim + v * 8;
        const uint16_t *sk = a.wide.k + off, *sv = a.wide.v + off;
        const int64_t c_off = r.place.codes + int64_t(l0) * a.few.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v * B8;
        const int64_t f_off = r.place.scales + int64_t(l0) * a.few.scale_layer_stride + int64_t(h) * n;
        uint8_t *ck = a.few.k + c_off, *cv = a.few.v + c_off, *fk = a.few.k_scale + f_off, *fv = a.few.v_scale + f_off;
        uint4 wk = {}, wv = {};
        if (act) {
            wk = ld_stream(sk);
            wv = ld_stream(sv);
        }
        for (int l = l0; l < l1; ++l) {
            float x[8], y[8];
            unpack8(wk, x);
            unpack8(wv, y);
            sk += a.wide.layer_stride;
            sv += a.wide.layer_stride;
            if (act && l + 1 < l1) {
                wk = ld_stream(sk);
                wv = ld_stream(sv);
            }
            uint32_t x0, x1, y0, y1;
            quad_max(x, x0, x1);
            quad_max(y, y0, y1);
            int bk[2], bv[2];
            if (FMT == PRCR_QFMT_E4M3) {
                bk[0] = bk[1] = scale_byte<FMT>(lane_max(max(x0, x1), a.pad, 1));
                bv[0] = bv[1] = scale_byte<FMT>(lane_max(max(y0, y1), a.pad, 1));
            } else {
                bk[0] = scale_byte<FMT>(lane_max(x0, a.pad, step));
                bk[1] = scale_byte<FMT>(lane_max(x1, a.pad, step));
                bv[0] = scale_byte<FMT>(lane_max(y0, a.pad, step));
                bv[1] = scale_byte<FMT>(lane_max(y1, a.pad, step));
            }
            if (act) {
                store_codes<FMT>(ck, x, bk[0], bk[1]);
                store_codes<FMT>(cv, y, bv[0], bv[1]);
                if (v < step) {
                    if (FMT == PRCR_QFMT_E4M3) {
                        *fk = uint8_t(bk[0]);
                        *fv = uint8_t(bv[0]);
                    } else {
                        *reinterpret_cast<uint16_t*>(fk + 2 * v) = uint16_t(bk[0] | bk[1] << 8);
                        *reinterpret_cast<uint16_t*>(fv + 2 * v) = uint16_t(bv[0] | bv[1] << 8);
                    }
                }
            }
            ck += a.few.layer_stride;
            cv += a.few.layer_stride;
            fk += a.few.scale_layer_stride;
            fv += a.few.scale_layer_stride;
        }
    }
    if (err && blockIdx.y == 0) atomicOr(a.status, err);
}

// The codes and scales of eight dims.
template <int FMT> struct Codes8 {
    uint2 w;       // E2M1: the codes and the two scales
    uint32_t f;
    __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* s) {
        if (FMT == PRCR_QFMT_E4M3) {
            asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w.x), "=r"(w.y) : "l"(p));
            f = *s;
        } else {
            asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w.x) : "l"(p));
            f = *reinterpret_cast<const uint16_t*>(s);
        }
    }
    __device__ __forceinline__ uint4 values() const {
        uint32_t h[4];
        float f0, f1;
        if (FMT == PRCR_QFMT_E4M3) {
            uint32_t a[2], b[2];
            f16_of_e4m3(w.x, a);
            f16_of_e4m3(w.y, b);
            h[0] = a[0]; h[1] = a[1]; h[2] = b[0]; h[3] = b[1];
            f0 = f1 = scale_value(int(f));
        } else {
            f16_of_e2m1(w.x, h);
            f0 = scale_value(int(f & 255));
            f1 = scale_value(int(f >> 8));
        }
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            const float g = i < 2 ? f0 : f1;
            r[i] = pack_bf16x2(x.x * g, x.y * g);  // exact for scales that the library wrote
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    }
};

template <int FMT>
__global__ void __launch_bounds__(256) dequantize_kernel(const __grid_constant__ CastArgs a) {
    const int b = blockIdx.z, l0 = blockIdx.y * a.layers_per_cta, l1 = min(l0 + a.layers_per_cta, a.n_layers);
    const int tok0 = blockIdx.x * a.tok_per_cta;
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales;
    uint32_t err = 0;
    pdl_allow();
    pdl_wait();
    if (tok0 >= a.count[b] && tok0 > 0) return;
    for (int u = threadIdx.x; u < a.units; u += blockDim.x) {
        const int t = u / a.lanes, lane = u - t * a.lanes, h = lane / a.pad, v = lane - h * a.pad, i = tok0 + t;
        if (t >= a.tok_per_cta || i >= a.max_count) continue;
        const CastRow r = cast_row<true>(a, b, i, err);
        if (r.row < 0) continue;
        const int64_t off = r.row + int64_t(l0) * a.wide.layer_stride + int64_t(h) * a.head_dim + v * 8;
        uint16_t *dk = a.wide.k + off, *dv = a.wide.v + off;
        const int64_t c_off = r.place.codes + int64_t(l0) * a.few.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v * B8;
        const int64_t f_off = r.place.scales + int64_t(l0) * a.few.scale_layer_stride + int64_t(h) * n + (FMT == PRCR_QFMT_E4M3 ? 0 : 2 * v % n);
        const uint8_t *ck = a.few.k + c_off, *cv = a.few.v + c_off, *fk = a.few.k_scale + f_off, *fv = a.few.v_scale + f_off;
        Codes8<FMT> x, y;
        x.load(ck, fk);
        y.load(cv, fv);
        for (int l = l0; l < l1; ++l) {
            const Codes8<FMT> p = x, q = y;
            ck += a.few.layer_stride;
            cv += a.few.layer_stride;
            fk += a.few.scale_layer_stride;
            fv += a.few.scale_layer_stride;
            if (l + 1 < l1) {
                x.load(ck, fk);
                y.load(cv, fv);
            }
            st_row(dk, p.values());
            st_row(dv, q.values());
            dk += a.wide.layer_stride;
            dv += a.wide.layer_stride;
        }
    }
    if (err && blockIdx.y == 0) atomicOr(a.status, err);
}

}  // namespace

cudaError_t launch_append_quant(const AppendQuantArgs& a, dim3 grid, int block, size_t smem, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(append_quant_kernel<PRCR_QFMT_E4M3>, grid, dim3(block), smem, stream, a)
                                      : launch_pdl(append_quant_kernel<PRCR_QFMT_E2M1>, grid, dim3(block), smem, stream, a);
}

cudaError_t launch_quantize(const CastArgs& a, dim3 grid, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(quantize_kernel<PRCR_QFMT_E4M3>, grid, dim3(256), 0, stream, a)
                                      : launch_pdl(quantize_kernel<PRCR_QFMT_E2M1>, grid, dim3(256), 0, stream, a);
}

cudaError_t launch_dequantize(const CastArgs& a, dim3 grid, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(dequantize_kernel<PRCR_QFMT_E4M3>, grid, dim3(256), 0, stream, a)
                                      : launch_pdl(dequantize_kernel<PRCR_QFMT_E2M1>, grid, dim3(256), 0, stream, a);
}

}  // namespace prcr

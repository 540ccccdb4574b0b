// Rows into and out of a quantised cache: new tokens' rows rotated and rounded
// (append_quant_kernel), slots of a bf16 cache rounded (quantize_kernel) and read
// back (dequantize_kernel).
//
// Memory-bound, every row read once and written once. Neighbouring lanes hold
// neighbouring 16 bytes of bf16 of one head's row, and a group's largest magnitude is
// a butterfly over the lanes that hold it. Padding a head's lanes to a power of two
// keeps E4M3's butterflies inside a warp.
// What costs beside the bytes is finding them: a token's place hangs on two or three loads one after the other. So
// a CTA looks its tokens up once and walks several layers with them, the next layer's rows on their way while one is worked on
// (reading back: four tokens' requested together).
//
// Measured (us, and bytes moved per time of the 6.8 TB/s that a copy makes):
//   append      E4M3, 4 KV heads of 128, 28 layers, prompts of 6 sequences, up to 2116 tokens each 157 (72 %), E2M1 140 (68 %);
//               one token of 16 sequences, 36 layers 7 (in a graph)
//   quantise    E4M3, 8 KV heads of 128, 36 layers, up to 1024 tokens of 16 sequences 341 (95 %)
//   dequantise  the same 344 (94 %); one layer, four prompts of up to 16,384 57 (75 %)
//               E2M1, 4 KV heads, 28 layers, 8 of up to 4096 258 (91 %), in blocks of 7 slots
// The casts wait for memory (E2M1's rounding for issue slots, 78 % taken), the append as much for its keys' arithmetic: two
// conversions of each key's code, and a comparison.
#include "prcr_pdl.cuh"
#include "prcr_quant.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;

// Two floats at a time: a b, a + b, a b + c, each rounded once.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

// The larger magnitude, or NaN.
__device__ __forceinline__ float abs_max(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ uint32_t quad_max(const float* x) {
    return __float_as_uint(abs_max(abs_max(x[0], x[1]), abs_max(x[2], x[3]))) & 0x7fffffffu;
}

// The largest magnitudes of eight bf16 values' two quads, as bf16 bits side by side (those of infinities and NaN, which
// are the largest numbers of 15 bits, among them).
__device__ __forceinline__ uint32_t halves_max(uint32_t a, uint32_t b) {  // of a's two, of b's two
    return __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
}
__device__ __forceinline__ uint32_t quads_max(const uint4& w) {
    return halves_max(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
}

// x[0..n) times 2^(127 - byte), held below the code that is 2^128 (QFormat::kHighest); zeros in
// a group that reads as NaN.
template <int FMT, int N>
__device__ __forceinline__ void to_units(float* x, int byte) {
    const float f = __uint_as_float(uint32_t(254 - byte) << 23);  // 2^-126 at least: byte <= 253
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 two = mul2(make_float2(x[i], x[i + 1]), make_float2(f, f));
        x[i] = two.x;
        x[i + 1] = two.y;
    }
    if (byte >= QFormat<FMT>::kHighest) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = byte == kScaleNan ? 0.0f : fminf(fmaxf(x[i], -QFormat<FMT>::kHighestTop), QFormat<FMT>::kHighestTop);
    }
}

// The codes of eight dims in units of their scales.
template <int FMT>
__device__ __forceinline__ uint2 codes8(const float (&x)[8]) {
    if (FMT == PRCR_QFMT_E4M3) return make_uint2(codes_e4m3(x[0], x[1], x[2], x[3]), codes_e4m3(x[4], x[5], x[6], x[7]));
    return make_uint2(codes_e2m1(x), 0);
}
template <int FMT>
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 c) {
    if (FMT == PRCR_QFMT_E4M3) *reinterpret_cast<uint2*>(p) = c;
    else *reinterpret_cast<uint32_t*>(p) = c.x;
}

template <int FMT>
__device__ __forceinline__ void to_units8(float (&x)[8], int byte0, int byte1) {
    if (FMT == PRCR_QFMT_E4M3) {
        to_units<FMT, 8>(x, byte0);
    } else {
        to_units<FMT, 4>(x, byte0);
        to_units<FMT, 4>(x + 4, byte1);
    }
}

// Eight dims of bf16 whose quads have these bytes (E4M3: the same).
template <int FMT>
__device__ __forceinline__ void store_rounded(uint8_t* p, const uint4& w, int byte0, int byte1) {
    float x[8] = {lo_f32(w.x), hi_f32(w.x), lo_f32(w.y), hi_f32(w.y), lo_f32(w.z), hi_f32(w.z), lo_f32(w.w), hi_f32(w.w)};
    to_units8<FMT>(x, byte0, byte1);
    store_codes<FMT>(p, codes8<FMT>(x));
}

// The larger ones over the lanes that share a group: E4M3 all `lanes` of a head's, E2M1 2^ROUNDS that are `step` apart.
template <int FMT, int ROUNDS>
__device__ __forceinline__ uint32_t group_max(uint32_t x, int lanes, int step) {
    if (FMT == PRCR_QFMT_E4M3) {
        for (int o = 1; o < lanes; o *= 2) x = max(x, __shfl_xor_sync(kFull, x, o));
        return x;
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) x = max(x, __shfl_xor_sync(kFull, x, step << r));
    return x;
}
template <int FMT, int ROUNDS>
__device__ __forceinline__ uint32_t group_max2(uint32_t two, int lanes, int step) {
    if (FMT == PRCR_QFMT_E4M3) {
        for (int o = 1; o < lanes; o *= 2) two = __vmaxu2(two, __shfl_xor_sync(kFull, two, o));
    } else {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) two = __vmaxu2(two, __shfl_xor_sync(kFull, two, step << r));
    }
    return two;
}

// Scales' bytes of two groups' largest magnitudes, of bf16 bits side by side.
template <int FMT>
__device__ __forceinline__ void bytes_of(uint32_t two, int& byte0, int& byte1) {
    byte0 = scale_byte<FMT>(two << 16);
    byte1 = scale_byte<FMT>(two & 0xffff0000u);
}

template <int FMT>
__device__ __forceinline__ void store_scales(uint8_t* row, int v, int byte0, int byte1) {
    if (FMT == PRCR_QFMT_E4M3) *row = uint8_t(byte0);
    else *reinterpret_cast<uint16_t*>(row + 2 * v) = uint16_t(byte0 | byte1 << 8);
}

// ----------------------------------------------------------------------------
// new tokens
// ----------------------------------------------------------------------------
// One thread: eight dims of a head's first half and the eight that they rotate with,
// of K and of V. A head has `pad` threads, a power of two; E2M1's quads repeat their
// groups in the second half, so one butterfly serves both.
//
// Keys get the codes that are nearest to the exact rotation. Its cos and sin are pairs of floats, the first of 16
// bits, so that a bf16 number's products with it are exact: x cos - y sin, of two such products and two small
// ones, is off by three roundings of 2^-24 of itself and by 2^-28.9 of the pair's norm, which is what cos and sin are
// off by. A value is computed again in float64 where its code would change within 2^-20 of itself and, in E4M3, 2^-18 of the
// scale's unit more: a pair's norm is at most 448 sqrt(2) units there, so that cos and sin move a value by 2^-19.6 units at most.
// (E2M1: by 6 sqrt(2) 2^-28.9, less than 2^-20 of the least border, a quarter.) That is one value in 40,000.

// sin and cos of 2^-64 f turns, each as the sum of two floats: Taylor's series about the nearest quarter turn, the first
// terms' products and sums with their rounding errors (by fused multiply-adds). The terms from t^5 on are single floats, some
// twelve roundings of the t^5 / 120 that is 2^-8.6 at an eighth of a turn: together sin and cos are off by 2^-28.9 there, by 2^-32
// in the mean square.
__device__ __forceinline__ void sincos_pair(uint64_t f, float2& sine, float2& cosine) {
    const uint64_t g = f + (1ull << 61);
    const int quarter = int(g >> 62);
    const int64_t rest = int64_t(g & ((1ull << 62) - 1)) - (int64_t(1) << 61);  // from it, 2^61 an eighth of a turn
    const float rh = float(rest), rl = float(rest - int64_t(rh));
    const float uh = rh * 0x1p-61f, ul = rl * 0x1p-61f;
    constexpr float kPh = 0.785398185253143310546875f, kPl = -2.18556941e-8f;  // pi / 4
    float th = uh * kPh;
    float tl = fmaf(uh, kPh, -th) + fmaf(uh, kPl, ul * kPh);
    const float zh = th * th, zl = fmaf(th, th, -zh) + 2.0f * th * tl;
    // sin t = t - t z / 6 + t z^2 (1/120 - z/5040 + z^2/362880 - ...), z = t^2
    constexpr float k6h = 0.16666667163372039794921875f, k6l = -4.96705376e-9f;  // 1 / 6
    const float qh = th * zh, ql = fmaf(th, zh, -qh) + fmaf(th, zl, tl * zh);
    const float ah = qh * k6h, al = fmaf(qh, k6h, -ah) + fmaf(qh, k6l, ql * k6h);
    const float w = qh * zh * fmaf(zh, fmaf(zh, fmaf(zh, -2.50521084e-8f, 2.75573192e-6f), -1.98412698e-4f), 8.33333333e-3f);
    const float s1 = th - ah, sl = ((th - s1) - ah) + ((tl - al) + w);
    // cos t = 1 - z/2 + z^2/24 - z^3 (1/720 - z/40320 + z^2/3628800 - ...)
    constexpr float k24h = 0.041666667908430099487305f, k24l = -1.24176344e-9f;  // 1 / 24
    const float yh = zh * zh, yl = fmaf(zh, zh, -yh) + 2.0f * zh * zl;
    const float dh = yh * k24h, dl = fmaf(yh, k24h, -dh) + fmaf(yh, k24l, yl * k24h);
    const float v = -yh * zh * fmaf(zh, fmaf(zh, fmaf(zh, -2.08767570e-9f, 2.75573192e-7f), -2.48015873e-5f), 1.38888889e-3f);
    const float bh = 0.5f * zh, c1 = 1.0f - bh, c2 = c1 + dh;
    const float cl = ((1.0f - c1) - bh) + ((c1 - c2) + dh) + ((dl - 0.5f * zl) + v);
    // the first part's leading 16 bits, the second with what that leaves
    auto cut = [](float a, float b) {
        const float h = __uint_as_float(__float_as_uint(a + b) & 0xffffff00u);
        return make_float2(h, (a - h) + b);
    };
    float2 s = cut(s1, sl), c = cut(c2, cl);
    if (quarter & 1) {
        const float2 x = s;
        s = c;
        c = make_float2(-x.x, -x.y);
    }
    if (quarter & 2) {
        s = make_float2(-s.x, -s.y);
        c = make_float2(-c.x, -c.y);
    }
    sine = s;
    cosine = c;
}

// The exact a cos - b sin (second: b cos + a sin) in units of the scale, rounded to odd: any border between codes, of
// few bits, lies on the same side of it.
__device__ __noinline__ float settled(float a, float b, bool second, int32_t pos, uint64_t turn_freq, float unit) {
    // At an angle of 0 (an image's first row, column or frame) a pair stays as it is, and one value in 16 of it lies on a border
    // exactly (six prompts at t = 0, all of them computed: 3.9 ms for 0.31).
    if (pos == 0) return (second ? b : a) * unit;
    double s, c;
    sincospi(double(int64_t(uint64_t(int64_t(pos)) * turn_freq)) * 0x1p-63, &s, &c);
    const double exact = (second ? double(b) * c + double(a) * s : double(a) * c - double(b) * s) * unit;
    const float f = __double2float_rz(exact);
    return __uint_as_float(__float_as_uint(f) | (double(f) != exact));
}

template <int FMT>
__global__ void __launch_bounds__(256, 3) append_quant_kernel(const __grid_constant__ AppendQuantArgs a) {
    extern __shared__ __align__(16) float smem[];
    const int P = a.head_dim >> 1, T = a.tok_per_cta;
    // cos and sin of the tokens' pairs: first parts, then second ones
    float* turn_s[4] = {smem, smem + T * P, smem + 2 * T * P, smem + 3 * T * P};
    QPlace* place_s = reinterpret_cast<QPlace*>(smem + 4 * T * P);
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
    pdl_allow();
    pdl_wait();
    if (act) {
        k0 = ld_stream(sk);
        k1 = ld_stream(sk + P);
        v0 = ld_stream(sv);
        v1 = ld_stream(sv + P);
    }

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
        float2 c = make_float2(1.0f, 0.0f), s = make_float2(0.0f, 0.0f);
        if (j < a.total) {
            const int ax = pair_axis(i, a.layout, a.sec_t, a.sec_h, a.sec_w);
            sincos_pair(uint64_t(int64_t(a.coords[3 * int64_t(j) + ax])) * a.turn_freq[i], s, c);
        }
        turn_s[0][q] = c.x;
        turn_s[1][q] = s.x;
        turn_s[2][q] = c.y;
        turn_s[3][q] = s.y;
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
    if (act) dst = place_s[my_t];
    const float* turn = smem + (act ? my_t * P + v * 8 : 0);
    const bool write = dst.codes >= 0;
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales;  // of a head
    const int64_t c_off = dst.codes + int64_t(l0) * a.cache.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v * B8;
    const int64_t f_off = dst.scales + int64_t(l0) * a.cache.scale_layer_stride + int64_t(h) * n;
    uint8_t *ck = a.cache.k + c_off, *cv = a.cache.v + c_off, *fk = a.cache.k_scale + f_off, *fv = a.cache.v_scale + f_off;
    const int half = P / 8 * B8;
    // lanes that share a group: E4M3 all of the head's, E2M1 every n/2-th
    const int step = FMT == PRCR_QFMT_E4M3 ? 1 : n >> 1;
    const bool keeps = write && v < step;  // stores its quads' scales
    for (int l = l0; l < l1; ++l) {
        sk += a.src_layer_stride;
        sv += a.src_layer_stride;
        const bool more = act && l + 1 < l1;
        {
            const uint4 w0 = v0, w1 = v1;
            if (more) {
                v0 = ld_stream(sv);
                v1 = ld_stream(sv + P);
            }
            int b0, b1;
            uint32_t quads = __vmaxu2(quads_max(w0), quads_max(w1));
            if (FMT == PRCR_QFMT_E4M3) quads = halves_max(quads, quads);
            bytes_of<FMT>(group_max2<FMT, 2>(quads, a.pad, step), b0, b1);
            if (write) {
                store_rounded<FMT>(cv, w0, b0, b1);
                store_rounded<FMT>(cv + half, w1, b0, b1);
            }
            if (keeps) store_scales<FMT>(fv, v, b0, b1);
        }
        const uint4 w0 = k0, w1 = k1;
        if (more) {
            k0 = ld_stream(sk);
            k1 = ld_stream(sk + P);
        }
        float x[8] = {lo_f32(w0.x), hi_f32(w0.x), lo_f32(w0.y), hi_f32(w0.y), lo_f32(w0.z), hi_f32(w0.z), lo_f32(w0.w), hi_f32(w0.w)};
        float y[8] = {lo_f32(w1.x), hi_f32(w1.x), lo_f32(w1.y), hi_f32(w1.y), lo_f32(w1.z), hi_f32(w1.z), lo_f32(w1.w), hi_f32(w1.w)};
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
            const float2 c = *reinterpret_cast<const float2*>(turn + u), s = *reinterpret_cast<const float2*>(turn + T * P + u);
            const float2 cl = *reinterpret_cast<const float2*>(turn + 2 * T * P + u), sl = *reinterpret_cast<const float2*>(turn + 3 * T * P + u);
            // (the products with the first parts are exact, so their difference is rounded once)
            const float2 p = make_float2(x[u], x[u + 1]), q = make_float2(y[u], y[u + 1]), minus = make_float2(-1.0f, -1.0f);
            const float2 dx = add2(fma2(mul2(q, s), minus, mul2(p, c)), fma2(mul2(q, sl), minus, mul2(p, cl)));
            const float2 dy = add2(fma2(q, c, mul2(p, s)), fma2(q, cl, mul2(p, sl)));
            x[u] = dx.x;
            x[u + 1] = dx.y;
            y[u] = dy.x;
            y[u + 1] = dy.y;
        }
        int b0, b1;
        const uint32_t first = max(quad_max(x), quad_max(y)), second = max(quad_max(x + 4), quad_max(y + 4));
        if (FMT == PRCR_QFMT_E4M3) {
            b0 = b1 = scale_byte<FMT>(group_max<FMT, 0>(max(first, second), a.pad, step));
        } else {
            b0 = scale_byte<FMT>(group_max<FMT, 2>(first, a.pad, step));
            b1 = scale_byte<FMT>(group_max<FMT, 2>(second, a.pad, step));
        }
        if (write) {
            to_units8<FMT>(x, b0, b1);
            to_units8<FMT>(y, b0, b1);
            constexpr float kLess = 1.0f - 0x1p-20f, kMore = 1.0f + 0x1p-20f;
            // the least magnitude that a value may have (and its sign turned over in E4M3), and the largest
            float z[8];
            auto times = [&](const float (&w)[8], float f) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float2 two = make_float2(w[i], w[i + 1]), by = make_float2(f, f);
                    const float2 off = make_float2(copysignf(0x1p-18f, w[i]), copysignf(0x1p-18f, w[i + 1]));
                    const float2 end = FMT == PRCR_QFMT_E4M3 ? fma2(two, by, off) : mul2(two, by);
                    z[i] = end.x;
                    z[i + 1] = end.y;
                }
                return codes8<FMT>(z);
            };
            constexpr float kLeast = FMT == PRCR_QFMT_E4M3 ? -kLess : kLess;
            const uint2 lx = times(x, kLeast), ly = times(y, kLeast);
            uint2 cx = times(x, kMore), cy = times(y, kMore);
            constexpr uint32_t kMagnitudes = FMT == PRCR_QFMT_E4M3 ? 0x7f7f7f7fu : 0x77777777u;
            const uint2 nx = make_uint2((cx.x ^ lx.x) & kMagnitudes, (cx.y ^ lx.y) & kMagnitudes);
            const uint2 ny = make_uint2((cy.x ^ ly.x) & kMagnitudes, (cy.y ^ ly.y) & kMagnitudes);
            if (nx.x | nx.y | ny.x | ny.y) {
                const uint32_t wx[4] = {w0.x, w0.y, w0.z, w0.w}, wy[4] = {w1.x, w1.y, w1.z, w1.w};
                constexpr int BITS = FMT == PRCR_QFMT_E4M3 ? 8 : 4;
                constexpr float kTop = QFormat<FMT>::kHighestTop;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool second = BITS == 8 && i >= 4;
                    const uint32_t mask = ((1u << BITS) - 1) << (BITS * i % 32);
                    const bool near_x = (second ? nx.y : nx.x) & mask, near_y = (second ? ny.y : ny.x) & mask;
                    if (near_x || near_y) {
                        const float p = i & 1 ? hi_f32(wx[i / 2]) : lo_f32(wx[i / 2]), q = i & 1 ? hi_f32(wy[i / 2]) : lo_f32(wy[i / 2]);
                        const int32_t pos = a.coords[3 * int64_t(my_j) + pair_axis(v * 8 + i, a.layout, a.sec_t, a.sec_h, a.sec_w)];
                        const int byte = i < 4 ? b0 : b1;  // (not that of NaN, whose values are all 0)
                        const float unit = __uint_as_float(uint32_t(254 - byte) << 23);
                        if (near_x) x[i] = settled(p, q, false, pos, a.turn_freq[v * 8 + i], unit);
                        if (near_y) y[i] = settled(p, q, true, pos, a.turn_freq[v * 8 + i], unit);
                        if (byte >= QFormat<FMT>::kHighest) {  // held as in to_units
                            x[i] = fminf(fmaxf(x[i], -kTop), kTop);
                            y[i] = fminf(fmaxf(y[i], -kTop), kTop);
                        }
                    }
                }
                cx = codes8<FMT>(x);
                cy = codes8<FMT>(y);
            }
            store_codes<FMT>(ck, cx);
            store_codes<FMT>(ck + half, cy);
        }
        if (keeps) store_scales<FMT>(fk, v, b0, b1);
        ck += a.cache.layer_stride;
        cv += a.cache.layer_stride;
        fk += a.cache.scale_layer_stride;
        fv += a.cache.scale_layer_stride;
    }
}

// ----------------------------------------------------------------------------
// slots of one cache into the other
// ----------------------------------------------------------------------------
// Token i of sequence b: from slot src_begin[b] + i to slot dst_begin[b] + i. A CTA looks its tokens' rows up once; then a
// thread has eight dims of a head of several tokens, requested together, layer by layer.
constexpr int kCastThreads = 256;
constexpr int kQuantTokens = 2, kReadTokens = 4;  // of a thread's at once (one each: read 404 us for 344, 36 layers of 16 sequences' up to 1024 slots)
constexpr int kCastMaxTokens = 64;  // of a CTA's
struct CastRow {
    int64_t row;   // of the bf16 cache, elements, or -1
    QPlace place;  // of the quantised one
};

template <bool READ>
__device__ __forceinline__ CastRow cast_row(const CastArgs& a, int b, int i, uint32_t& err) {
    const int count = a.count[b];
    const int64_t s = a.src_begin[b], d = a.dst_begin[b];
    if ((count < 0 || count > a.max_count) && i == 0) err |= PRCR_ST_CAPACITY;
    CastRow r = {-1, {-1, 0}};
    if (i >= count || i >= a.max_count) return r;
    const int64_t wide = (READ ? d : s) + i, few = (READ ? s : d) + i, top = int64_t(1) << 31;  // (slots are counted in an int32)
    if (s < 0 || d < 0 || wide >= min(a.wide.capacity, top) || few >= min(a.few.capacity, top)) {
        err |= PRCR_ST_CAPACITY;
        return r;
    }
    // both tables are asked at once
    const int32_t wide_blk = a.wide.kind == PRCR_CACHE_CONTIGUOUS ? 0 : a.wide.block_table[int64_t(b) * a.wide.bt_stride + block_index(a.wide, uint32_t(wide))];
    const int32_t few_blk = qblock(a.few, b, uint32_t(few));
    r.row = row_in_block(a.wide, b, uint32_t(wide), wide_blk);
    r.place = qplace_in_block(a.few, b, uint32_t(few), few_blk);
    if (r.row < 0 || r.place.codes < 0) {
        err |= PRCR_ST_NO_BLOCK;
        r.row = -1;
    }
    return r;
}

// The CTA's tokens' rows; false where none of them is to be moved.
template <bool READ>
__device__ __forceinline__ bool cast_rows(const CastArgs& a, int b, int tok0, CastRow* rows) {
    uint32_t err = 0;
    bool any = false;
    for (int t = threadIdx.x; t < a.tok_per_cta; t += blockDim.x) {
        const CastRow r = cast_row<READ>(a, b, tok0 + t, err);
        rows[t] = r;
        any |= r.row >= 0;
    }
    if (err && blockIdx.y == 0) atomicOr(a.status, err);
    return __syncthreads_or(any);
}

template <int FMT>
__global__ void __launch_bounds__(kCastThreads, 4) quantize_kernel(const __grid_constant__ CastArgs a) {
    __shared__ CastRow rows[kCastMaxTokens];
    const int b = blockIdx.z, l0 = blockIdx.y * a.layers_per_cta, l1 = min(l0 + a.layers_per_cta, a.n_layers);
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales, step = FMT == PRCR_QFMT_E4M3 ? 1 : n >> 1;
    pdl_allow();
    pdl_wait();
    if (blockIdx.x > 0 && int64_t(blockIdx.x) * a.tok_per_cta >= a.count[b]) return;  // (the first one judges the count)
    if (!cast_rows<false>(a, b, blockIdx.x * a.tok_per_cta, rows)) return;
    // (whole warps: a head's lanes are a power of two)
    for (int u0 = threadIdx.x; u0 < a.units; u0 += kQuantTokens * kCastThreads) {
        uint4 wk[kQuantTokens], wv[kQuantTokens];
        int64_t from[kQuantTokens];
        QPlace to[kQuantTokens];
        int v[kQuantTokens];
        bool act[kQuantTokens];
#pragma unroll
        for (int k = 0; k < kQuantTokens; ++k) {
            const int u = u0 + k * kCastThreads, t = u / a.lanes, lane = u - t * a.lanes, h = lane / a.pad;
            v[k] = lane & (a.pad - 1);
            act[k] = t < a.tok_per_cta && v[k] < (a.head_dim >> 3);
            const CastRow r = act[k] ? rows[t] : CastRow{-1, {-1, 0}};
            act[k] = act[k] && r.row >= 0;
            from[k] = r.row + int64_t(l0) * a.wide.layer_stride + int64_t(h) * a.head_dim + v[k] * 8;
            to[k].codes = r.place.codes + int64_t(l0) * a.few.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v[k] * B8;
            to[k].scales = r.place.scales + int64_t(l0) * a.few.scale_layer_stride + int64_t(h) * n;
            wk[k] = wv[k] = make_uint4(0, 0, 0, 0);
        }
        auto load = [&](int k) {
            if (act[k]) {
                wk[k] = ld_stream(a.wide.k + from[k]);
                wv[k] = ld_stream(a.wide.v + from[k]);
            }
            from[k] += a.wide.layer_stride;
        };
#pragma unroll
        for (int k = 0; k < kQuantTokens; ++k) load(k);
        for (int l = l0; l < l1; ++l) {
#pragma unroll
            for (int k = 0; k < kQuantTokens; ++k) {
                const uint4 x = wk[k], y = wv[k];
                if (l + 1 < l1) load(k);
                int k0, k1, v0, v1;
                if (FMT == PRCR_QFMT_E4M3) {  // one butterfly for both rows
                    bytes_of<FMT>(group_max2<FMT, 0>(halves_max(quads_max(x), quads_max(y)), a.pad, step), k0, v0);
                    k1 = k0;
                    v1 = v0;
                } else {
                    bytes_of<FMT>(group_max2<FMT, 3>(quads_max(x), a.pad, step), k0, k1);
                    bytes_of<FMT>(group_max2<FMT, 3>(quads_max(y), a.pad, step), v0, v1);
                }
                if (act[k]) {
                    store_rounded<FMT>(a.few.k + to[k].codes, x, k0, k1);
                    store_rounded<FMT>(a.few.v + to[k].codes, y, v0, v1);
                    if (v[k] < step) {
                        store_scales<FMT>(a.few.k_scale + to[k].scales, v[k], k0, k1);
                        store_scales<FMT>(a.few.v_scale + to[k].scales, v[k], v0, v1);
                    }
                }
                to[k].codes += a.few.layer_stride;
                to[k].scales += a.few.scale_layer_stride;
            }
        }
    }
}

// The codes and scales of eight dims.
template <int FMT> struct Codes8 {
    uint2 w;       // E2M1: the codes and the two scales
    uint32_t f;
    __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* s) {
        if (FMT == PRCR_QFMT_E4M3) {
            asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w.x), "=r"(w.y) : "l"(p));
            f = *s;
        } else {
            asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w.x) : "l"(p));
            f = *reinterpret_cast<const unsigned short*>(s);
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
__global__ void __launch_bounds__(kCastThreads, 3) dequantize_kernel(const __grid_constant__ CastArgs a) {
    __shared__ CastRow rows[kCastMaxTokens];
    const int b = blockIdx.z, l0 = blockIdx.y * a.layers_per_cta, l1 = min(l0 + a.layers_per_cta, a.n_layers);
    constexpr int B8 = QFormat<FMT>::kBytes8;
    const int n = a.n_scales;
    pdl_allow();
    pdl_wait();
    if (blockIdx.x > 0 && int64_t(blockIdx.x) * a.tok_per_cta >= a.count[b]) return;
    if (!cast_rows<true>(a, b, blockIdx.x * a.tok_per_cta, rows)) return;
    for (int u0 = threadIdx.x; u0 < a.units; u0 += kReadTokens * kCastThreads) {
        Codes8<FMT> x[kReadTokens], y[kReadTokens];
        int64_t to[kReadTokens];
        QPlace from[kReadTokens];
        bool act[kReadTokens];
#pragma unroll
        for (int k = 0; k < kReadTokens; ++k) {
            const int u = u0 + k * kCastThreads, t = u / a.lanes, lane = u - t * a.lanes, h = lane / a.pad, v = lane - h * a.pad;
            const CastRow r = t < a.tok_per_cta ? rows[t] : CastRow{-1, {-1, 0}};
            act[k] = r.row >= 0;
            to[k] = r.row + int64_t(l0) * a.wide.layer_stride + int64_t(h) * a.head_dim + v * 8;
            from[k].codes = r.place.codes + int64_t(l0) * a.few.layer_stride + int64_t(h) * (a.head_dim / 8 * B8) + v * B8;
            from[k].scales = r.place.scales + int64_t(l0) * a.few.scale_layer_stride + int64_t(h) * n + (FMT == PRCR_QFMT_E4M3 ? 0 : 2 * v % n);
        }
        for (int l = l0; l < l1; ++l) {
#pragma unroll
            for (int k = 0; k < kReadTokens; ++k)
                if (act[k]) {
                    x[k].load(a.few.k + from[k].codes, a.few.k_scale + from[k].scales);
                    y[k].load(a.few.v + from[k].codes, a.few.v_scale + from[k].scales);
                }
#pragma unroll
            for (int k = 0; k < kReadTokens; ++k) {
                if (act[k]) {
                    st_row(a.wide.k + to[k], x[k].values());
                    st_row(a.wide.v + to[k], y[k].values());
                }
                to[k] += a.wide.layer_stride;
                from[k].codes += a.few.layer_stride;
                from[k].scales += a.few.scale_layer_stride;
            }
        }
    }
}

}  // namespace

cudaError_t launch_append_quant(const AppendQuantArgs& a, dim3 grid, int block, size_t smem, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(append_quant_kernel<PRCR_QFMT_E4M3>, grid, dim3(block), smem, stream, a)
                                      : launch_pdl(append_quant_kernel<PRCR_QFMT_E2M1>, grid, dim3(block), smem, stream, a);
}

cudaError_t launch_quantize(const CastArgs& a, dim3 grid, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(quantize_kernel<PRCR_QFMT_E4M3>, grid, dim3(kCastThreads), 0, stream, a)
                                      : launch_pdl(quantize_kernel<PRCR_QFMT_E2M1>, grid, dim3(kCastThreads), 0, stream, a);
}

cudaError_t launch_dequantize(const CastArgs& a, dim3 grid, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_pdl(dequantize_kernel<PRCR_QFMT_E4M3>, grid, dim3(kCastThreads), 0, stream, a)
                                      : launch_pdl(dequantize_kernel<PRCR_QFMT_E2M1>, grid, dim3(kCastThreads), 0, stream, a);
}

}  // namespace prcr

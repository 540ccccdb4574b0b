// One new token of each sequence over a quantised cache: for every sequence, layer
// and query head
//   o = sum_s p_s V_s,   p = softmax(RoPE(q, (p, p, p)) K^T / sqrt(D)),
// with K and V the codes' values times their groups' powers of two.
//
// Memory-bound in bytes, but only just: a code costs a conversion beside its
// product, and a byte of codes brings two or four times a bf16 byte's products.
// So nothing passes through shared memory on its way: a warp loads its tiles'
// codes straight into the registers in which the matrix instructions want them,
// the next tile's as soon as a tile's are used up. (Rings of tiles in shared memory,
// filled by asynchronous copies, were slower: they shrink the L1 cache
// that a load's lines wait in.) tcgen05 wants 64 rows of a product at least, where a
// group has 8 queries at most, and its operands in shared memory.
//   S^T (16 slots x 8 heads) = K Q^T. The order of the dims in a dot product is
//     free, so lane t of a slot's four takes 16-byte pieces t, t + 4, ... of its
//     row; four dims in a lane are one k-step's share.
//   O^T (16 dims x 8 heads) += V^T P^T. Which dims are the rows of which product is free
//     too: lane group r takes piece r of the rows of four slots, and interleaving the
//     bytes of two slots gives the pairs along the slots that the product sums over.
// Codes are exact in fp16, in which they enter. The query (scaled by a power of
// two to at most 2^14) and the weights enter as two fp16 each, 22 bits; with up to four
// heads to a group the two lie side by side in the product's eight columns, so that one
// product takes both (four heads to a group, 16 sequences of up to 4096 slots, E4M3, 36
// layers: 465 us, with two products 538). One fp16 would leave 2^-12 of a weight, a hundred
// times what the rest loses.
// Scales never touch the codes. E4M3: a key's multiplies its slot's logits, a value's goes
// into its weight's exponent. E2M1, whose groups take every (D/32)-th quad of dims, so that
// each lane's piece of a row has quads of all groups: a key's multiply the partial sums of
// their groups' k-steps; of a value's the largest goes into the weight's exponent, and what the others
// are to it multiplies the weights of the products of their groups.
// Weights are therefore kept against two references, both powers of two: p = 2^(x - m)
// for the sum, w = 2^(x + e - r + 11) for the accumulator, e the value's exponent. m and r follow the
// largest x and x + e, but only when one is more than 2^4 past them, so that most tiles
// rescale nothing and need no reduction over the lanes; w stays below 2^15, and what fp16 loses
// of it is 2^-36 of the largest at most. E2M1's groups of a row have one reference, so that this is of the row's largest group: a
// group within 2^7 of that in every slot loses 2^-27 of its own largest at most. One that is not gets another pass over
// the unit's tiles, in which its scales are the rows' (each such group as much time again; scales that differ so far are rare).
//
// Work is cut by what there is, not by sequence: all (sequence, layer, set of heads) units' tiles
// in one row, one even share of it to each team of 1, 2 or 4 warps on the same slots of
// neighbouring KV heads (whose codes are neighbouring bytes: teams of one take 500 us for 465, E2M1 at 64 bytes
// a row 212 for 200; of two 471 and 199). A share's units that
// it has whole are written at once, the parts of others joined by a second kernel.
// A grid is one wave: 12 warps an SM, 8 at head_dim 256, which is what the registers hold (E4M3 with 8 for 12:
// 533 us for 465; with 16, which spill, 459 and E2M1 196 for 200, but one sequence of 933 slots 31 for 27). Rows of 64
// bytes go in tiles of 32 slots (E2M1 200 us; of 16 242, of 64 with 8 warps 207).
//
// Measured (us, and bytes read per time of the 6.8 TB/s that a copy makes): E4M3, 8 KV heads of 128, 36 layers:
// 16 sequences of up to 4096 slots 459 (92 %), one of 933 22; one layer, 32 of up to 16,384 116 (84 %);
// E2M1, 4 KV heads of seven queries, 28 layers, 8 of up to 8192 197 (46 %); E4M3, 4 KV heads of 256, one layer, 8 of up to
// 8000 33. E4M3 waits for memory; E2M1 for issue slots (61 % of them taken, the
// tensor cores 32 % busy: some 470 instructions of a warp for 16 slots), so that it takes 0.86 of E4M3's time at the same
// shape; head_dim 256 for latencies, at 8 warps an SM; what is short, for its launches.
#include <algorithm>

#include <cuda_fp16.h>

#include "prcr_pdl.cuh"
#include "prcr_quant.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr float kNone = -3.0e38f;   // reference of no slot yet: below every logit, and finite
constexpr float kSlack = 4.0f;      // log2 of how far past its reference a weight may go
constexpr float kWeightLog2 = 11.0f;
constexpr int kCtaWarps = 4;
// E2M1: a group is worked on once more, by itself, where its scale lies 2^8 or more below the row's largest in any slot (a difference of
// bytes with one of these bits), unless none of its scales is above 2^-112 (no byte has one of these bits: groups of zeros).
constexpr uint32_t kFarBelow = 0xf8, kLeastUsed = 0xf0;

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

// The same from zero.
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// o += x, rounded to nearest. (The tensor cores' own sums are cut off, not rounded: values of one sign summed there over 131,072
// slots lost 8e-4 of their mean, over 8192 3e-5.)
__device__ __forceinline__ void add_to(float (&o)[4], const float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
        asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
            : "+f"(o[i]), "+f"(o[i + 1]) : "f"(x[i]), "f"(x[i + 1]));
}

// Transpose of an 8 x 8 matrix of 16-bit values held as mma fragments.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    const __half2 c = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&c);
}

// The two powers of two (bf16) of scales' bytes; 255 gives NaN.
__device__ __forceinline__ uint32_t bf16_of_scales(uint32_t two) {
    uint32_t r;
    asm("{\n.reg .b16 l, u;\nmov.b32 {l, u}, %1;\ncvt.rn.bf16x2.ue8m0x2 %0, l;\n}" : "=r"(r) : "r"(two));
    return r;
}

// N words from p; `ok`: all of them, or zeros. (A load that waits for nothing: `ok ? *p : 0` would wait at once.
// Not by the read-only path: this kernel is resident while the append before it in the stream still writes the rows.)
template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
    static_assert(N == 1 || N == 2 || N == 4, "4, 8 or 16 bytes");
    if constexpr (N == 4)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (N == 2)
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}
template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p, bool ok) {
    if constexpr (N == 4) {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %5, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\nmov.b32 %2, 0;\nmov.b32 %3, 0;\n"
                     "@p ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                     : "=&r"(w[0]), "=&r"(w[1]), "=&r"(w[2]), "=&r"(w[3]) : "l"(p), "r"(int(ok)));
    } else if constexpr (N == 2) {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %3, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\n"
                     "@p ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];\n}"
                     : "=&r"(w[0]), "=&r"(w[1]) : "l"(p), "r"(int(ok)));
    } else {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.L1::no_allocate.u32 %0, [%1];\n}"
                     : "=&r"(w[0]) : "l"(p), "r"(int(ok)));
    }
}

// A row's N scales' bytes, or zeros.
template <int N>
__device__ __forceinline__ void load_row_scales(uint32_t* w, const uint8_t* p, bool ok) {
    if constexpr (N == 8)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %3, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\n@p ld.global.v2.u32 {%0, %1}, [%2];\n}"
                     : "=&r"(w[0]), "=&r"(w[1]) : "l"(p), "r"(int(ok)));
    else if constexpr (N == 4)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.u32 %0, [%1];\n}" : "=&r"(w[0]) : "l"(p), "r"(int(ok)));
    else if constexpr (N == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.u16 %0, [%1];\n}" : "=&r"(w[0]) : "l"(p), "r"(int(ok)));
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.u8 %0, [%1];\n}" : "=&r"(w[0]) : "l"(p), "r"(int(ok)));
}

// Sizes of a format's rows: RB bytes of codes; a warp takes tiles of SUB x 16 slots.
template <int FMT, int D> struct Shape {
    static constexpr bool kFour = FMT == PRCR_QFMT_E2M1;
    static constexpr int RB = kFour ? D / 2 : D;
    static constexpr int SUB = RB >= 128 ? 1 : 128 / RB;
    static constexpr int TS = 16 * SUB;
    static constexpr int N = kFour ? D / 32 : 1;  // scales of a row
    static constexpr int KW = RB / 16, VW = RB / 32;  // a lane's words of a row
    static constexpr int KP = KW < 4 ? KW : 4, VP = VW < 4 ? VW : 4;  // of which it loads so many at once
    static constexpr int KS = D / 16;  // k-steps of S^T, products of O^T
    static constexpr int SW = (N + 3) / 4;  // words of a row's scales
    static constexpr int OWN = (TS + 31) / 32;  // slots whose scales a lane loads
    static constexpr int kThreads = 32 * decode_quant_warps(D);
    // a warp's shared memory: a group's rows of floats, or its queries' fragments
    static constexpr __host__ __device__ int warp_bytes(bool pair, int group) {
        const int rows = group * (D + 4) * 4, fragments = KS * (pair ? 1 : 2) * 256;
        return rows > fragments ? rows : fragments;
    }
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

// Whether a byte of the word is 255.
__device__ __forceinline__ bool any_255(uint32_t w) { return ((~w - 0x01010101u) & w & 0x80808080u) != 0; }

// Tiles of TS slots of a sequence, and its length: none where its position or its length allows none.
template <int TS>
__device__ __forceinline__ int tiles_of(const DecodeQuantArgs& a, int b, int& len, uint32_t& err) {
    const int64_t pos = a.q_pos[b];
    len = a.seq_len[b];
    if (len < 0 || len > a.max_len) {  // (max_len is at most the capacity)
        err |= PRCR_ST_CAPACITY;
        len = len < 0 ? 0 : a.max_len;
    }
    if (pos <= -2147483648LL || pos >= 2147483648LL) {
        err |= PRCR_ST_POS_RANGE;
        len = 0;
    }
    return (len + TS - 1) / TS;
}

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {  // of numbers that are not negative, mostly small ones
    return (a | b) >> 32 ? a / b : int64_t(uint32_t(a) / uint32_t(b));
}

// How `total` tiles are cut into the teams' shares: the first `more` have one tile more than the others.
struct Cut {
    int64_t each, more;
    __device__ __forceinline__ int64_t begin_of(int w) const { return w * each + min(int64_t(w), more); }
    __device__ __forceinline__ int team_of(int64_t tile) const {
        const int64_t big = more * (each + 1);
        return int(tile < big ? quotient(tile, each + 1) : more + quotient(tile - big, each));
    }
};
__device__ __forceinline__ Cut cut_of(const DecodeQuantArgs& a, int64_t total) {
    // Shares of one tile at least, or of two where a unit has over 64 on average, whose parts cost more to join than they
    // save (one layer of one sequence, 8 heads: of 16 slots 6.1 us | 9.2 with two, of 933 8.4 | 9.9, but of 4000 16.4 | 13.1).
    const int64_t most = total > 64 * int64_t(a.n_seqs) * a.n_layers * a.head_sets ? total / 2 : total;
    const int64_t teams = max(int64_t(1), min(int64_t(a.teams), most));
    Cut c;
    c.each = quotient(total, teams);
    c.more = total - c.each * teams;
    return c;
}

// A team's share of all sequences', layers' and sets of KV heads' tiles, in that order: tiles begin .. end - 1, the
// first one tile `tile` of `tiles` of unit `unit` (layer, set of heads) of sequence `b`.
struct Share {
    Cut cut;
    int64_t begin, end;
    int team, b, unit, tile, tiles, len;
};
template <int TS>
__device__ __forceinline__ Share share_of(const DecodeQuantArgs& a, int team, uint32_t& err) {
    const int lane = threadIdx.x & 31, per_seq = a.n_layers * a.head_sets;
    Share s;
    s.team = team;
    uint32_t e = 0;
    int len, n = 0;
    int64_t sum = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 32) {
        n = b0 + lane < a.n_seqs ? tiles_of<TS>(a, b0 + lane, len, e) : 0;
        // (2^31 together at most: 2^30 slots each, sixteen to a tile, 32 of them)
        sum += __reduce_add_sync(kFull, unsigned(n));
    }
    err = __reduce_or_sync(kFull, e);
    const Cut cut = s.cut = cut_of(a, sum * per_seq);
    s.begin = min(sum * per_seq, cut.begin_of(s.team));
    s.end = min(sum * per_seq, cut.begin_of(s.team + 1));
    s.b = s.unit = s.tile = s.tiles = s.len = 0;
    if (s.begin >= s.end) return s;
    int64_t before = 0;  // tiles of a unit of the sequences passed
    for (int b0 = 0; b0 < a.n_seqs; b0 += 32) {
        if (a.n_seqs > 32) n = b0 + lane < a.n_seqs ? tiles_of<TS>(a, b0 + lane, len, e) : 0;
        uint32_t upto = uint32_t(n);  // (2^31 at most, as above)
        for (int k = 1; k < 32; k *= 2) {
            const uint32_t x = __shfl_up_sync(kFull, upto, k);
            if (lane >= k) upto += x;
        }
        const uint32_t behind = __ballot_sync(kFull, (before + upto) * per_seq > s.begin);
        if (behind) {
            const int at = __ffs(int(behind)) - 1;
            s.b = b0 + at;
            s.tiles = __shfl_sync(kFull, n, at);
            s.len = __shfl_sync(kFull, len, at);
            before += int64_t(__shfl_sync(kFull, upto, at)) - s.tiles;
            break;
        }
        before += __shfl_sync(kFull, upto, 31);
    }
    const int64_t in = s.begin - before * per_seq;
    s.unit = int(quotient(in, s.tiles));
    s.tile = int(in - int64_t(s.unit) * s.tiles);
    return s;
}

// RUNS: sixteen slots from a multiple of sixteen on lie slot_stride apart (a contiguous cache,
// or blocks of a multiple of 16 slots), so that a lane's rows follow from where the first one
// is. Otherwise lanes look a slot up each and pass its place on (taken for every cache: 502 us for
// 465, 16 sequences of up to 4096 slots, 36 layers).
template <int FMT, int D, bool PAIR, bool RUNS>
__global__ void __launch_bounds__(Shape<FMT, D>::kThreads, 1) decode_quant_kernel(const __grid_constant__ DecodeQuantArgs a) {
    using S = Shape<FMT, D>;
    constexpr bool kFour = S::kFour;
    constexpr int SUB = S::SUB, TS = S::TS, N = S::N, KW = S::KW, VW = S::VW, KP = S::KP, VP = S::VP, KS = S::KS, SW = S::SW, OWN = S::OWN;
    constexpr int P = D / 2, PITCH = D + 4, NP = PAIR ? 1 : 2, LS = PAIR ? 1 : 2;  // products for the pieces of a query or a weight, slots of a lane's logits
    // look places up a tile earlier than they are loaded from, and ask for the rows then (E4M3: 465 us, without 534; E2M1, which
    // does not wait for memory: 201, without 200)
    constexpr bool EARLY = !kFour;
    extern __shared__ __align__(16) float smem[];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, gid = lane >> 2, t = lane & 3;
    const int H = a.n_kv_heads, g = a.group, per_seq = a.n_layers * a.head_sets;
    const int member = warp % a.team;  // (teams do not cross CTAs)
    // a warp's own: its query, as numbers and then as B fragments, and at the end its accumulators
    float* mine = smem + warp * (S::warp_bytes(PAIR, g) / 4);
    uint2* q_frag = reinterpret_cast<uint2*>(mine);
    pdl_wait();
    pdl_allow();  // (the grid is one wave: CTAs that follow take the place of those that are done)
    uint32_t err;
    const int cta_warp = __shfl_sync(kFull, int(blockIdx.x * kCtaWarps + (threadIdx.x >> 5)), 0);
    const Share share = share_of<TS>(a, cta_warp / a.team, err);
    if (cta_warp > 0) err = 0;  // (one tells of lengths and positions)
    if (share.begin >= share.end) {
        if (err) atomicOr(a.status, err);
        return;
    }

    // where the next tile to load is: tile `at` of `n` of unit `unit` of sequence `b`
    bool there;  // whether the set of heads has this warp's
    int b = share.b, unit = share.unit, at = share.tile, n = share.tiles, s_end = share.len;
    const uint8_t *kb, *vb, *kf, *vf;
    auto point = [&]() {  // at the unit's rows
        const int l = unit / a.head_sets, kh = (unit - l * a.head_sets) * a.team + member;
        there = kh < H;
        const int64_t codes = int64_t(l) * a.cache.layer_stride + int64_t(kh) * S::RB;
        const int64_t scales = int64_t(l) * a.cache.scale_layer_stride + int64_t(kh) * N;
        kb = a.cache.k + codes;
        vb = a.cache.v + codes;
        kf = a.cache.k_scale + scales;
        vf = a.cache.v_scale + scales;
    };
    point();
    int64_t left = share.end - share.begin;  // tiles to load
    auto advance = [&]() {
        if (--left <= 0) return;
        if (++at < n) return;
        at = 0;
        if (++unit == per_seq) {
            unit = 0;
            do {
                if (++b == a.n_seqs) {  // (tiles are left: not unless lengths change under the call)
                    left = 0;
                    return;
                }
                n = tiles_of<TS>(a, b, s_end, err);
            } while (n == 0);
        }
        point();
    };

    // A lane's pieces of a run's rows (RUNS: from the run's first one; strides are below 2^27). Lanes whose slots
    // are not there have the last one's that is, whatever they make of it.
    const uint32_t k_off = S::RB >= 64 ? 16 * t : 8 * t, v_off = gid * (S::RB == 256 ? 16 : S::RB / 8);
    uint32_t k_row[SUB][2], v_row[SUB][4], f_row[OWN];
    int rows[SUB];  // of a run that are there
    auto lay_out = [&]() {
        const uint32_t stride = uint32_t(a.cache.slot_stride);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const int last = rows[u] - 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) k_row[u][i] = uint32_t(min(gid + 8 * i, last)) * stride + k_off;
#pragma unroll
            for (int i = 0; i < 4; ++i) v_row[u][i] = uint32_t(min(2 * t + (i & 1) + 8 * (i >> 1), last)) * stride + v_off;
        }
#pragma unroll
        for (int j = 0; j < OWN; ++j)
            f_row[j] = uint32_t(min(lane & 15, (SUB > 1 && lane >= 16 ? rows[(2 * j + 1) % SUB] : rows[2 * j % SUB]) - 1)) * uint32_t(a.cache.scale_slot_stride);
    };
    // Blocks and places of the tile's runs (RUNS), or of slots (lane + 32 j) % TS.
    constexpr int LOOK = RUNS ? SUB : OWN;
    int32_t blk[LOOK];
    auto looked = [&](int j) { return at * TS + (RUNS ? 16 * j : TS == 16 ? lane & 15 : lane + 32 * j); };
    auto blocks = [&]() {
#pragma unroll
        for (int j = 0; j < LOOK; ++j) {
            const int s = looked(j);
            blk[j] = left > 0 && there && s < s_end ? qblock(a.cache, b, uint32_t(s)) : -1;
        }
    };
    QPlace place[LOOK];
    bool full;  // whether all of the tile's slots are there
    if (RUNS) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) rows[u] = 16;
        lay_out();
    }
    const uint8_t *kb_at, *vb_at, *kf_at, *vf_at;  // at the rows of the unit that `place` is in
    auto places = [&]() {
        bool same = true;
        full = true;
        kb_at = kb;
        vb_at = vb;
        kf_at = kf;
        vf_at = vf;
#pragma unroll
        for (int j = 0; j < LOOK; ++j) {
            const int s = looked(j);
            place[j] = {-1, 0};
            if (left > 0 && there && s < s_end) {
                place[j] = qplace_in_block(a.cache, b, uint32_t(s), blk[j]);
                if (place[j].codes < 0) err |= PRCR_ST_NO_BLOCK;
            }
            if (RUNS) {
                const int n = place[j].codes < 0 ? 0 : min(16, s_end - s);
                same = same && n == rows[j];
                rows[j] = n;
                full = full && n == 16;
            } else {
                full = full && place[j].codes >= 0;
            }
        }
        if (RUNS) {
            if (!same) lay_out();
        } else {
            full = __all_sync(kFull, full);
        }
        // towards the L2 cache, so that the loads, which hold registers, are short: a lane a slot's key or value
#pragma unroll
        for (int j = 0; j < (!EARLY ? 0 : RUNS ? SUB : 2 * OWN); ++j) {
            const uint8_t* base = (RUNS ? lane < 16 : j % 2 == 0) ? kb : vb;
            const int64_t at = RUNS ? place[j % LOOK].codes + (lane & 15) * int64_t(a.cache.slot_stride) : place[j / 2 % LOOK].codes;
            const bool ok = RUNS ? (lane & 15) < rows[j % SUB] : at >= 0 && (TS > 16 || lane < 16);
#pragma unroll
            for (int c = 0; c < S::RB; c += 128)
                if (ok) prefetch_l2(base + at + c);
        }
    };
    uint32_t ks[OWN][SW], vs[OWN][SW];  // scales' bytes of slots lane + 32 j
    float bias[OWN];                    // added to their logits: 0, or -inf for a slot that is not there
    auto load_scales = [&]() {
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            int64_t at = place[RUNS ? 0 : j].scales;
            bool ok = place[RUNS ? 0 : j].codes >= 0, row = ok;
            if (RUNS) {
                const bool second = SUB > 1 && lane >= 16;
                const int n = second ? rows[(2 * j + 1) % SUB] : rows[2 * j % SUB];
                at = (second ? place[(2 * j + 1) % SUB].scales : place[2 * j % SUB].scales) + f_row[j];
                ok = (lane & 15) < n;
                row = n > 0;
            }
            bias[j] = ok ? 0.0f : -INFINITY;
            load_row_scales<N>(ks[j], kf_at + at, row);
            load_row_scales<N>(vs[j], vf_at + at, row);
        }
    };
    uint32_t kw[SUB][2][KW], vw[SUB][4][VW];
    auto load_k = [&]() {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            if (RUNS) {
                if (rows[u] > 0) {
                    const uint8_t* run = kb_at + place[u % LOOK].codes;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int c = 0; c < KW / KP; ++c) load_words<KP>(kw[u][i] + KP * c, run + k_row[u][i] + 64 * c);
                } else {
#pragma unroll
                    for (int i = 0; i < 2 * KW; ++i) kw[u][i / KW][i % KW] = 0;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int64_t at = __shfl_sync(kFull, place[u / 2 % LOOK].codes, (16 * u + gid + 8 * i) & 31);
#pragma unroll
                    for (int c = 0; c < KW / KP; ++c) load_words<KP>(kw[u][i] + KP * c, kb_at + at + k_off + 64 * c, at >= 0);
                }
            }
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            if (RUNS) {
                if (rows[u] > 0) {
                    const uint8_t* run = vb_at + place[u % LOOK].codes;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < VW / VP; ++c) load_words<VP>(vw[u][i] + VP * c, run + v_row[u][i] + 128 * c);
                } else {
#pragma unroll
                    for (int i = 0; i < 4 * VW; ++i) vw[u][i / VW][i % VW] = 0;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t at = __shfl_sync(kFull, place[u / 2 % LOOK].codes, (16 * u + 2 * t + (i & 1) + 8 * (i >> 1)) & 31);
#pragma unroll
                    for (int c = 0; c < VW / VP; ++c) load_words<VP>(vw[u][i] + VP * c, vb_at + at + v_off + 128 * c, at >= 0);
                }
            }
        }
    };

    // A group's query rows: a lane has pairs 2 (lane + 32 i) and the next of every head (D = 64: half of the lanes).
    constexpr int G = PAIR ? 4 : 8, PR = P / 64 > 0 ? P / 64 : 1;
    const bool has = P >= 64 || lane < P / 2;
    uint32_t qx[G][PR], qy[G][PR];
    auto load_query = [&](int b, int unit) {
        const int layer = unit / a.head_sets, kh = min((unit - layer * a.head_sets) * a.team + member, H - 1);
        const uint32_t* q = reinterpret_cast<const uint32_t*>(a.q + ((int64_t(b) * a.n_layers + layer) * H + kh) * g * D) + lane;
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
            for (int i = 0; i < PR; ++i) {
                const bool ok = has && h < g;
                qx[h][i] = ok ? q[h * P + 32 * i] : 0u;
                qy[h][i] = ok ? q[h * P + 32 * i + P / 2] : 0u;
            }
    };

    // the first tile is requested before the query is worked on
    bool whole_tile;  // whether all slots of the tile that is loaded are there
    auto load_first = [&]() {
        blocks();
        places();
        load_k();
        load_scales();
        load_v();
        whole_tile = full;
        advance();
        blocks();
        if (EARLY) {
            places();
            advance();
            blocks();
        }
    };
    load_query(share.b, share.unit);
    load_first();

    // the unit that is attended to
    int ub = share.b, uu = share.unit, first = share.tile, un = share.tiles;
    int64_t todo = share.end - share.begin;
    bool step0 = true;  // the share's first unit
    uint32_t again = 0;  // E2M1: groups of the unit's dims that are worked on once more, the lowest one now
    const int h0 = PAIR ? 2 * (t & 1) : 2 * t;  // this lane's heads are h0 and h0 + 1, in S^T's columns and in O^T's
    while (true) {
    const int layer = uu / a.head_sets, kh = (uu - layer * a.head_sets) * a.team + member;
    const int64_t head0 = ((int64_t(ub) * a.n_layers + layer) * H + min(kh, H - 1)) * g;  // its group's first query head
    float qs[2] = {0.0f, 0.0f};
    {
        // the group's queries, rotated at (p, p, p): pair i turns by p * rate i whatever its band
        const double pos = double(a.q_pos[ub]);
        float cs[PR][2], sn[PR][2];
#pragma unroll
        for (int i = 0; i < PR; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (has) sincos_turns(pos, a.turn_freq[2 * (lane + 32 * i) + k], &sn[i][k], &cs[i][k]);
        if (!step0 || (kFour && again)) load_query(ub, uu);
#pragma unroll
        for (int h = 0; h < G; ++h) {
            if (h >= g) break;
            float x[PR][2], y[PR][2];
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < PR; ++i) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float u = k ? hi_f32(qx[h][i]) : lo_f32(qx[h][i]), v = k ? hi_f32(qy[h][i]) : lo_f32(qy[h][i]);
                    x[i][k] = has ? fmaf(u, cs[i][k], -v * sn[i][k]) * a.scale_log2 : 0.0f;
                    y[i][k] = has ? fmaf(v, cs[i][k], u * sn[i][k]) * a.scale_log2 : 0.0f;
                    most = max(most, max(__float_as_uint(x[i][k]) & 0x7fffffffu, __float_as_uint(y[i][k]) & 0x7fffffffu));
                }
            }
            most = __reduce_max_sync(kFull, most);
            // times 2^up: below 2^14 (2^40 at most, so that a logit times it stays finite)
            const int up = min(40, 13 - (int(most >> 23) - 127));
            const float f = __uint_as_float(uint32_t(127 + up) << 23), down = __uint_as_float(uint32_t(127 - up) << 23);
            if (has) {
#pragma unroll
                for (int i = 0; i < PR; ++i) {
                    *reinterpret_cast<float2*>(mine + h * PITCH + 2 * (lane + 32 * i)) = make_float2(x[i][0] * f, x[i][1] * f);
                    *reinterpret_cast<float2*>(mine + h * PITCH + 2 * (lane + 32 * i) + P) = make_float2(y[i][0] * f, y[i][1] * f);
                }
            }
            if (h == h0) qs[0] = down;
            if (h == h0 + 1) qs[1] = down;
        }
        __syncwarp();
        // B fragments. Column r of a product is head r, or with pairs head r % 4, r / 4 its first or second piece.
        const int h = PAIR ? gid & 3 : gid;
        const bool hv = h < g;
        const float* row = mine + (hv ? h : 0) * PITCH;
        uint2 f[KS][NP];
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const float4 v = *reinterpret_cast<const float4*>(row + (kFour ? S::kdim(t, j >> 1) + 4 * (j & 1) : S::kdim(t, j)));
            uint2 hi, lo;
            split_f16x2(hv ? v.x : 0.0f, hv ? v.y : 0.0f, hi.x, lo.x);
            split_f16x2(hv ? v.z : 0.0f, hv ? v.w : 0.0f, hi.y, lo.y);
            f[j][0] = PAIR && gid >= 4 ? lo : hi;
            if (!PAIR) f[j][NP - 1] = lo;
        }
        __syncwarp();  // every lane has read them
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int z = 0; z < NP; ++z) q_frag[(j * NP + z) * 32 + lane] = f[j][z];
    }

    float o[KS][4];
#pragma unroll
    for (int j = 0; j < KS; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
    // references: m of the sums; r, less kWeightLog2, of the accumulators
    float m[2] = {kNone, kNone}, r[2] = {kNone, kNone}, sum[2] = {0.0f, 0.0f};
    uint32_t nan_groups = 0;  // E2M1: groups of dims that a value makes NaN
    uint32_t below[SW], used[SW];  // E2M1: bits of how far the groups' scales were below their rows' largest, and of the scales
#pragma unroll
    for (int i = 0; i < SW; ++i) below[i] = used[i] = 0;

    const int steps = int(min(int64_t(un - first), todo));
    for (int step = 0; step < steps; ++step) {
        // what the lanes know of this tile's slots: the key's scale (E4M3; E2M1: bf16 of its groups'), the value's exponent
        // (E2M1: the largest, and fp16 of its groups' scales in units of that one)
        float kx[OWN], vx[OWN];
        uint32_t kg[OWN][(N + 1) / 2], vg[OWN][(N + 1) / 2];
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            if constexpr (kFour) {
                if (again) {  // all groups as if they had this one's scale
                    const int only = __ffs(int(again)) - 1;
                    const uint32_t byte = ((SW > 1 && only >= 4 ? vs[j][SW - 1] : vs[j][0]) >> (8 * (only & 3))) & 255;
#pragma unroll
                    for (int i = 0; i < SW; ++i) vs[j][i] = byte * 0x01010101u;
                }
                bool nan = false;
#pragma unroll
                for (int i = 0; i < SW; ++i) nan |= any_255(vs[j][i]);
                if (nan) {  // noted for the end, and without influence on the other groups
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (((vs[j][i / 4] >> (8 * (i % 4))) & 255) == kScaleNan) {
                            nan_groups |= 1u << i;
                            vs[j][i / 4] &= ~(255u << (8 * (i % 4)));
                        }
                }
                int top = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) top = max(top, int((vs[j][i / 4] >> (8 * (i % 4))) & 255));
#pragma unroll
                for (int i = 0; i < SW; ++i) {
                    below[i] |= uint32_t(top) * 0x01010101u - vs[j][i];
                    used[i] |= vs[j][i];
                }
                // (a byte behind the bits of 2^23 is 2^23 + byte)
                const float most = __uint_as_float(0x4b000000u + top);
                vx[j] = most - 8388735.0f;
#pragma unroll
                for (int i = 0; i < N; i += 2) {
                    kg[j][i / 2] = bf16_of_scales(ks[j][i / 4] >> (8 * (i % 4)));
                    vg[j][i / 2] = pack_f16x2(ex2(__uint_as_float(__byte_perm(vs[j][i / 4], 0x4b000000u, 0x7650u + i % 4)) - most),
                                              ex2(__uint_as_float(__byte_perm(vs[j][i / 4], 0x4b000000u, 0x7651u + i % 4)) - most));
                }
            } else {
                kx[j] = scale_value(int(ks[j][0]));
                vx[j] = vs[j][0] == kScaleNan ? __uint_as_float(0x7fffffffu) : float(int(vs[j][0]) - 127);
            }
        }

        // S^T of all subtiles, so that a fragment of the query is read once
        constexpr int NC = kFour ? N : 2;  // sums: of the groups, or two to be shorter
        float x[SUB][LS][2], ve[SUB][LS], c[SUB][NC][4];
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            uint32_t p[SUB][4], q[SUB][4];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if constexpr (kFour) {
                    f16_of_e2m1(kw[u][0][i], p[u]);
                    f16_of_e2m1(kw[u][1][i], q[u]);
                } else {
                    uint32_t a2[2], b2[2];
                    f16_of_e4m3(kw[u][0][i], a2);
                    f16_of_e4m3(kw[u][1][i], b2);
                    p[u][0] = a2[0]; p[u][1] = a2[1]; q[u][0] = b2[0]; q[u][1] = b2[1];
                }
            }
            constexpr int E = kFour ? 2 : 1;  // k-steps of a word
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int z = 0; z < NP; ++z) {
                    const uint2 f = q_frag[((E * i + e) * NP + z) * 32 + lane];
                    const int to = kFour ? (2 * i + e) % N : (i + z) & 1;
                    const bool begins = kFour ? 2 * i + e < N && z == 0 : i + z < 2 && (i == 0 || NP == 1);
#pragma unroll
                    for (int u = 0; u < SUB; ++u) {
                        if (begins) mma_f16_first(c[u][to], p[u][2 * e], q[u][2 * e], p[u][2 * e + 1], q[u][2 * e + 1], f.x, f.y);
                        else mma_f16(c[u][to], p[u][2 * e], q[u][2 * e], p[u][2 * e + 1], q[u][2 * e + 1], f.x, f.y);
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            float d[4];
            if constexpr (kFour) {
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    const uint32_t wa = __shfl_sync(kFull, kg[u / 2][k], (16 * u + gid) & 31);
                    const uint32_t wb = __shfl_sync(kFull, kg[u / 2][k], (16 * u + gid + 8) & 31);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float fa = e ? hi_f32(wa) : lo_f32(wa), fb = e ? hi_f32(wb) : lo_f32(wb);
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const float v = c[u][2 * k + e][y], f = y < 2 ? fa : fb;
                            d[y] = k + e == 0 ? v * f : fmaf(v, f, d[y]);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = c[u][0][i] + c[u][1][i];
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
                ve[u][i] = __shfl_sync(kFull, vx[u / 2], from);
                const float f = kFour ? 1.0f : __shfl_sync(kFull, kx[u / 2], from);
#pragma unroll
                for (int z = 0; z < 2; ++z) x[u][i][z] = (kFour ? d[2 * i + z] : d[2 * i + z] * f) * qs[z];
                if (!whole_tile) {
                    const float add = __shfl_sync(kFull, bias[u / 2], from);
                    x[u][i][0] += add;
                    x[u][i][1] += add;
                }
            }
        }
        // the keys' registers are free: the next tile's
        if (!EARLY) places();
        load_k();
        load_scales();
        whole_tile = full;

        // a logit past its reference by more than the slack moves the references
        bool far = false;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < LS; ++i)
#pragma unroll
                for (int z = 0; z < 2; ++z)
                    far |= x[u][i][z] - m[z] > kSlack || (x[u][i][z] + ve[u][i]) - r[z] > kSlack + kWeightLog2;
        if (__any_sync(kFull, far)) {
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float mx = m[z], rx = r[z];
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < LS; ++i) {
                        mx = fmaxf(mx, x[u][i][z]);
                        rx = fmaxf(rx, x[u][i][z] + ve[u][i] - kWeightLog2);
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
        // B fragments of P^T: [first and second piece][slots 0..7, 8..15]; E2M1: factors of them for its groups
        uint32_t pf[SUB][NP][2], rel[SUB][2];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            {
                uint32_t hi[LS], lo[LS];
#pragma unroll
                for (int i = 0; i < LS; ++i) {
                    float w[2];
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        sum[z] += ex2(x[u][i][z] - m[z]);
                        w[z] = ex2((x[u][i][z] + ve[u][i]) - r[z]);
                    }
                    split_f16x2(w[0], w[1], hi[i], lo[i]);
                }
                if (PAIR) {
                    const uint32_t got = __shfl_xor_sync(kFull, t < 2 ? lo[0] : hi[0], 2);
                    pf[u][0][0] = transposed(t < 2 ? hi[0] : got);
                    pf[u][0][1] = transposed(t < 2 ? got : lo[0]);
                } else {
#pragma unroll
                    for (int i = 0; i < LS; ++i) {
                        pf[u][0][i] = transposed(hi[i]);
                        pf[u][NP - 1][i] = transposed(lo[i]);
                    }
                }
            }
            if constexpr (kFour) {
                // The groups' scales as factors of P^T's pairs of slots: a matrix of slots by groups, transposed as P is; its rows
                // (N = 2, 4: of slots 0..7, then of 8..15) are read by every lane.
                if (N == 8) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int from = (16 * u + gid + 8 * i) & 31;
                        const uint32_t w0 = __shfl_sync(kFull, vg[u / 2][0], from), w1 = __shfl_sync(kFull, vg[u / 2][1 % ((N + 1) / 2)], from);
                        const uint32_t w2 = __shfl_sync(kFull, vg[u / 2][2 % ((N + 1) / 2)], from), w3 = __shfl_sync(kFull, vg[u / 2][3 % ((N + 1) / 2)], from);
                        rel[u][i] = transposed(t < 2 ? (t == 0 ? w0 : w1) : (t == 2 ? w2 : w3));
                    }
                } else if (N == 4) {
                    const int from = (16 * u + gid + 8 * (t >> 1)) & 31;
                    const uint32_t w0 = __shfl_sync(kFull, vg[u / 2][0], from), w1 = __shfl_sync(kFull, vg[u / 2][1 % ((N + 1) / 2)], from);
                    rel[u][0] = transposed(t & 1 ? w1 : w0);
                } else {
                    rel[u][0] = transposed(__shfl_sync(kFull, vg[u / 2][0], (16 * u + gid + 8 * (t & 1)) & 31));
                }
            }
        }
        // O^T, summed over a tile before it joins the accumulators
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            float part[kFour ? 4 : 2][4];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if constexpr (kFour) {
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
                        const uint32_t f0 = __shfl_sync(kFull, rel[u][0], 4 * grp + t);
                        const uint32_t f1 = N == 8 ? __shfl_sync(kFull, rel[u][1], 4 * grp + t) : __shfl_sync(kFull, rel[u][0], 4 * (grp + N) + t);
#pragma unroll
                        for (int z = 0; z < NP; ++z) {
                            const uint32_t b0 = mul_f16x2(pf[u][z][0], f0), b1 = mul_f16x2(pf[u][z][1], f1);
#pragma unroll
                            for (int k = 2 * e; k < 2 * e + 2; ++k) {
                                if (u + z == 0) mma_f16_first(part[k], ev[0][k], od[0][k], ev[1][k], od[1][k], b0, b1);
                                else mma_f16(part[k], ev[0][k], od[0][k], ev[1][k], od[1][k], b0, b1);
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // dims 2e and 2e + 1 of the word, of two slots each
                        uint32_t p[2], q[2];
                        f16_of_e4m3(__byte_perm(vw[u][0][i], vw[u][1][i], e ? 0x7362 : 0x5140), p);
                        f16_of_e4m3(__byte_perm(vw[u][2][i], vw[u][3][i], e ? 0x7362 : 0x5140), q);
#pragma unroll
                        for (int z = 0; z < NP; ++z) {
                            if (u + z == 0) mma_f16_first(part[e], p[0], p[1], q[0], q[1], pf[u][z][0], pf[u][z][1]);
                            else mma_f16(part[e], p[0], p[1], q[0], q[1], pf[u][z][0], pf[u][z][1]);
                        }
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < (kFour ? 4 : 2); ++k) add_to(o[(kFour ? 4 : 2) * i + k], part[k]);
        }
        load_v();
        if (EARLY) places();
        advance();
        blocks();
    }

    // join the lanes' sums and the two pieces
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
    if (kFour) nan_groups = __reduce_or_sync(kFull, nan_groups);
    // the whole unit: its outputs; a part of one: what is joined later, in place 0 where it begins with
    // this team's share, else in place 1
    const bool whole = first == 0 && steps == un;
    float* dst = whole ? a.out + head0 * D
                       : a.partial + ((int64_t(share.team) * 2 + (step0 ? 0 : 1)) * a.team + member) * g * (D + 2);
    const int pitch = whole ? D : D + 2;
    __syncwarp();  // the fragments are read
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const int h = h0 + z;
        if (h >= g || kh >= H || (PAIR && t >= 2)) continue;
        const float to_m = kFour && again && !whole ? dst[h * pitch + D] : m[z];  // (that of the part's sums, kept the first time)
        const float f = ex2(r[z] - to_m) * (!whole ? 1.0f : sum[z] == 0.0f ? 0.0f : 1.0f / sum[z]);  // to the sums' reference
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const int d = kFour ? S::vdim(gid, j / 4) + 2 * (j % 4) : S::vdim(gid, j / 2) + 2 * (j % 2);
            const float to = kFour && (nan_groups >> (d / 4 % N) & 1) ? __uint_as_float(0x7fffffffu) : f;
            *reinterpret_cast<float2*>(mine + h * PITCH + d) = make_float2(o[j][z] * to, o[j][2 + z] * to);
        }
        if (gid == 0 && !whole && !(kFour && again)) *reinterpret_cast<float2*>(dst + h * pitch + D) = make_float2(m[z], sum[z]);
    }
    __syncwarp();
    for (int e = lane; e < (kh < H ? g * P : 0); e += 32) {
        const int h = e / P, d = 2 * (e - h * P);
        if (kFour && again && d / 4 % N != __ffs(int(again)) - 1) continue;
        *reinterpret_cast<float2*>(dst + h * pitch + d) = *reinterpret_cast<const float2*>(mine + h * PITCH + d);
    }
    __syncwarp();
    if constexpr (kFour) {
        if (again) {
            again &= again - 1;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t low = __reduce_or_sync(kFull, below[i / 4] >> (8 * (i % 4)) & kFarBelow);
                const uint32_t any = __reduce_or_sync(kFull, used[i / 4] >> (8 * (i % 4)) & kLeastUsed);
                if (low && any && !(nan_groups >> i & 1)) again |= 1u << i;
            }
        }
        if (again) {  // back to the unit's first tile
            b = ub;
            unit = uu;
            at = first;
            n = un;
            left = todo;
            tiles_of<TS>(a, b, s_end, err);
            point();
            load_first();
            continue;
        }
    }
    todo -= steps;
    if (todo <= 0) break;
    step0 = false;
    first = 0;
    if (++uu == per_seq) {
        uu = 0;
        int len;
        do un = ++ub < a.n_seqs ? tiles_of<TS>(a, ub, len, err) : -1; while (un == 0);
        if (un < 0) break;
    }
    }
    if (err) atomicOr(a.status, err);
}

// What the join kernels do to a query head's row, a warp or a CTA: parts of teams w0 .. w1, eight of them requested at once.
template <int D, int WARPS>
__device__ __forceinline__ void join_row(const DecodeQuantArgs& a, float* out, const Cut& cut, int64_t u0, int w0, int w1, int member, int h) {
    constexpr int NV = D / 64, AHEAD = 8;
    __shared__ float2 s_acc[WARPS][D / 2];
    __shared__ float s_top[WARPS], s_den[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = a.group;
    const int place0 = cut.begin_of(w0) != u0 ? 1 : 0;  // in the first team's parts; the others' begin with their shares
    float M = kNone, den = 0.0f;
    float2 acc[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) acc[k] = make_float2(0.0f, 0.0f);
    for (int w = w0 + (WARPS > 1 ? warp : 0); w <= w1; w += AHEAD * WARPS) {
        float2 mz[AHEAD], y[AHEAD][NV];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int at = w + i * WARPS;
            const float* part = a.partial + (((int64_t(at) * 2 + (at == w0 ? place0 : 0)) * a.team + member) * g + h) * (D + 2);
            const bool ok = at <= w1;
            mz[i] = ok ? *reinterpret_cast<const float2*>(part + D) : make_float2(kNone, 0.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k) y[i][k] = ok ? *reinterpret_cast<const float2*>(part + 2 * lane + 64 * k) : make_float2(0.0f, 0.0f);
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, mz[i].x);
        const float old = ex2(M - top);
        M = top;
        den *= old;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            acc[k].x *= old;
            acc[k].y *= old;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = ex2(mz[i].x - top);
            den = fmaf(mz[i].y, f, den);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                acc[k].x = fmaf(y[i][k].x, f, acc[k].x);
                acc[k].y = fmaf(y[i][k].y, f, acc[k].y);
            }
        }
    }
    if constexpr (WARPS > 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) s_acc[warp][lane + 32 * k] = acc[k];
        if (lane == 0) {
            s_top[warp] = M;
            s_den[warp] = den;
        }
        __syncthreads();
        if (warp > 0) return;
        for (int w = 1; w < WARPS; ++w) {
            const float top = fmaxf(M, s_top[w]), fa = ex2(M - top), fb = ex2(s_top[w] - top);
            M = top;
            den = den * fa + s_den[w] * fb;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                acc[k].x = acc[k].x * fa + s_acc[w][lane + 32 * k].x * fb;
                acc[k].y = acc[k].y * fa + s_acc[w][lane + 32 * k].y * fb;
            }
        }
    }
    const float inv = den == 0.0f ? 0.0f : 1.0f / den;
#pragma unroll
    for (int k = 0; k < NV; ++k) *reinterpret_cast<float2*>(out + 2 * lane + 64 * k) = make_float2(acc[k].x * inv, acc[k].y * inv);
}

// Joins the parts of the units that several teams shared, and writes zeros for sequences without any slot: a query
// head's row a warp, or, where eight teams or more share a unit, a CTA (8 sequences of one layer, 4 heads of 256: 38 us, by
// warps 45; 16 of 36 layers: 465 by warps, by CTAs 495).
template <int D, int TS, int WARPS>
__global__ void __launch_bounds__(128) decode_quant_join_kernel(const __grid_constant__ DecodeQuantArgs a) {
    pdl_allow();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = a.group;
    const int64_t row = WARPS > 1 ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + warp;
    const int per_seq = a.n_layers * a.head_sets, heads = a.n_layers * a.n_kv_heads;
    const int64_t head = min(quotient(row, g), int64_t(a.n_seqs) * heads - 1);
    const int h = int(row - head * g), b = int(quotient(head, heads)), lh = int(head - int64_t(b) * heads);
    const int layer = lh / a.n_kv_heads, kh = lh - layer * a.n_kv_heads, unit = layer * a.head_sets + kh / a.team, member = kh % a.team;
    // the sequences' tiles again, while the kernel before this one ends (lengths and positions are the call's inputs: whatever wrote
    // them was complete before that kernel began)
    int64_t before = 0, total = 0;
    int n = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 32) {
        uint32_t e;
        int len;
        const int x = b0 + lane < a.n_seqs ? tiles_of<TS>(a, b0 + lane, len, e) : 0;
        before += __reduce_add_sync(kFull, unsigned(b0 + lane < b ? x : 0));
        total += __reduce_add_sync(kFull, unsigned(x));
        n += __reduce_add_sync(kFull, unsigned(b0 + lane == b ? x : 0));
    }
    const Cut cut = cut_of(a, total * per_seq);
    const int64_t u0 = before * per_seq + int64_t(unit) * n, u1 = u0 + n;
    const int w0 = n ? cut.team_of(u0) : 0, w1 = n ? cut.team_of(u1 - 1) : 0;
    pdl_wait();
    if (h >= g) return;  // (past the last row)
    float* out = a.out + row * D;
    if (n == 0) {
        if (WARPS == 1 || warp == 0)
            for (int d = lane; d < D; d += 32) out[d] = 0.0f;
        return;
    }
    if (w0 != w1) join_row<D, WARPS>(a, out, cut, u0, w0, w1, member, h);
}

// The same where there are twice as many rows as teams and heads of theirs, or more, so that most units are one team's: a warp for
// a row of the unit in which a team's share begins, if that is the unit's first such share (32 sequences of 100 slots, 36 layers: 68
// us for 80, 1024 of them 1.7 ms for 3.6; but 8 sequences, 28 layers of 4 heads 204 for 200).
template <int D, int TS>
__global__ void __launch_bounds__(128) decode_quant_join_teams_kernel(const __grid_constant__ DecodeQuantArgs a) {
    pdl_allow();
    const int lane = threadIdx.x & 31, warp = int(blockIdx.x * 4 + (threadIdx.x >> 5)), rows = a.team * a.group;
    const int w = warp / rows, member = (warp - w * rows) / a.group, h = warp % a.group;
    uint32_t e;
    const Share s = share_of<TS>(a, w, e);
    pdl_wait();
    const int layer = s.unit / a.head_sets, kh = (s.unit - layer * a.head_sets) * a.team + member;
    const int64_t u0 = s.begin - s.tile;
    if (s.begin < s.end && s.tile > 0 && kh < a.n_kv_heads && s.cut.begin_of(w - 1) <= u0) {
        const int64_t row = ((int64_t(s.b) * a.n_layers + layer) * a.n_kv_heads + kh) * a.group + h;
        join_row<D, 1>(a, a.out + row * D, s.cut, u0, w - 1, s.cut.team_of(u0 + s.tiles - 1), member, h);
    }
    const int64_t all = int64_t(a.n_layers) * a.n_kv_heads * a.group * D;
    for (int b = warp; b < a.n_seqs; b += int(gridDim.x) * 4) {
        int len;
        if (tiles_of<TS>(a, b, len, e)) continue;
        for (int64_t i = lane; i < all / 4; i += 32) reinterpret_cast<float4*>(a.out + b * all)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
}

template <int FMT, int D>
cudaError_t launch_fd(const DecodeQuantArgs& a, cudaStream_t stream) {
    using S = Shape<FMT, D>;
    const bool pair = a.group <= 4;
    const bool runs = (a.cache.kind == PRCR_CACHE_CONTIGUOUS || a.cache.block_size % 16 == 0) &&
                      std::max(a.cache.slot_stride, a.cache.scale_slot_stride) < (int64_t(1) << 27);
    const size_t smem = size_t(kCtaWarps) * S::warp_bytes(pair, a.group);
    auto k = pair ? (runs ? decode_quant_kernel<FMT, D, true, true> : decode_quant_kernel<FMT, D, true, false>)
                  : (runs ? decode_quant_kernel<FMT, D, false, true> : decode_quant_kernel<FMT, D, false, false>);
    static_assert(kCtaWarps * S::warp_bytes(false, 8) <= 48 * 1024 && kCtaWarps * S::warp_bytes(true, 4) <= 48 * 1024,
                  "a launch takes up to 48 KB as it is");
    const cudaError_t e = launch_pdl(k, dim3(unsigned((a.teams * a.team + kCtaWarps - 1) / kCtaWarps)), dim3(kCtaWarps * 32), smem, stream, a);
    if (e != cudaSuccess) return e;
    const int64_t units = int64_t(a.n_seqs) * a.n_layers * a.head_sets, rows = int64_t(a.n_seqs) * a.n_layers * a.n_kv_heads * a.group;
    const int64_t by_team = int64_t(a.teams) * a.team * a.group;
    if (rows >= 2 * by_team) return launch_pdl(decode_quant_join_teams_kernel<D, S::TS>, dim3(unsigned((by_team + 3) / 4)), dim3(128), 0, stream, a);
    return a.teams >= 8 * units ? launch_pdl(decode_quant_join_kernel<D, S::TS, 4>, dim3(unsigned(rows)), dim3(128), 0, stream, a)
                                : launch_pdl(decode_quant_join_kernel<D, S::TS, 1>, dim3(unsigned((rows + 3) / 4)), dim3(128), 0, stream, a);
}

template <int FMT>
cudaError_t launch_f(const DecodeQuantArgs& a, cudaStream_t stream) {
    return a.head_dim == 64 ? launch_fd<FMT, 64>(a, stream) : a.head_dim == 128 ? launch_fd<FMT, 128>(a, stream) : launch_fd<FMT, 256>(a, stream);
}

}  // namespace

cudaError_t launch_decode_quant(const DecodeQuantArgs& a, cudaStream_t stream) {
    return a.format == PRCR_QFMT_E4M3 ? launch_f<PRCR_QFMT_E4M3>(a, stream) : launch_f<PRCR_QFMT_E2M1>(a, stream);
}

template <int FMT>
int tile_of(int head_dim) {
    return head_dim == 64 ? Shape<FMT, 64>::TS : head_dim == 128 ? Shape<FMT, 128>::TS : Shape<FMT, 256>::TS;
}

int decode_quant_tile(int format, int head_dim) {
    return format == PRCR_QFMT_E4M3 ? tile_of<PRCR_QFMT_E4M3>(head_dim) : tile_of<PRCR_QFMT_E2M1>(head_dim);
}

}  // namespace prcr

// The formats of a quantised cache on the device: where a slot's codes and scales
// lie, and the rounding of bf16 or float32 rows to codes and back.
//
// A group's scale is 2^e, e >= -117 the least with amax <= top * 2^e (top 448 in
// E4M3, 6 in E2M1), held as the byte e + 127. A value times a power of two is exact,
// so the only rounding is the conversion's own (nearest, ties to even), and what a
// code stands for, of at most four significant bits, is exact in bf16.
#pragma once

#include "prcr_cache.cuh"

namespace prcr {

constexpr int kScaleLeast = 10;  // the byte of 2^-117
constexpr int kScaleNan = 255;   // of a group with an infinity or NaN: it reads as NaN

template <int FMT> struct QFormat;
template <> struct QFormat<PRCR_QFMT_E4M3> {
    // 448 = 1.75 * 2^8: a magnitude 1.m * 2^E takes 2^(E - 8), or 2^(E - 7) above 1.75
    static constexpr uint32_t kCarry = 0x1fffff;  // carries into the exponent where m > 0.75
    static constexpr int kShift = 8;
    // In the highest scale a value could round up to 2^128, which bf16 does not hold: it is
    // rounded down, to the code below that.
    static constexpr int kHighest = 247;
    static constexpr float kHighestTop = 240.0f;
    static constexpr int kBytes8 = 8;  // of codes of eight dims
};
template <> struct QFormat<PRCR_QFMT_E2M1> {
    static constexpr uint32_t kCarry = 0x3fffff;  // 6 = 1.5 * 2^2
    static constexpr int kShift = 2;
    static constexpr int kHighest = 253;
    static constexpr float kHighestTop = 3.0f;
    static constexpr int kBytes8 = 4;
};

// The scale's byte of a group whose largest magnitude has these float32 bits.
template <int FMT>
__device__ __forceinline__ int scale_byte(uint32_t amax) {
    if (amax >= 0x7f800000u) return kScaleNan;
    return max(kScaleLeast, int((amax + QFormat<FMT>::kCarry) >> 23) - QFormat<FMT>::kShift);
}

// 2^(byte - 127): NaN for 255 (0 is the subnormal 2^-127).
__device__ __forceinline__ float scale_value(int byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == kScaleNan ? 0x7fffffffu : uint32_t(byte) << 23);
}

// Codes of x[0..3] (low bits first) in a group with this scale byte.
__device__ __forceinline__ uint32_t codes_e4m3(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return uint32_t(lo) | uint32_t(hi) << 16;
}
__device__ __forceinline__ uint32_t codes_e2m1(const float (&x)[8]) {
    uint32_t r;
    asm("{\n.reg .b8 p0, p1, p2, p3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 p0, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 p1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 p2, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 p3, %8, %7;\n"
        "mov.b32 %0, {p0, p1, p2, p3};\n}"
        : "=r"(r)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}

// f16x2 of two codes each: a word of E4M3's four, or of E2M1's eight.
__device__ __forceinline__ void f16_of_e4m3(uint32_t w, uint32_t (&h)[2]) {
    asm("{\n.reg .b16 l, u;\nmov.b32 {l, u}, %2;\n"
        "cvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, u;\n}"
        : "=r"(h[0]), "=r"(h[1]) : "r"(w));
}
__device__ __forceinline__ void f16_of_e2m1(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n.reg .b8 p0, p1, p2, p3;\nmov.b32 {p0, p1, p2, p3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, p0;\ncvt.rn.f16x2.e2m1x2 %1, p1;\n"
        "cvt.rn.f16x2.e2m1x2 %2, p2;\ncvt.rn.f16x2.e2m1x2 %3, p3;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}

// Where a slot's rows begin (layer and head terms excluded), in bytes; codes -1: nowhere.
struct QPlace {
    int64_t codes, scales;
};

__device__ __forceinline__ QPlace qplace_in_block(const QCacheView& c, int b, uint32_t slot, int32_t blk) {
    if (c.kind == PRCR_CACHE_CONTIGUOUS)
        return {int64_t(b) * c.seq_stride + int64_t(slot) * c.slot_stride,
                int64_t(b) * c.scale_seq_stride + int64_t(slot) * c.scale_slot_stride};
    if (blk < 0 || blk >= c.n_blocks) return {-1, 0};
    const uint32_t o = slot - uint32_t((uint64_t(slot) * c.div_mul) >> c.div_shift) * uint32_t(c.block_size);
    return {int64_t(blk) * c.block_stride + int64_t(o) * c.slot_stride,
            int64_t(blk) * c.scale_block_stride + int64_t(o) * c.scale_slot_stride};
}

// The entry of a sequence's table that a slot's block has (0 for a contiguous cache).
__device__ __forceinline__ int32_t qblock(const QCacheView& c, int b, uint32_t slot) {
    if (c.kind == PRCR_CACHE_CONTIGUOUS) return 0;
    return c.block_table[int64_t(b) * c.bt_stride + uint32_t((uint64_t(slot) * c.div_mul) >> c.div_shift)];
}

__device__ __forceinline__ QPlace qplace(const QCacheView& c, int b, int64_t slot, uint32_t& err) {
    if (slot < 0 || slot >= c.capacity || slot >= (int64_t(1) << 31)) {
        err |= PRCR_ST_CAPACITY;
        return {-1, 0};
    }
    const QPlace p = qplace_in_block(c, b, uint32_t(slot), qblock(c, b, uint32_t(slot)));
    if (p.codes < 0) err |= PRCR_ST_NO_BLOCK;
    return p;
}

}  // namespace prcr

// twk_cache.cuh -- the pages of a cache held in 4 bits: layout, and the rounding of a group of
// values to codes.
//
// A page holds kPage slots of one unit.  Rows (one slot's key or value, D values) are held in
// groups of 64: per group a bf16 scale s, a zero z in 0..15, and a code c in 0..15 per value,
// which stands for s (c - z).
//
// The layout is the one in which the attention kernel's threads find their operands.  In an
// m16n8k16 multiplication thread 4 g + t of a warp holds rows g and g + 8 of the left operand, and
// of each row the columns 2 t, 2 t + 1, 2 t + 8, 2 t + 9 (sums may take the columns in any order,
// as long as both operands do).
//   keys     rows are slots, columns are dimensions.  A slot's codes are D / 2 bytes; thread t's
//            share of them, the dimensions 64 G + 16 t + [0, 16) of every group G, is contiguous.
//            The 8 codes of a word are pairs (2 p, 2 p + 1) in nibbles p and 4 + p, so that
//            (word >> 4 p) & 0x000f000f holds a pair in two halves.
//   values   rows are dimensions, columns are slots: 16 bytes of thread (g, t) hold the dimensions
//            16 m + g and 16 m + 8 + g of 16 slots each, the 8 codes of a word again as 4 pairs.
//   zeros    -(128 + z) as bf16, so that z is in the last bits and a code as the bf16 number 128 + c
//            plus it is c - z.  Beside the scale for keys; for values in the order of the slots in
//            the operand.
#pragma once
#include <cstdint>

namespace twk {

constexpr int kPage = 64;   // slots

template <int D>
struct PageLayout {
    static constexpr int kGroups = D / 64;
    static constexpr int kRow = D / 2;                              // a slot's key codes, bytes
    static constexpr int kKeyGroups = kPage * kRow;                 // u32 [slot][G]
    static constexpr int kValCodes = kKeyGroups + kPage * kGroups * 4;
    static constexpr int kValScales = kValCodes + kPage * kRow;     // bf16 [slot][G]
    static constexpr int kValZeros = kValScales + kPage * kGroups * 2;
    static constexpr int kPos = kValZeros + kPage * kGroups * 2;    // int32 [slot]
    static constexpr int kBytes = kPos + kPage * 4;

    // byte offset of the word with a slot's key dimensions 8 j .. 8 j + 7
    __host__ __device__ static constexpr int key_word(int slot, int j)
    {
        return slot * kRow + (j % 8 / 2) * (8 * kGroups) + (j / 8) * 8 + (j & 1) * 4;
    }
    // element of kValZeros
    __host__ __device__ static constexpr int val_zero(int group, int slot)
    {
        return group * kPage + slot % 8 / 2 * 16 + slot / 16 * 4 + slot % 16 / 8 * 2 + (slot & 1);
    }
};

// a pair of codes as bf16 numbers 128 + c: the code sits in the last bits of 128's fraction
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int p)
{
    return ((word >> (4 * p)) & 0x000f000fu) | 0x43004300u;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// f32 -> bf16 bits, nearest even; two values, the first in the low half
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// two bf16 numbers at a time; a NaN stays one
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// (a x + b, a y + b) in one instruction
__device__ __forceinline__ void fma_pair(float& x, float& y, float a, float b)
{
    asm("{.reg .b64 v, m, c;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 m, {%2, %2};\n\t"
        "mov.b64 c, {%3, %3};\n\tfma.rn.f32x2 v, v, m, c;\n\tmov.b64 {%0, %1}, v;}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b));
}
__device__ __forceinline__ void add_pair(float& x, float& y, float b)
{
    asm("{.reg .b64 v, c;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 c, {%2, %2};\n\t"
        "add.rn.f32x2 v, v, c;\n\tmov.b64 {%0, %1}, v;}"
        : "+f"(x), "+f"(y)
        : "f"(b));
}

// 16 values of a group (bf16 pairs) as two words of codes (pairs as above), and the group's scale and
// zero.  The lanes l ^ 1, l ^ 2 and l ^ 3 hold the group's other values (with 8 values in each of 8
// lanes half of the instructions were the group's own).
//
//   lo = min(0, x..), hi = max(0, x..), s = bf16((hi - lo) / 15) (0 below 2^-126),
//   z = rint(-lo / s), c = min(15, rint(x / s) + z); rint: to nearest, ties to even.
//
// The result is that of exact arithmetic, without a division:
//   x / s    x and s have 8-bit significands and |x / s| <= 15.06, so x / s is k + 1/2 exactly or more
//            than 2^-10 away from it.  x r, r about 1 / s, is within 2^-17 of x / s.  Adding 12288 in
//            one rounding with the product gives a multiple of 2^-10: a tie becomes a tie again, and
//            nothing else becomes one or crosses one; adding up to 2^23 + 2^22 then rounds to an
//            integer, ties to even, in the sum's last bits.
//   s        hi - lo is exact in float32 unless the two are 2^15 apart, and then (hi - lo) / 15 is not
//            near a point where the rounding to bf16 turns (15 times such a point has more
//            significant bits than hi).  The quotient is correctly rounded: the product with RN(1 / 15) and
//            one step with its exact remainder (Markstein 1990).
// Codes need no lower clamp: rint is odd, and -lo is among the values.
//
// A group with a value that is not finite, or 2^120 or more in size, becomes s = z = c = 0; returns
// whether this is one.
constexpr float kMostValue = 0x1p120f;
__device__ __forceinline__ bool quantize16(const uint32_t (&x)[8], uint32_t (&w)[2], float* scale,
                                           int* zero)
{
    uint32_t low = x[0], high = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        low = min_pair(low, x[i]);
        high = max_pair(high, x[i]);
    }
    // (largest, -smallest) of the lane's values and 0, then of the group's
    uint32_t ends = max_pair(max_pair(__byte_perm(high, low, 0x5410) ^ 0x80000000u,
                                      __byte_perm(high, low, 0x7632) ^ 0x80000000u), 0u);
    ends = max_pair(ends, __shfl_xor_sync(0xffffffffu, ends, 1));
    ends = max_pair(ends, __shfl_xor_sync(0xffffffffu, ends, 2));
    const float up = bf16_lo(ends), down = bf16_hi(ends), range = up + down;
    const bool beyond = !(up < kMostValue && down < kMostValue);
    constexpr float kFifteenth = 1.0f / 15.0f;
    const float q = range * kFifteenth;
    float s = fmaf(fmaf(-15.0f, q, range), kFifteenth, q);
    s = bf16_hi(bf16_pair(0.0f, s));
    const bool flat = !(s >= 0x1p-126f) || beyond;
    s = flat ? 0.0f : s;
    const float r = flat ? 0.0f : rcp_approx(s);
    constexpr float kFine = 12288.0f, kUnit = 12582912.0f;   // kUnit's last 16 bits are 0
    const int z = min(__float_as_int(fmaf(down, r, kFine) + (kUnit - kFine)) & 0xff, 15);
    const uint32_t zz = z * 0x00010001u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[i] = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float a = bf16_lo(x[4 * i + p]), b = bf16_hi(x[4 * i + p]);
            fma_pair(a, b, r, kFine);
            add_pair(a, b, kUnit - kFine);
            // both numbers' last 16 bits, plus z, at most 15
            const uint32_t v = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410);
            w[i] += __viaddmin_s16x2(v, zz, 0x000f000fu) << (4 * p);
        }
    }
    if (beyond) w[0] = w[1] = 0;      // 0 times such a value is no number
    *scale = s;
    *zero = beyond ? 0 : z;
    return beyond;
}

}  // namespace twk

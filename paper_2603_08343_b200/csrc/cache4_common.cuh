// The cache held in 4 bits: how a row is held and where its bytes lie.
//
// A row x of D channels (a key after its rotation, or a value) is held as
//     lo = bf16(min x),  step = bf16((max x - lo) / 15),  code_i = clamp(rint((x_i - lo) / step), 0, 15)
// and stands for lo + step * code_i.  All in fp32, each operation rounded on its own; the divisions are products with the rounded
// reciprocals.  lo and step are rounded before the codes are found: a channel is held to half a step (that the step may come out short, by up to 2^-8, moves the
// row's top by 15 / 256 of a step, which is less), or where lo is rounded up to that, 2^-8 of the least value's size.  A row whose offset is far above its spread
// loses its codes to the latter: one from 100.3 to 100.6 has lo = 100.5.  A step below 2^-100 (a row of equal channels) counts as 0, all codes 0.  A row
// with a NaN or an infinity (or one whose spread passes fp32) stands for NaN.
//
// A page of a key head is cut into tiles of 16 keys, each one contiguous piece of 16 D + 128 bytes that one asynchronous copy fetches:
// the codes of the keys, those of the values, then (step, lo) of the key and of the value, 8 bytes a key.  Inside a
// tile the codes lie so that the lanes of a warp find the operands of m16n8k16 products by wide loads without bank
// conflicts and without exchanging anything.  The unit is a half word: the codes of four neighbouring channels 32 g + 4 u .. + 3, the
// lowest channel in the lowest bits (g < D / 32, u < 8).
//   keys     row j: lane u / 2 of four finds its eight channels of every g side by side: words [u / 2][g], half u & 1
//   values   row j at place j' = (b2 b1 | b0 | b3 of j turned so that rows 0, 2, 4, 6 lie side by side): lane u of eight finds its
//            halves of all g side by side (D = 96: two of them, the third in a section of its own behind the 16 rows); D = 128: pieces
//            u ^ 4 for keys 4 .. 7 and 12 .. 15
#pragma once
#include "attn_kernels.cuh"

namespace wht {

constexpr int kTileKeys = 16;
constexpr float kLeastStep = 7.888609052210118e-31f;  // 2^-100

__host__ __device__ constexpr int tile4_bytes(int d) { return 16 * d + 128; }
__host__ __device__ constexpr int tile4_rows(int d) { return 16 * d; }  // offset of (step, lo)

// Byte offsets in a tile of the half word of row j, channels 32 g + 4 u .. + 3.
__device__ __forceinline__ int key4_at(int d, int j, int g, int u) { return j * (d >> 1) + (u >> 1) * (d >> 3) + 4 * g + 2 * (u & 1); }
__device__ __forceinline__ int value4_place(int j) { return ((j >> 1) & 3) | ((j & 1) << 2) | (j & 8); }
__device__ __forceinline__ int value4_at(int d, int j, int g, int u) {
    const int at = value4_place(j);
    if (d == 128) return 8 * d + at * 64 + ((u ^ (j & 4)) << 3) + 2 * g;
    if (d == 64 || g < 2) return 8 * d + at * 32 + u * 4 + 2 * g;
    return 8 * d + 16 * 32 + at * 16 + u * 2;
}

// lo and step of a row with these extremes; finite: whether the row stands for its values at all.
struct Hold4 {
    float lo, step, inverse;
    __device__ __forceinline__ Hold4(float least, float most, bool finite) {
        lo = __bfloat162float(__float2bfloat16_rn(least));
        const float spread = __fsub_rn(most, lo);
        step = __bfloat162float(__float2bfloat16_rn(__fmul_rn(spread, 1.0f / 15.0f)));
        if (!finite || !(fabsf(spread) < INFINITY)) {
            lo = __uint_as_float(0x7fc00000u);
            step = 0.0f;
        }
        if (!(step >= kLeastStep)) step = 0.0f;
        inverse = step > 0.0f ? __fdiv_rn(1.0f, step) : 0.0f;
    }
    __device__ __forceinline__ unsigned code(float x) const {
        // rounded to a whole number by the addition (2^23: the fraction has no bits left), which is cheaper than a conversion.  (A row that stands
        // for NaN has inverse 0 and lo NaN: fmaxf makes 0 of NaN.)
        const float y = fminf(fmaxf(__fmul_rn(__fsub_rn(x, lo), inverse), 0.0f), 15.0f);
        return __float_as_uint(__fadd_rn(y, 8388608.0f)) & 15u;
    }
    // step in the lower half, lo in the upper
    __device__ __forceinline__ unsigned word() const { return (__float_as_uint(step) >> 16) | (__float_as_uint(lo) & 0xffff0000u); }
};

// the whole number that code e of a word stands for, without a conversion
__device__ __forceinline__ float code4_value(unsigned word, int e) {
    return __uint_as_float(((word >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f;
}

__device__ __forceinline__ float step4_of(unsigned word) { return __uint_as_float(word << 16); }
__device__ __forceinline__ float lo4_of(unsigned word) { return __uint_as_float(word & 0xffff0000u); }

}  // namespace wht

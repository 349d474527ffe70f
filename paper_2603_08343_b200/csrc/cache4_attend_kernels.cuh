// Attention over the cache held in 4 bits, by warp-level matrix products on the codes themselves.
//
//     k_j = lo_j + step_j c_j,   v_j = lo'_j + step'_j c'_j      (codes c, c' whole numbers 0 .. 15)
//     score_j = scale (step_j (q . c_j) + lo_j sum(q))
//     o = sum_j p_j v_j / sum_j p_j = (sum_j (p_j step'_j) (c'_j - z_j) + sum_j p_j (lo'_j + z_j step'_j)) / sum_j p_j,   p_j = exp(score_j - m)
//
// in one pass over the keys.  (Inputs are read by ordinary loads: the kernel before may have written them while this one was resident.)
// The codes are never turned into values.  A half word of a key's codes masked with 0x000f or 0x00f0 IS an fp16 number, c 2^-24 or 16 c 2^-24
// (a subnormal one; the tensor core takes these as they are, but aligns a product by its operands' exponents, so that sums keep about
// 20 bits), so that eight codes take four masks and one shift, exactly, and the powers of two go into the
// queries and the result.  z_j keeps the two sums small: with z = 0 for all keys they are large, of opposite signs, and the result is their small
// difference.  For bf16 results z is 0 for the keys of even places and 15 for the others, whose codes are turned over as they are loaded (15 - c) and whose
// steps change sign, which costs next to nothing; for fp32 ones, whose values' codes become ordinary numbers by one exact subtraction a pair, z
// is 8 and 7 (64 x 16384 in bf16 would then take 192 us instead of 164).
// The tensor core's accumulation truncates towards zero, by up to 2^-23 of a sum in each addition, so that the loss grows with their number, and equal
// weights that are added one by one round alike: after kFold4 steps all sums are added to others in shared memory, with rounding, and begin
// anew.  (With z = 0 and one accumulation a run, 131072 keys of even weight were off by 0.38 of the result's norm and 1048576 by 15 times the norm; now by
// 0.0004 and 0.0007 beside the rounding to bf16.)
// Queries enter as fp16 after a shift of each row by a power of two (bf16 ones keep all their bits but what lies below 2^-33 of the row's
// maximum; fp32 ones are two terms, 22 bits of it), and the weights p step' as fp16 times a power of two per row that keeps them in range: one
// term of 11 bits where the output is rounded to 8, two where it is fp32.
//
// What bounds it: memory, 2 (D / 2 + 4) bytes a key and key head, and instructions next to it.  At 23 B a clock and SM a tile of 16 keys of 128 channels has
// 378 clocks of an SM's quarter; it takes 239 instructions for up to 8 rows, about 100 of which mask, select and shift, two clocks each, and 208 for up to 4.
// So products are taken transposed, S^T = C Q^T and O^T = C'^T P^T: codes of 16 keys (channels) fill the 16-row operand and the rows sit on the 8-column one, so
// that 8 rows waste nothing, a key's step and least value are wanted by the four lanes that hold its scores, and P^T changes from accumulator to operand
// layout by one 8x8 transposition.  Up to four rows take every other column, half of the softmax's instructions (200 x 1000 keys 56 -> 51 us, 1 x 4096 8.7 ->
// 8.2).  64 sequences of up to 16384 keys of 8 key heads of 128, 32 heads: 157-159 us, 5.4 TB/s (DRAM 65 % busy, issue slots 53 %, ALU
// 58 %; with the rows on the 16-row operand, half of it empty, 364 instructions a tile and 242 us).  Two tiles a step, so that their latencies overlap (one:
// 165-167).  200 x 1000 keys of 16 heads of 64: 52.6 us, 3.3 TB/s: a tile has half the bytes, but the softmax of as many scores.
//
// The division of work goes by the lengths themselves, which are on the device: the tiles of all units (sequence, key head, row tile)
// are counted one after the other, and each warp (a block of its own) takes an equal run of them, whatever units it touches.  A unit that lies in one
// run is finished there; the parts of the others are joined by a second kernel, in the order of the keys.
#pragma once
#include <cuda_fp16.h>

#include "cache4_common.cuh"

namespace wht {

struct Attn4Params {
    AttnParams a;            // queries, output, tables, lengths, sizes; part_ml, part_o: [2 * warps][part_rows]
    const unsigned char* cache;
    int warps;               // runs
    int least;               // grains of a run, at least
    int part_rows;           // rows of a part: those that a unit can have
    int grain;               // log2 of a grain's tiles: work is counted in grains, in 32 bits
    float* lse;              // [T * Hq] log2 of a row's softmax sum, or NULL
    float* scores;           // [B * Hkv][tile][part_rows][16] log2 scores, or NULL: they are taken anew for the received weight
    const float* weights;    // [B x Hkv x table_width * page]: received so far
    float* weights_out;
};

// NR: 8-row tiles of a unit.
template <typename T, int D, int NR>
struct Attn4Geo {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NG = D / 32;
    static constexpr int ROWS = 8 * NR;
    static constexpr int TERMS = F32 ? 2 : 1;                   // of queries and of weights
    static constexpr int TILE = tile4_bytes(D);
    static constexpr int U = NR == 1 ? 2 : 1;                   // tiles of a step
    static constexpr int STAGES = U == 2 ? 2 : 4;               // steps of the ring
    static constexpr bool Q_SHARED = NR * TERMS > 2;            // query operands in shared memory
    static constexpr int Q_BYTES = Q_SHARED ? NR * TERMS * NG * 512 : 0;
    static constexpr int OFF_Q = STAGES * U * TILE;
    static constexpr int OFF_FOLD = OFF_Q + Q_BYTES;            // a lane's sums of the steps before: [accumulator, then l and r of each row][lane]; then the rows' m
    static constexpr int FOLD_O = NR * (D / 4), FOLD = FOLD_O + 4 * NR;
    static constexpr int OFF_BARS = OFF_FOLD + FOLD * 128 + ROWS * 4;
    static constexpr int BYTES = OFF_BARS + STAGES * 8;
    static constexpr int BLOCKS = NR * TERMS > 2 ? 8 : NR * TERMS > 1 ? 12 : 16;  // on an SM
};

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t minus_half2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float half_lo(uint32_t w) { return __half2float(__ushort_as_half(static_cast<unsigned short>(w))); }
__device__ __forceinline__ float half_hi(uint32_t w) { return __half2float(__ushort_as_half(static_cast<unsigned short>(w >> 16))); }
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((127 + e) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int exponent_of(float x) { return ((__float_as_int(x) >> 23) & 255) - 127; }
__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(kFullMask, x, 1));
    return fmaxf(x, __shfl_xor_sync(kFullMask, x, 2));
}
// over the eight lanes that hold one row's accumulators
__device__ __forceinline__ float column_max(float x) {
#pragma unroll
    for (int i = 4; i < 32; i <<= 1) x = fmaxf(x, __shfl_xor_sync(kFullMask, x, i));
    return x;
}
__device__ __forceinline__ float column_sum(float x) {
#pragma unroll
    for (int i = 4; i < 32; i <<= 1) x += __shfl_xor_sync(kFullMask, x, i);
    return x;
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(kFullMask, x, 1);
    return x + __shfl_xor_sync(kFullMask, x, 2);
}

// A row of queries: this lane's channels 32 g + 8 c4 .. + 7 as operands of the steps 2 g and 2 g + 1; [g][step][0]: contraction indices
// 2 c4, + 1, [1]: + 8.  They stand for the channels whose codes lie there (the odd ones with codes times 16, hence queries / 16).
template <typename T, int NG>
struct Query4 {
    uint32_t lead[NG][2][2], rest[NG][2][2];
    float factor, sum;       // score = step * (product) * factor + lo * sum, in log2
    float lead0, rest0;      // fp32: what the products begin with, so that they are those of code - 8
    __device__ __forceinline__ void load(const T* src, bool there, float scale_log2) {
        const int c4 = threadIdx.x & 3;
        float v[NG][8];
        float top = 0.0f, total = 0.0f;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            if (there) {
                load8_written(src + g * 32 + c4 * 8, v[g]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[g][i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = fmaxf(top, fabsf(v[g][i]));
                total += v[g][i];
            }
        }
        top = quad_max(top);
        total = quad_sum(total);
        const int e = top > 0.0f ? max(exponent_of(top) - 13, -113) : 0;  // the largest becomes 2^13 and up to 2^14
        const float shift = power_of_two(-e);
        factor = scale_log2 * power_of_two(e) * 16777216.0f;
        sum = scale_log2 * total;
        float leads = 0.0f, rests = 0.0f;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float by = i & 1 ? 0.0625f : 1.0f;
                float x = v[g][i] * shift, y = v[g][4 + i] * shift;
                if constexpr (std::is_same<T, float>::value) {
                    const float xl = rintf(x * 0.125f) * 8.0f, yl = rintf(y * 0.125f) * 8.0f;
                    x -= xl;
                    y -= yl;
                    lead[g][i >> 1][i & 1] = pack_half2(xl * by, yl * by);
                    const uint32_t w = pack_half2(x * by, y * by);
                    rest[g][i >> 1][i & 1] = w;
                    leads += xl + yl;
                    rests += x + y;
                } else {
                    lead[g][i >> 1][i & 1] = pack_half2(x * by, y * by);
                    rest[g][i >> 1][i & 1] = 0u;
                }
            }
        lead0 = quad_sum(leads) * -0x1p-21f;
        rest0 = quad_sum(rests) * -0x1p-21f;
    }
};

// The rows of a unit as the products take them: in column r4 of tile n row 8 n + r4, and what belongs to the rows of columns 2 c4 + e, e < E, whose accumulators a lane
// holds.  E = 1: up to four rows, in the even columns alone, so that a lane has the softmax of one row for each key, not of two.
template <typename T, int D, int NR, int E>
struct Rows4 {
    using Geo = Attn4Geo<T, D, NR>;
    static constexpr int TERMS = Geo::TERMS;
    uint32_t q[Geo::Q_SHARED ? 1 : NR][TERMS][Geo::NG][2][2];
    float factor[NR][E], sum[NR][E];
    float first[NR][TERMS][E];                                       // (fp32) what the products of each term begin with
    __device__ __forceinline__ void load(const AttnParams& p, int64_t token0, int head, int row0, int rows, unsigned char* smem) {
        const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int row = row0 + (E == 1 ? r4 >> 1 : n * 8 + r4), tok = row / p.group;
            const T* src = static_cast<const T*>(p.q) + (token0 + tok) * p.q_st +
                           (static_cast<int64_t>(head) * p.group + (row - tok * p.group)) * p.q_sh;
            Query4<T, Geo::NG> x;
            x.load(src, row < rows && (E == 2 || !(r4 & 1)), p.scale_log2);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int from = (2 * c4 + e) * 4;
                factor[n][e] = __shfl_sync(kFullMask, x.factor, from);
                sum[n][e] = __shfl_sync(kFullMask, x.sum, from);
                if constexpr (Geo::F32) {
                    first[n][0][e] = __shfl_sync(kFullMask, x.lead0, from);
                    first[n][1][e] = __shfl_sync(kFullMask, x.rest0, from);
                }
            }
#pragma unroll
            for (int g = 0; g < Geo::NG; ++g)
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    auto& f = t ? x.rest[g] : x.lead[g];
                    if constexpr (Geo::Q_SHARED) {
                        *reinterpret_cast<uint4*>(smem + ((n * TERMS + t) * Geo::NG + g) * 512 + lane * 16) =
                            make_uint4(f[0][0], f[0][1], f[1][0], f[1][1]);
                    } else {
#pragma unroll
                        for (int s = 0; s < 2; ++s)
#pragma unroll
                            for (int i = 0; i < 2; ++i) q[n][t][g][s][i] = f[s][i];
                    }
                }
        }
    }
    __device__ __forceinline__ void get(int n, int t, int g, const unsigned char* smem, uint32_t (&f)[2][2]) const {
        if constexpr (Geo::Q_SHARED) {
            const uint4 w = *reinterpret_cast<const uint4*>(smem + ((n * TERMS + t) * Geo::NG + g) * 512 + (threadIdx.x & 31) * 16);
            f[0][0] = w.x; f[0][1] = w.y; f[1][0] = w.z; f[1][1] = w.w;
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) f[s][i] = q[n][t][g][s][i];
        }
    }
};

// (step, lo) of the keys r4 and r4 + 8 of a tile and of their values.
struct Params4 {
    uint2 lower, upper;
    __device__ __forceinline__ void load(const unsigned char* rows) {
        const int r4 = (threadIdx.x & 31) >> 2;
        lower = *reinterpret_cast<const uint2*>(rows + r4 * 8);
        upper = *reinterpret_cast<const uint2*>(rows + 64 + r4 * 8);
    }
    __device__ __forceinline__ uint32_t key(int k) const { return k ? upper.x : lower.x; }
    __device__ __forceinline__ uint32_t value(int k) const { return k ? upper.y : lower.y; }
};

// A key's base: its least value; for fp32 what code 8 stands for, since lo and the sum of codes, all positive, are several times what they weigh
// together in the end.
template <typename T>
__device__ __forceinline__ float base4_of(unsigned word) {
    return std::is_same<T, float>::value ? fmaf(8.0f, step4_of(word), lo4_of(word)) : lo4_of(word);
}

// What the code z of a value stands for.
__device__ __forceinline__ float value4_of(unsigned word, float z) { return fmaf(z, step4_of(word), lo4_of(word)); }
// A step with the sign that `turn` (0 or the sign's bit) gives it: one multiply-add.
__device__ __forceinline__ float turned_step4_of(unsigned word, unsigned turn) { return __uint_as_float(word * 65536u + turn); }

// S^T = C Q^T of a tile: s[n][2 k + e] = key r4 + 8 k, row 8 n + 2 c4 + e.
// fp32 rows: the tensor core's accumulation truncates to about 24 bits of the largest product.  The first term of a query is therefore a
// whole number of eighths of 2^-10 of the row's range: products with codes and sums of 128 of them take 22 bits, so nothing is lost.
template <typename T, int D, int NR, int E>
__device__ __forceinline__ void scores4(const Rows4<T, D, NR, E>& rows, const unsigned char* tile, const unsigned char* q_smem,
                                        float (&s)[NR][4]) {
    constexpr int NG = D / 32, TERMS = Rows4<T, D, NR, E>::TERMS;
    const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
    uint32_t w[2][NG];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned char* at = tile + (r4 + 8 * k) * (D / 2) + c4 * (D / 8);
        if constexpr (NG == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(at);
            w[k][0] = x.x; w[k][1] = x.y; w[k][2] = x.z; w[k][3] = x.w;
        } else if constexpr (NG == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            w[k][0] = x.x; w[k][1] = x.y;
        } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) w[k][g] = reinterpret_cast<const uint32_t*>(at)[g];
        }
    }
    float acc[TERMS][NR][4];
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][n][i] = TERMS == 2 && (i & 1) < E ? rows.first[n][t][E == 2 ? i & 1 : 0] : 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint32_t a[2][4];
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t x = st ? w[k][g] >> 8 : w[k][g];
                a[st][k] = x & 0x000f000fu;
                a[st][2 + k] = x & 0x00f000f0u;
            }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
                uint32_t b[2][2];
                rows.get(n, t, g, q_smem, b);
#pragma unroll
                for (int st = 0; st < 2; ++st) mma_f16_16816(acc[t][n], a[st], b[st][0], b[st][1]);
            }
    }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = TERMS == 2 ? acc[0][n][i] + acc[TERMS - 1][n][i] : acc[0][n][i];
}

// O^T += (C' - z)^T P^T of a tile; b[n][t]: the weights times the values' steps as operands (row r4; keys 2 c4, + 1 and 8 + 2 c4, + 1; bf16: those of odd
// keys with the other sign).  o[n][2 g + i][2 j + e]: channel 32 g + 4 r4 + 2 i + j, row 8 n + 2 c4 + e.
template <typename T, int D, int NR>
__device__ __forceinline__ void add_values4(const unsigned char* tile, const uint32_t (&b)[NR][Attn4Geo<T, D, NR>::TERMS][2], float (&o)[NR][D / 16][4]) {
    constexpr int NG = D / 32;
    constexpr bool F32 = std::is_same<T, float>::value;
    const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
    // this lane's codes of the keys 2 c4, 2 c4 + 1, 8 + 2 c4, 9 + 2 c4, halves u = r4; two neighbouring keys side by side.  bf16: those of odd keys turned over
    const unsigned char* vt = tile + 8 * D;
    uint32_t pair[NG][2];
    if constexpr (NG == 4) {
        uint2 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = *reinterpret_cast<const uint2*>(vt + (c4 + 4 * i) * 64 + ((r4 ^ ((c4 & 2) << 1)) << 3));
            if (!F32 && (i & 1)) v[i] = make_uint2(~v[i].x, ~v[i].y);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            pair[0][i] = __byte_perm(v[2 * i].x, v[2 * i + 1].x, 0x5410);
            pair[1][i] = __byte_perm(v[2 * i].x, v[2 * i + 1].x, 0x7632);
            pair[2][i] = __byte_perm(v[2 * i].y, v[2 * i + 1].y, 0x5410);
            pair[3][i] = __byte_perm(v[2 * i].y, v[2 * i + 1].y, 0x7632);
        }
    } else {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = *reinterpret_cast<const uint32_t*>(vt + (c4 + 4 * i) * 32 + r4 * 4);
            if (!F32 && (i & 1)) v[i] = ~v[i];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            pair[0][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x5410);
            pair[1][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x7632);
        }
        if constexpr (NG == 3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = *reinterpret_cast<const unsigned short*>(vt + 512 + (c4 + 4 * i) * 16 + r4 * 2);
                if (!F32 && (i & 1)) v[i] = ~v[i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) pair[2][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x5410);
        }
    }
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            uint32_t a[4];                                           // channels j = 0, 1 of keys 0 .. 7, then of 8 .. 15
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t x = st ? pair[g][k] >> 8 : pair[g][k];
                if constexpr (F32) {                                 // 1024 + c less 1024 + z; the lower half is the even key's
                    a[2 * k] = minus_half2((x & 0x000f000fu) | 0x64006400u, 0x64076408u);
                    a[2 * k + 1] = minus_half2((x & 0x00f000f0u) | 0x64006400u, 0x64706480u);
                } else {
                    a[2 * k] = x & 0x000f000fu;
                    a[2 * k + 1] = x & 0x00f000f0u;
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                if constexpr (F32) {
                    // (the tensor core's accumulation truncates: one tile at a time, added up with rounding)
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    mma_f16_16816(sum, a, b[n][1][0], b[n][1][1]);
                    mma_f16_16816(sum, a, b[n][0][0], b[n][0][1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][2 * g + st][e] += sum[e];
                } else {
                    mma_f16_16816(o[n][2 * g + st], a, b[n][0][0], b[n][0][1]);
                }
            }
        }
}

// The tiles of one unit in one run.
struct Segment4 {
    int64_t token0;          // first token of the sequence
    int count, keys;         // its tokens in this call, its keys
    const int32_t* table;    // its pages
    int head, row0;          // key head, first row of the unit: row r is token r / group, query head head * group + r % group
    int tile0, tile1;        // of the unit's tiles
    int64_t slot;            // where the part goes, or -1: the unit is finished here
    float* scores;           // where the scores of the sequence and key head go, or NULL
};

// A warp's ring of tiles: how many have been asked for and taken since the start, over all its segments.
struct Ring4 {
    unsigned char* base;
    uint64_t* full;
    unsigned taken;
};

// The tile numbers (in the cache) of 32 of a segment's tiles, one a lane: tiles first + lane < end.
__device__ __forceinline__ int tiles4_of(const AttnParams& p, const int32_t* table, int head, int first, int end) {
    const int t = first + static_cast<int>(threadIdx.x & 31), shift = p.page_shift - 4;
    if (t >= end) return 0;
    int pg = table[t >> shift];
    if (pg < 0 || pg >= p.num_pages) {
        attn_report(kAttnErrIndex);
        pg = 0;
    }
    return ((pg * p.hkv + head) << shift) + (t & ((1 << shift) - 1));
}

// How far a weight times a value's step may go before the row's reference moves, and a weight and that times what the value's z stands for.
constexpr float kMostProduct4 = 16384.0f, kMostWeight4 = 0x1p100f;
// What z stands for counts in a reference only where it is larger than this (and then costs two logarithms a key).
constexpr float kLargeBase4 = 256.0f;
// Steps of which the tensor core holds the sum: 1024 keys (512 in units of 16 rows).
constexpr int kFold4 = 32;

template <typename T, int D, int NR, int E>
__device__ __forceinline__ void attn4_segment(const Attn4Params& p, const Segment4& u, Ring4& ring, unsigned char* smem) {
    using Geo = Attn4Geo<T, D, NR>;
    constexpr bool F32 = Geo::F32;
    constexpr int NG = Geo::NG, STAGES = Geo::STAGES, U = Geo::U, TERMS = Geo::TERMS;
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
    // z of this lane's keys (with the sign of their steps); bf16: odd ones take their steps, and with them the products, with the other sign
    const float zero_code = F32 ? (r4 & 1 ? 7.0f : 8.0f) : r4 & 1 ? -15.0f : 0.0f;
    const unsigned turn = !F32 && (r4 & 1) ? 0x80000000u : 0u;
    const int rows = u.count * a.group;
    // the unit's last row sees the most keys, its first row the fewest
    const int last_row = min(rows, u.row0 + Geo::ROWS) - 1;
    const int first_limit = u.keys - u.count + 1;                    // keys that the sequence's first token sees
    const int end = static_cast<int>(min(static_cast<int64_t>(u.tile1) * kTileKeys, static_cast<int64_t>(first_limit + last_row / a.group)));
    const int least_limit = min(end, first_limit + u.row0 / a.group);
    const int tiles = max(0, (end - u.tile0 * kTileKeys + kTileKeys - 1) / kTileKeys);
    const int steps = (tiles + U - 1) / U;

    int now = tiles4_of(a, u.table, u.head, u.tile0, u.tile0 + tiles);
    int next = tiles > 32 ? tiles4_of(a, u.table, u.head, u.tile0 + 32, u.tile0 + tiles) : 0;
    auto ask = [&](unsigned stage, int j, const int (&tile)[U]) {    // lane 0: step j
        const int there = min(U, tiles - j * U);
        mbar_expect_tx(ring.full + stage, there * Geo::TILE);
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (i < there)
                bulk_load(ring.base + (stage * U + i) * Geo::TILE, p.cache + static_cast<int64_t>(tile[i]) * Geo::TILE, Geo::TILE, ring.full + stage);
    };
#pragma unroll
    for (int j = 0; j < STAGES; ++j) {
        int tile[U];
#pragma unroll
        for (int i = 0; i < U; ++i) tile[i] = __shfl_sync(kFullMask, now, j * U + i);
        if (lane == 0 && j < steps) ask((ring.taken + j) % STAGES, j, tile);
    }
    unsigned char* q_smem = smem + Geo::OFF_Q;
    Rows4<T, D, NR, E> rw;
    rw.load(a, u.token0, u.head, u.row0, rows, q_smem);
    if constexpr (Geo::Q_SHARED) __syncwarp();

    // m: the reference of a row's weights exp2(score - m), which it shares with its products (weight times step): the largest product so far is 2^6 or
    // a little more, at most 2^14, so that products are fp16 numbers of full precision, whatever the values' size.
    float m[NR][E], l[NR][E], r[NR][E];
    float o[NR][D / 16][4];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            m[n][e] = -INFINITY;
            l[n][e] = r[n][e] = 0.0f;
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[n][d][0] = o[n][d][1] = o[n][d][2] = o[n][d][3] = 0.0f;
    }
    // the row of this lane's column 2 c4 + e
    auto column_row = [&](int n, int e) { return E == 1 ? c4 : n * 8 + 2 * c4 + e; };
    // keys that it sees of these (rows that are not there see zeros); a step's second tile may lie behind the end
    auto limit = [&](int n, int e) {
        const int row = u.row0 + column_row(n, e);
        return row < rows ? min(end, first_limit + row / a.group) : end;
    };

    unsigned stage = ring.taken % STAGES, parity = (ring.taken / STAGES) & 1u;
    ring.taken += steps;
    auto step = [&](int j, auto masked) {
        constexpr bool mask = masked.value;                          // rows may see less than all of these keys
        mbar_wait_bounded(ring.full + stage, parity);
        const unsigned char* tile = ring.base + stage * U * Geo::TILE;
        const int base = (u.tile0 + j * U) * kTileKeys;

        float s[U][NR][4];
        Params4 w[U];
#pragma unroll
        for (int t = 0; t < U; ++t) {
            scores4<T, D, NR, E>(rw, tile + t * Geo::TILE, q_smem, s[t]);
            w[t].load(tile + t * Geo::TILE + tile4_rows(D));
        }
        if (NR == 1 && u.scores != nullptr) {
#pragma unroll
            for (int t = 0; t < U; ++t)
#pragma unroll
                for (int i = 0; i < 2 * E; ++i) {
                    const int k = i / E, e = i % E, at = u.tile0 + j * U + t, row = column_row(0, e);
                    if (row < rows && j * U + t < tiles)
                        u.scores[(static_cast<int64_t>(at) * p.part_rows + row) * kTileKeys + 8 * k + r4] =
                            fmaf(step4_of(w[t].key(k)) * s[t][0][2 * k + e], rw.factor[0][e], base4_of<T>(w[t].key(k)) * rw.sum[0][e]);
                }
        }
        auto hidden = [&](int t, int n, int i) { return base + t * kTileKeys + 8 * (i >> 1) + r4 >= limit(n, i & 1); };
        // One score against the row's reference: its weight, and that times its value's step.
        auto weigh = [&](int t, int n, int i, float& x, float& y) {
            const int k = i >> 1, e = i & 1;
            x = exp2_fast(fmaf(step4_of(w[t].key(k)) * s[t][n][i], rw.factor[n][e], fmaf(base4_of<T>(w[t].key(k)), rw.sum[n][e], -m[n][e])));
            y = x * turned_step4_of(w[t].value(k), turn);
        };
        // What z stands for in a value of this lane.
        auto value_base = [&](int t, int k) { return fmaf(zero_code, turned_step4_of(w[t].value(k), turn), lo4_of(w[t].value(k))); };
        // This lane's sums of a row: weights, weights times base values, products; and the products as operands, before their transposition.
        float sx[NR][E], sr[NR][E], sy[NR][E];
        uint32_t b[U][NR][TERMS][2];
        auto add_up = [&] {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int e = 0; e < E; ++e) sx[n][e] = sr[n][e] = sy[n][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < U; ++t)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float base_value = value_base(t, k);
                        float y[2] = {0.0f, 0.0f};
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float x;
                            weigh(t, n, 2 * k + e, x, y[e]);
                            bool seen = true;
                            if constexpr (mask) seen = !hidden(t, n, 2 * k + e);
                            if (!seen) y[e] = x = 0.0f;
                            sx[n][e] += x;
                            sy[n][e] += y[e];
                            sr[n][e] = fmaf(x, seen ? base_value : 0.0f, sr[n][e]);
                        }
                        b[t][n][0][k] = pack_half2(y[0], y[1]);
                        if constexpr (F32) b[t][n][1][k] = pack_half2(y[0] - half_lo(b[t][n][0][k]), y[1] - half_hi(b[t][n][0][k]));
                    }
            }
        };
        add_up();
        float all_x = 0.0f, all_y = 0.0f;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                all_x += sx[n][e] + fabsf(sr[n][e]);
                all_y += sy[n][e];
            }
        }
        // (NaN fails; the sum over a lane's rows passes whenever one of its rows' does; a lane's products have one sign)
        if (!__all_sync(kFullMask, all_x <= kMostWeight4 && fabsf(all_y) <= kMostProduct4)) {
            bool far = false;
#pragma unroll
            for (int t = 0; t < U; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) far |= fabsf(value_base(t, k)) > kLargeBase4;
            far = __any_sync(kFullMask, far);
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    // (a row moves its reference by its own scores alone: its result does not depend on the rows beside it)
                    int moves = !(sx[n][e] + fabsf(sr[n][e]) <= kMostWeight4 && fabsf(sy[n][e]) <= kMostProduct4);
#pragma unroll
                    for (int i = 4; i < 32; i <<= 1) moves |= __shfl_xor_sync(kFullMask, moves, i);
                    if (!__any_sync(kFullMask, moves)) continue;
                    float top = -INFINITY, heavy = -INFINITY;        // the largest score, and score plus log2 of the step
#pragma unroll
                    for (int t = 0; t < U; ++t)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if (mask && hidden(t, n, 2 * k + e)) continue;
                            const float score = fmaf(step4_of(w[t].key(k)) * s[t][n][2 * k + e], rw.factor[n][e], base4_of<T>(w[t].key(k)) * rw.sum[n][e]);
                            top = fmaxf(top, score);
                            heavy = fmaxf(heavy, score + __log2f(step4_of(w[t].value(k))));
                        }
                    top = column_max(top);
                    heavy = column_max(heavy);
                    float wide = top;                                // and score plus log2 of what z stands for, if that is large anywhere
                    if (far) {
#pragma unroll
                        for (int t = 0; t < U; ++t)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                if (mask && hidden(t, n, 2 * k + e)) continue;
                                const float score = fmaf(step4_of(w[t].key(k)) * s[t][n][2 * k + e], rw.factor[n][e], base4_of<T>(w[t].key(k)) * rw.sum[n][e]);
                                wide = fmaxf(wide, score + __log2f(fabsf(value_base(t, k))));
                            }
                        wide = column_max(wide);
                    }
                    // (without a step above 0 there are no products)
                    float to = fmaxf(heavy > -INFINITY ? heavy - 6.0f : top, wide - 90.0f);
                    to = moves ? fmaxf(to, m[n][e]) : m[n][e];
                    const float f = to > m[n][e] ? exp2_fast(m[n][e] - to) : 1.0f;
                    m[n][e] = to;
                    l[n][e] *= f;
                    r[n][e] *= f;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[n][d][e] *= f;
                        o[n][d][2 + e] *= f;
                    }
                }
            add_up();
        }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                l[n][e] += sx[n][e];
                r[n][e] += sr[n][e];
            }
#pragma unroll
        for (int t = 0; t < U; ++t) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int i = 0; i < TERMS; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) b[t][n][i][k] = transpose_8x8(b[t][n][i][k]);
            add_values4<T, D, NR>(tile + t * Geo::TILE, b[t], o);
        }
        __syncwarp();                                                // every lane has read the slot
        const int ahead = (j + STAGES) * U;                          // (a multiple of U, which divides 32)
        if (ahead < tiles) {
            if ((ahead & 31) == 0) {
                now = next;
                next = ahead + 32 < tiles ? tiles4_of(a, u.table, u.head, u.tile0 + ahead + 32, u.tile0 + tiles) : 0;
            }
            int to[U];
#pragma unroll
            for (int i = 0; i < U; ++i) to[i] = __shfl_sync(kFullMask, now, (ahead + i) & 31);
            if (lane == 0) ask(stage, j + STAGES, to);
        }
        if (++stage == STAGES) {
            stage = 0;
            parity ^= 1u;
        }
    };
    // steps whose keys all rows see, then the others
    const int open = least_limit > u.tile0 * kTileKeys ? min(steps, (least_limit - u.tile0 * kTileKeys) / (U * kTileKeys)) : 0;
    float *fold = reinterpret_cast<float*>(smem + Geo::OFF_FOLD) + lane, *fold_m = reinterpret_cast<float*>(smem + Geo::OFF_FOLD) + Geo::FOLD * 32;
    for (int j = 0;;) {
        const int stop = min(steps, j + kFold4), begin = j;
        for (; j < min(stop, open); ++j) step(j, std::false_type{});
        for (; j < stop; ++j) step(j, std::true_type{});
        // the sums of the steps before, in the present reference
        if (begin > 0) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float* before = fold + (Geo::FOLD_O + 4 * n + 2 * e) * 32;
                    const float was = fold_m[n * 8 + 2 * c4 + e], f = m[n][e] > was ? exp2_fast(was - m[n][e]) : 1.0f;
                    l[n][e] = fmaf(before[0], f, l[n][e]);
                    r[n][e] = fmaf(before[32], f, r[n][e]);
#pragma unroll
                    for (int d = 0; d < D / 16; ++d)
#pragma unroll
                        for (int i = e; i < 4; i += 2) o[n][d][i] = fmaf(fold[((n * (D / 16) + d) * 4 + i) * 32], f, o[n][d][i]);
                }
        }
        if (j >= steps) break;
        __syncwarp();                                                // (all have read the rows' references)
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float* to = fold + (Geo::FOLD_O + 4 * n + 2 * e) * 32;
                to[0] = l[n][e];
                to[32] = r[n][e];
                if (r4 == 0) fold_m[n * 8 + 2 * c4 + e] = m[n][e];
                l[n][e] = r[n][e] = 0.0f;
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int i = e; i < 4; i += 2) {
                        fold[((n * (D / 16) + d) * 4 + i) * 32] = o[n][d][i];
                        o[n][d][i] = 0.0f;
                    }
            }
    }

    // the results, four channels of a row at a time
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int local = column_row(n, e), row = u.row0 + local, tok = row / a.group;
            const float ll = column_sum(l[n][e]), rr = column_sum(r[n][e]);
            if (row >= rows) continue;
            const int64_t at = (u.token0 + tok) * a.hq + static_cast<int64_t>(u.head) * a.group + (row - tok * a.group);
            const float inv = u.slot >= 0 ? 1.0f : ll > 0.0f ? 1.0f / ll : 0.0f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                constexpr float even = F32 ? 1.0f : 0x1p24f, odd = even * 0.0625f;
                const float4 v = make_float4((o[n][2 * g][e] * even + rr) * inv, (o[n][2 * g][2 + e] * odd + rr) * inv,
                                             (o[n][2 * g + 1][e] * even + rr) * inv, (o[n][2 * g + 1][2 + e] * odd + rr) * inv);
                const int ch = g * 32 + r4 * 4;
                if (F32 || u.slot >= 0)
                    *reinterpret_cast<float4*>(u.slot >= 0 ? a.part_o + (u.slot * p.part_rows + local) * D + ch : static_cast<float*>(a.out) + at * D + ch) = v;
                else
                    *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * D + ch) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
            }
            if (r4 != 0) continue;
            if (u.slot >= 0) a.part_ml[u.slot * p.part_rows + local] = make_float2(m[n][e], ll);
            else if (p.lse) p.lse[at] = ll > 0.0f || ll != ll ? m[n][e] + log2f(ll) : INFINITY;
        }
}

// ---- the division of the work

// Grains of sequence b: units (key heads times row tiles) times grains of its keys, one at least where it has tokens.
struct Share4 {
    int64_t token0;
    int count, keys;
    unsigned row_tiles, grains;
    __device__ __forceinline__ Share4(const AttnParams& p, int b, int unit_rows, int grain) : token0(0), count(0), keys(0), row_tiles(0), grains(1) {
        if (b >= p.B) return;
        attn_tokens(p, b, token0, count);
        keys = attn_length(p, b);
        row_tiles = (static_cast<unsigned>(count) * p.group + unit_rows - 1) / unit_rows;
        const unsigned keys_of_grain = static_cast<unsigned>(kTileKeys) << grain;
        grains = max(1u, (static_cast<unsigned>(keys) + keys_of_grain - 1) / keys_of_grain);
    }
    __device__ __forceinline__ unsigned cost(int hkv) const { return hkv * row_tiles * grains; }
};

// Where a run (or a unit) lies among all grains: the sequence that holds grain `at`, the grains before that sequence, and all of them.
struct Place4 {
    int b;
    unsigned before, total;
};
__device__ __forceinline__ unsigned run4_grains(unsigned total, int warps, int least) {
    return max((total + warps - 1) / warps, static_cast<unsigned>(least));
}
__device__ __forceinline__ unsigned upto_lane(unsigned x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 1; i < 32; i <<= 1) {
        const unsigned y = __shfl_up_sync(kFullMask, x, i);
        if (lane >= i) x += y;
    }
    return x;
}
// The place of run `run_no`; b = B where it has nothing to do.
__device__ __forceinline__ Place4 find_run4(const Attn4Params& p, int unit_rows, unsigned run_no, unsigned& run) {
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31;
    unsigned upto = upto_lane(Share4(a, lane, unit_rows, p.grain).cost(a.hkv));
    unsigned total = __shfl_sync(kFullMask, upto, 31);
    if (a.B > 32) {
        unsigned more = 0;
#pragma unroll 4
        for (int b = 32 + lane; b < a.B; b += 32) more += Share4(a, b, unit_rows, p.grain).cost(a.hkv);
        total += __reduce_add_sync(kFullMask, more);
    }
    run = run4_grains(total, p.warps, p.least);
    Place4 at{0, 0, total};
    const unsigned f = run * run_no;                   // (run * warps < 2^32: the host sees to it)
    if (f >= total) return Place4{a.B, total, total};
    for (;;) {
        const unsigned past = __ballot_sync(kFullMask, at.before + upto > f);
        if (past) {
            const int i = __ffs(past) - 1;
            const unsigned skipped = __shfl_sync(kFullMask, upto, max(i - 1, 0));
            at.b += i;
            at.before += i > 0 ? skipped : 0;
            return at;
        }
        at.before += __shfl_sync(kFullMask, upto, 31);
        at.b += 32;
        if (at.b >= a.B) return at;                    // (lengths that changed meanwhile)
        upto = upto_lane(Share4(a, at.b + lane, unit_rows, p.grain).cost(a.hkv));
    }
}

template <typename T, int D, int NR, int E>
__global__ void __launch_bounds__(32, (Attn4Geo<T, D, NR>::BLOCKS))
attn4_kernel(const Attn4Params p) {
    using Geo = Attn4Geo<T, D, NR>;
    extern __shared__ __align__(128) unsigned char smem4[];
    const AttnParams& a = p.a;
    const int lane = threadIdx.x;
    Ring4 ring{smem4, reinterpret_cast<uint64_t*>(smem4 + Geo::OFF_BARS), 0};
    if (lane == 0) {
        for (int s = 0; s < Geo::STAGES; ++s) mbar_init(ring.full + s, 1);
        fence_mbar_init();
    }
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();                          // (never before the wait: see the join and the received weight)
    if (a.q_start != nullptr)
        for (int head = blockIdx.x; head < a.hkv; head += gridDim.x) attn_uncovered<T, D>(a, head);
    unsigned run;
    const Place4 at = find_run4(p, Geo::ROWS, blockIdx.x, run);
    unsigned f = run * blockIdx.x, before = at.before;
    const unsigned stop = min(f + run, at.total);
    for (int b = at.b; f < stop && b < a.B; ++b) {
        const Share4 s(a, b, Geo::ROWS, p.grain);
        const unsigned cost = s.cost(a.hkv);
        while (f < stop && f - before < cost) {
            const unsigned unit = (f - before) / s.grains, start = before + unit * s.grains;
            Segment4 u;
            u.token0 = s.token0;
            u.count = s.count;
            u.keys = s.keys;
            u.table = a.page_table + static_cast<int64_t>(b) * a.table_width;
            u.head = static_cast<int>(unit / s.row_tiles);
            u.row0 = static_cast<int>(unit - u.head * s.row_tiles) * Geo::ROWS;
            const unsigned g0 = f - start, g1 = min(stop - start, s.grains);
            u.tile0 = static_cast<int>(g0 << p.grain);
            u.tile1 = static_cast<int>(g1 << p.grain);
            // a unit that began in an earlier run leaves its part in this one's first place, one that goes on in its second
            u.slot = g0 > 0 ? 2ll * blockIdx.x : g1 < s.grains ? 2ll * blockIdx.x + 1 : -1;
            u.scores = p.scores == nullptr ? nullptr : p.scores + (static_cast<int64_t>(b) * a.hkv + u.head) * (static_cast<int64_t>(a.table_width) << a.page_shift) * p.part_rows;
            attn4_segment<T, D, NR, E>(p, u, ring, smem4);
            __syncwarp();
            f = start + g1;
        }
        before += cost;
    }
}

// Joins the parts of the rows whose unit lies in several runs: out = sum_s exp(m_s - m) o_s / sum_s exp(m_s - m) l_s.  One warp per row,
// lanes over the channels.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attn4_join_kernel(const Attn4Params p, int unit_rows) {
    // This kernel starts once every block of the attention is past its wait, so whatever came before the attention has ended: the call's inputs (lengths,
    // offsets) may be read before this one's wait, the parts may not.
    grid_launch_dependents();
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    // where the row's parts lie follows from the call's inputs alone: found before the parts are there
    int64_t w0 = 0;
    int parts = 1, local = 0, rt = 0;
    if (row < a.T * a.hq) {
        const int64_t t = row / a.hq;
        const int h = static_cast<int>(row - t * a.hq), head = h / a.group;
        const int b = attn_sequence_of(a, t);
        const Share4 s(a, b, unit_rows, p.grain);
        unsigned total = 0, before = 0;
#pragma unroll 4
        for (int i = lane; i < a.B; i += 32) {
            const unsigned c = Share4(a, i, unit_rows, p.grain).cost(a.hkv);
            total += c;
            before += i < b ? c : 0;
        }
        total = __reduce_add_sync(kFullMask, total);
        before = __reduce_add_sync(kFullMask, before);
        if (t >= s.token0 && t < s.token0 + s.count) {  // (else a token of no sequence)
            local = static_cast<int>(t - s.token0) * a.group + (h - head * a.group);
            rt = local / unit_rows;
            const unsigned run = run4_grains(total, p.warps, p.least), start = before + (head * s.row_tiles + rt) * s.grains;
            w0 = start / run;
            parts = static_cast<int>((start + s.grains - 1) / run - w0) + 1;
            if (w0 + parts > p.warps) parts = 1;       // (offsets that make no sense)
        }
    }
    grid_dependency_wait();
    if (parts == 1) return;
    const int at = local - rt * unit_rows;
    auto slot = [&](int i) { return (2 * (w0 + i) + (i == 0 ? 1 : 0)) * p.part_rows + at; };
    float m = -INFINITY;
    for (int i = lane; i < parts; i += 32) m = fmaxf(m, a.part_ml[slot(i)].x);
#pragma unroll
    for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(kFullMask, m, i));
    const float z = m == -INFINITY ? 0.0f : m;
    constexpr int PER = 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.0f;
    for (int s0 = 0; s0 < parts; s0 += 32) {
        float2 mine = make_float2(-INFINITY, 0.0f);
        if (s0 + lane < parts) mine = a.part_ml[slot(s0 + lane)];
        const float f = exp2_fast(mine.x - z);
        l += f * mine.y;
        const int n = min(32, parts - s0);
        for (int s1 = 0; s1 < n; s1 += 8) {
            float4 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s1 + i < n && lane * PER < D) x[i] = *reinterpret_cast<const float4*>(a.part_o + slot(s0 + s1 + i) * D + lane * PER);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = __shfl_sync(kFullMask, f, s1 + i);
                acc.x += w * x[i].x; acc.y += w * x[i].y; acc.z += w * x[i].z; acc.w += w * x[i].w;
            }
        }
    }
#pragma unroll
    for (int i = 16; i; i >>= 1) l += __shfl_xor_sync(kFullMask, l, i);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (lane * PER < D) {
        T* dst = static_cast<T*>(a.out) + row * D + lane * PER;
        if constexpr (std::is_same<T, float>::value)
            *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
        else
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
    if (lane == 0 && p.lse) p.lse[row] = l > 0.0f || l != l ? m + log2f(l) : INFINITY;
}

// ---- the weight that each key receives: weights_out = weights + sum over the sequence's tokens and the group's heads of exp(score - lse).
// Sequences of up to eight rows a key head: the attention has left the scores, four bytes a row and key; to take them again from the
// codes costs D / 2 + 8 bytes a key and the products (32 x up to 8192 keys of 8 key heads, 4 rows: 48 us against 12).
// Four keys a thread.
__global__ static void __launch_bounds__(256)
attn4_weigh_scores_kernel(const Attn4Params p, int chunks) {
    const AttnParams& a = p.a;
    const int chunk = static_cast<int>(blockIdx.x % chunks);
    const int head = static_cast<int>((blockIdx.x / chunks) % a.hkv), b = static_cast<int>(blockIdx.x / chunks / a.hkv);
    const int64_t width = static_cast<int64_t>(a.table_width) << a.page_shift;
    const int64_t key0 = static_cast<int64_t>(chunk) * 1024 + 4 * threadIdx.x, at = (static_cast<int64_t>(b) * a.hkv + head) * width + key0;
    int64_t token0;
    int count;
    attn_tokens(a, b, token0, count);
    const int keys = attn_length(a, b), rows = count * a.group;
    const bool there = key0 < keys;
    // (lengths, offsets and what has been received so far are read before the wait: this kernel starts after the attention's blocks are past theirs, hence after
    // whatever wrote them has ended)
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (there && p.weights != nullptr) v = *reinterpret_cast<const float4*>(p.weights + at);
    grid_dependency_wait();                                          // scores and sums come from the kernels before
    if (key0 >= width) return;
    if (there) {
        const float* score = p.scores + (at - key0 % kTileKeys) * p.part_rows + key0 % kTileKeys;
        float4 add = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int row = 0; row < rows; ++row) {
            const int tok = row / a.group;
            const float lse = __ldcg(p.lse + (token0 + tok) * a.hq + static_cast<int64_t>(head) * a.group + (row - tok * a.group));
            const float4 x = __ldcg(reinterpret_cast<const float4*>(score + row * kTileKeys));
            const int64_t limit = static_cast<int64_t>(keys) - count + tok + 1 - key0;     // of these keys, those that the row sees
            if (limit > 0) add.x += exp2_fast(x.x - lse);
            if (limit > 1) add.y += exp2_fast(x.y - lse);
            if (limit > 2) add.z += exp2_fast(x.z - lse);
            if (limit > 3) add.w += exp2_fast(x.w - lse);
        }
        const int64_t here = keys - key0;
        v = make_float4(v.x + add.x, here > 1 ? v.y + add.y : 0.0f, here > 2 ? v.z + add.z : 0.0f, here > 3 ? v.w + add.w : 0.0f);
    }
    *reinterpret_cast<float4*>(p.weights_out + at) = v;
}

// More rows, or more scores than there should be memory for:
// A warp takes chunk_tiles (kWeightTiles at most) tiles of one sequence and key head and goes through all rows that read them; one owner per key, so the sum has
// one order.  Places from the sequence's length on become 0.
constexpr int kWeightTiles = 32;

template <typename T, int D, int NR>
struct Weigh4Geo {
    static constexpr int STAGE = 8 * D + 128;                        // codes of the keys, then (step, lo)
    static constexpr int STAGES = 4;
    static constexpr int OFF_SUMS = STAGES * STAGE;
    static constexpr int OFF_BARS = OFF_SUMS + kWeightTiles * kTileKeys * 4;
    static constexpr int BYTES = OFF_BARS + STAGES * 8;
};

template <typename T, int D, int NR>
__global__ void __launch_bounds__(32, 16)
attn4_weigh_kernel(const Attn4Params p, int chunk_tiles, int chunks) {
    using Geo = Weigh4Geo<T, D, NR>;
    constexpr int STAGES = Geo::STAGES;
    extern __shared__ __align__(128) unsigned char smem4[];
    const AttnParams& a = p.a;
    const int lane = threadIdx.x, r4 = lane >> 2, c4 = lane & 3;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem4 + Geo::OFF_BARS);
    float* sums = reinterpret_cast<float*>(smem4 + Geo::OFF_SUMS);
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(full + s, 1);
        fence_mbar_init();
    }
    const int chunk = static_cast<int>(blockIdx.x % chunks);
    const int head = static_cast<int>((blockIdx.x / chunks) % a.hkv), b = static_cast<int>(blockIdx.x / chunks / a.hkv);
    const int width = a.table_width << a.page_shift;
    const int chunk_keys = chunk_tiles * kTileKeys, key0 = chunk * chunk_keys;
    const int64_t at = (static_cast<int64_t>(b) * a.hkv + head) * width;
    for (int i = lane; i < chunk_keys; i += 32) sums[i] = 0.0f;
    __syncwarp();
    grid_dependency_wait();                                          // the rows' sums come from the kernels before
    int64_t token0;
    int count;
    attn_tokens(a, b, token0, count);
    const int keys = attn_length(a, b), first_limit = keys - count + 1;
    const int32_t* table = a.page_table + static_cast<int64_t>(b) * a.table_width;
    const int rows = count * a.group;
    const int here = max(0, min(keys - key0, chunk_keys));             // keys of this chunk (its end may pass 31 bits)
    const int tiles = (here + kTileKeys - 1) / kTileKeys;
    const int tile_no = tiles4_of(a, table, head, key0 / kTileKeys, key0 / kTileKeys + tiles);
    unsigned taken = 0;
    auto ask = [&](unsigned s, int tile) {
        const unsigned char* src = p.cache + static_cast<int64_t>(tile) * tile4_bytes(D);
        mbar_expect_tx(full + s, Geo::STAGE);
        bulk_load(smem4 + s * Geo::STAGE, src, 8 * D, full + s);
        bulk_load(smem4 + s * Geo::STAGE + 8 * D, src + tile4_rows(D), 128, full + s);
    };
    for (int row0 = 0; row0 < rows; row0 += 8 * NR) {
        // rows that see nothing here are passed over: the last of these rows sees the most
        const int end = first_limit + (min(rows, row0 + 8 * NR) - 1) / a.group;
        const int n = min(tiles, max(0, (end - key0 + kTileKeys - 1) / kTileKeys));
        if (n == 0) continue;
#pragma unroll
        for (int j = 0; j < STAGES; ++j) {
            const int tile = __shfl_sync(kFullMask, tile_no, j);
            if (lane == 0 && j < n) ask((taken + j) % STAGES, tile);
        }
        Rows4<T, D, NR, 2> rw;
        rw.load(a, token0, head, row0, rows, nullptr);
        int limit[NR][2];
        float lse[NR][2];
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = row0 + i * 8 + 2 * c4 + e, tok = row / a.group;
                limit[i][e] = row < rows ? first_limit + tok : 0;    // (rows that are not there weigh nothing)
                lse[i][e] = row < rows ? __ldcg(p.lse + (token0 + tok) * a.hq + static_cast<int64_t>(head) * a.group + (row - tok * a.group)) : INFINITY;
            }
        for (int j = 0; j < n; ++j, ++taken) {
            const unsigned stage = taken % STAGES;
            mbar_wait_bounded(full + stage, (taken / STAGES) & 1u);
            const unsigned char* tile = smem4 + stage * Geo::STAGE;
            float s[NR][4];
            scores4<T, D, NR, 2>(rw, tile, nullptr, s);
            Params4 w;
            w.load(tile + 8 * D);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int key = key0 + j * kTileKeys + 8 * k + r4;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float z = fmaf(step4_of(w.key(k)) * s[i][2 * k + e], rw.factor[i][e], fmaf(base4_of<T>(w.key(k)), rw.sum[i][e], -lse[i][e]));
                        if (key < limit[i][e]) sum += exp2_fast(z);
                    }
                sum = quad_sum(sum);
                if (c4 == 0) sums[j * kTileKeys + 8 * k + r4] += sum;
            }
            __syncwarp();
            const int tile_next = __shfl_sync(kFullMask, tile_no, (j + STAGES) & 31);
            if (lane == 0 && j + STAGES < n) ask(stage, tile_next);
        }
    }
    __syncwarp();
    const int stop = min(width - key0, chunk_keys);
    for (int i = lane * 4; i < stop; i += 128) {                     // (a page holds whole tiles: widths are multiples of 16)
        float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p.weights && i < here) old = *reinterpret_cast<const float4*>(p.weights + at + key0 + i);
        const float4 add = *reinterpret_cast<const float4*>(sums + i);
        float4 v = make_float4(old.x + add.x, old.y + add.y, old.z + add.z, old.w + add.w);
        if (i >= here) v.x = 0.0f;
        if (i + 1 >= here) v.y = 0.0f;
        if (i + 2 >= here) v.z = 0.0f;
        if (i + 3 >= here) v.w = 0.0f;
        *reinterpret_cast<float4*>(p.weights_out + at + key0 + i) = v;
    }
}

}  // namespace wht

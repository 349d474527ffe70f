// Attention over the cache held in 4 bits, by warp-level matrix products on the codes themselves.
//
//     k_j = lo_j + step_j c_j,   v_j = lo'_j + step'_j c'_j      (codes c, c' whole numbers 0 .. 15)
//     score_j = scale (step_j (q . c_j) + lo_j sum(q))
//     o = sum_j p_j v_j / sum_j p_j = (sum_j (p_j step'_j) c'_j + sum_j p_j lo'_j) / sum_j p_j,   p_j = exp(score_j - m)
//
// in one pass over the keys.  The codes are never turned into values: a half word of codes masked with 0x000f or 0x00f0 IS an fp16
// number, c 2^-24 or 16 c 2^-24 (a subnormal one; the tensor core takes these as they are, but aligns a product by its operands'
// exponents, so that sums keep about 20 bits), so that eight codes take four masks and one shift, exactly, and the powers of two go into the
// queries and the result.  For fp32 results the values' codes become ordinary numbers, c - 8, by one exact subtraction a pair.
// Queries enter as fp16 after a shift of each row by a power of two (bf16 ones keep all their bits but what lies below 2^-35 of the row's
// maximum; fp32 ones are two terms, 22 bits of it), and the weights p step' as fp16 times a power of two per row that keeps them in range: one
// term of 11 bits where the output is rounded to 8, two where it is fp32.
//
// What bounds it: memory, 2 (D / 2 + 4) bytes a key and key head.  At 23 B a clock and SM a tile of 16 keys of 128 channels has 378 clocks of an SM's
// quarter; its 170 mask, select and shift instructions take two clocks each.
// Hence products with the rows on the 16-row operand: the weights leave the first product in the layout in which the second wants
// them; codes of keys and of values are the 8-column operand.
//
// The division of work goes by the lengths themselves, which are on the device: the tiles of all units (sequence, key head, row tile)
// are counted one after the other, and each warp (a block of its own) takes an equal run of them, whatever units it touches.  A unit that lies in one
// run is finished there; the parts of the others are joined by a second kernel, in the order of the keys.
#pragma once
#include <cuda_fp16.h>

#include "cache4_common.cuh"

namespace wht {

struct Attn4Params {
    AttnParams a;            // queries, output, tables, lengths, sizes; part_ml, part_o: [2 * warps][rows of a unit]
    const unsigned char* cache;
    int warps;               // runs
    int least;               // tiles of a run, at least
    float* lse;              // [T * Hq] log2 of a row's softmax sum, or NULL
    const float* weights;    // [B x Hkv x table_width * page]: received so far
    float* weights_out;
};

// HR: rows of a lane.  1: a 16-row operand holds 8 rows, the upper half being their second terms (fp32) or nothing.  2: 16 rows.
// NT: 16-row operands of a unit.
template <typename T, int D, int HR, int NT>
struct Attn4Geo {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static_assert(!F32 || HR == 1, "fp32 queries are two terms");
    static constexpr int NG = D / 32;
    static constexpr int ROWS = 8 * HR * NT;
    static constexpr int TILE = tile4_bytes(D);
    static constexpr int STAGES = 4;
    static constexpr bool Q_SHARED = NT > 1;                    // query operands in shared memory
    static constexpr int Q_BYTES = Q_SHARED ? NT * 2 * NG * 512 : 0;
    static constexpr int OFF_Q = STAGES * TILE;
    static constexpr int OFF_BARS = OFF_Q + Q_BYTES;
    static constexpr int BYTES = OFF_BARS + STAGES * 8;
    static constexpr int BLOCKS = NT > 1 ? 8 : HR > 1 || F32 ? 12 : 16;  // on an SM
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
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(kFullMask, x, 1);
    return x + __shfl_xor_sync(kFullMask, x, 2);
}

// A row of queries: this lane's channels 32 g + 8 c4 .. + 7 as operands of the steps 2 g and 2 g + 1; a[g][step][0]: contraction indices
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
                load8(src + g * 32 + c4 * 8, v[g]);
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
        const int e = top > 0.0f ? max(exponent_of(top) - 13, -100) : 0;  // the largest becomes 2^13 and up to 2^14
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

// The rows of a unit as the products take them, and what belongs to each.
template <typename T, int D, int HR, int NT>
struct Rows4 {
    using Geo = Attn4Geo<T, D, HR, NT>;
    uint32_t q[Geo::Q_SHARED ? 1 : NT][Geo::NG][2][4];
    float factor[NT][HR], sum[NT][HR];
    float first[NT][2];                                              // (fp32) what the products of the two terms begin with
    __device__ __forceinline__ void load(const AttnParams& p, int64_t token0, int head, int row0, int rows, unsigned char* smem) {
        const int lane = threadIdx.x & 31, r4 = lane >> 2;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint32_t f[Geo::NG][2][4];
#pragma unroll
            for (int h = 0; h < HR; ++h) {
                const int row = row0 + (n * HR + h) * 8 + r4, tok = row / p.group;
                const T* src = static_cast<const T*>(p.q) + (token0 + tok) * p.q_st +
                               (static_cast<int64_t>(head) * p.group + (row - tok * p.group)) * p.q_sh;
                Query4<T, Geo::NG> x;
                x.load(src, row < rows, p.scale_log2);
                factor[n][h] = x.factor;
                sum[n][h] = x.sum;
                first[n][0] = Geo::F32 ? x.lead0 : 0.0f;
                first[n][1] = Geo::F32 ? x.rest0 : 0.0f;
#pragma unroll
                for (int g = 0; g < Geo::NG; ++g)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            f[g][s][2 * i + h] = x.lead[g][s][i];
                            if (HR == 1) f[g][s][2 * i + 1] = x.rest[g][s][i];
                        }
            }
#pragma unroll
            for (int g = 0; g < Geo::NG; ++g)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if constexpr (Geo::Q_SHARED) {
                        *reinterpret_cast<uint4*>(smem + ((n * Geo::NG + g) * 2 + s) * 512 + lane * 16) =
                            make_uint4(f[g][s][0], f[g][s][1], f[g][s][2], f[g][s][3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) q[n][g][s][i] = f[g][s][i];
                    }
                }
        }
    }
    __device__ __forceinline__ void get(int n, int g, int s, const unsigned char* smem, uint32_t (&f)[4]) const {
        if constexpr (Geo::Q_SHARED) {
            const uint4 w = *reinterpret_cast<const uint4*>(smem + ((n * Geo::NG + g) * 2 + s) * 512 + (threadIdx.x & 31) * 16);
            f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = q[n][g][s][i];
        }
    }
};

// One row against the keys 2 c4, 2 c4 + 1, 8 + 2 c4, 9 + 2 c4 of a tile: log2 scores.
struct Params4 {
    uint4 lower, upper;      // (step, lo) of key and value, of the keys 2 c4 and 2 c4 + 1, of 8 + 2 c4 and 9 + 2 c4
    __device__ __forceinline__ void load(const unsigned char* tile, int rows_at) {
        const int c4 = threadIdx.x & 3;
        lower = *reinterpret_cast<const uint4*>(tile + rows_at + c4 * 16);
        upper = *reinterpret_cast<const uint4*>(tile + rows_at + 64 + c4 * 16);
    }
    __device__ __forceinline__ uint32_t key(int j) const { return j == 0 ? lower.x : j == 1 ? lower.z : j == 2 ? upper.x : upper.z; }
    __device__ __forceinline__ uint32_t value(int j) const { return j == 0 ? lower.y : j == 1 ? lower.w : j == 2 ? upper.y : upper.w; }
};

// S = Q C^T of a tile: s[n][t][e], e < 2 rows r4, keys 8 t + 2 c4 + e, e >= 2 the upper half of the operand (fp32: added to the lower).
// fp32 rows: the tensor core's accumulation truncates to about 24 bits of the largest product.  The first term of a query is therefore a
// whole number of eighths of 2^-10 of the row's range: products with codes and sums of 128 of them take 22 bits, so nothing is lost.
template <typename T, int D, int HR, int NT>
__device__ __forceinline__ void scores4(const Rows4<T, D, HR, NT>& rows, const unsigned char* tile, const unsigned char* q_smem,
                                        float (&s)[NT][2][4]) {
    constexpr int NG = D / 32;
    constexpr bool F32 = std::is_same<T, float>::value;
    const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
    uint32_t w[2][NG];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const unsigned char* at = tile + (r4 + 8 * t) * (D / 2) + c4 * (D / 8);
        if constexpr (NG == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(at);
            w[t][0] = x.x; w[t][1] = x.y; w[t][2] = x.z; w[t][3] = x.w;
        } else if constexpr (NG == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            w[t][0] = x.x; w[t][1] = x.y;
        } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) w[t][g] = reinterpret_cast<const uint32_t*>(at)[g];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[n][t][0] = s[n][t][1] = F32 ? rows.first[n][0] : 0.0f;
            s[n][t][2] = s[n][t][3] = F32 ? rows.first[n][1] : 0.0f;
        }
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            uint32_t b[2][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t x = st ? w[t][g] >> 8 : w[t][g];
                b[t][0] = x & 0x000f000fu;
                b[t][1] = x & 0x00f000f0u;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t a[4];
                rows.get(n, g, st, q_smem, a);
#pragma unroll
                for (int t = 0; t < 2; ++t) mma_f16_16816(s[n][t], a, b[t][0], b[t][1]);
            }
        }
    if constexpr (F32) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) s[n][t][e] += s[n][t][2 + e];
    }
}

// A row's base: its least value; for fp32 what code 8 stands for, since lo and the sum of codes, all positive, are several times what they weigh
// together in the end.
template <typename T>
__device__ __forceinline__ float base4_of(unsigned word) {
    return std::is_same<T, float>::value ? fmaf(8.0f, step4_of(word), lo4_of(word)) : lo4_of(word);
}

// The tiles of one unit in one run.
struct Segment4 {
    int64_t token0;          // first token of the sequence
    int count, keys;         // its tokens in this call, its keys
    const int32_t* table;    // its pages
    int head, row0;          // key head, first row of the unit: row r is token r / group, query head head * group + r % group
    int tile0, tile1;        // of the unit's tiles
    int64_t slot;            // where the part goes, or -1: the unit is finished here
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
    int pg = __ldg(table + (t >> shift));
    if (pg < 0 || pg >= p.num_pages) {
        attn_report(kAttnErrIndex);
        pg = 0;
    }
    return ((pg * p.hkv + head) << shift) + (t & ((1 << shift) - 1));
}

template <typename T, int D, int HR, int NT>
__device__ __forceinline__ void attn4_segment(const Attn4Params& p, const Segment4& u, Ring4& ring, unsigned char* smem) {
    using Geo = Attn4Geo<T, D, HR, NT>;
    constexpr bool F32 = Geo::F32;
    constexpr int NG = Geo::NG, STAGES = Geo::STAGES;
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31, r4 = lane >> 2, c4 = lane & 3;
    const int rows = u.count * a.group;
    // the unit's last row sees the most keys, its first row the fewest
    const int last_row = min(rows, u.row0 + Geo::ROWS) - 1;
    const int first_limit = u.keys - u.count + 1;                    // keys that the sequence's first token sees
    const int end = min(u.tile1 * kTileKeys, first_limit + last_row / a.group);
    const int least_limit = first_limit + u.row0 / a.group;
    const int tiles = max(0, (end - u.tile0 * kTileKeys + kTileKeys - 1) / kTileKeys);

    int now = tiles4_of(a, u.table, u.head, u.tile0, u.tile0 + tiles);
    int next = tiles > 32 ? tiles4_of(a, u.table, u.head, u.tile0 + 32, u.tile0 + tiles) : 0;
    auto ask = [&](int j, int tile) {                                // lane 0
        const unsigned s = (ring.taken + j) % STAGES;
        mbar_expect_tx(ring.full + s, Geo::TILE);
        bulk_load(ring.base + s * Geo::TILE, p.cache + static_cast<int64_t>(tile) * Geo::TILE, Geo::TILE, ring.full + s);
    };
#pragma unroll
    for (int j = 0; j < STAGES; ++j) {
        const int tile = __shfl_sync(kFullMask, now, j);
        if (lane == 0 && j < tiles) ask(j, tile);
    }
    unsigned char* q_smem = smem + Geo::OFF_Q;
    Rows4<T, D, HR, NT> rw;
    rw.load(a, u.token0, u.head, u.row0, rows, q_smem);
    if constexpr (Geo::Q_SHARED) __syncwarp();

    int limit[NT][HR];
    float m[NT][HR], l[NT][HR], r[NT][HR], most[NT][HR];             // most: the largest p step' so far, which sets the weights' range
    float range[NT][HR];                                             // weights enter times this power of two
    float o[NT][4 * NG][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int h = 0; h < HR; ++h) {
            const int row = u.row0 + (n * HR + h) * 8 + r4;
            limit[n][h] = row < rows ? first_limit + row / a.group : 0x7fffffff;   // (rows that are not there see zeros)
            m[n][h] = -INFINITY;
            l[n][h] = r[n][h] = most[n][h] = 0.0f;
            range[n][h] = 1.0f;
        }
#pragma unroll
        for (int d = 0; d < 4 * NG; ++d) o[n][d][0] = o[n][d][1] = o[n][d][2] = o[n][d][3] = 0.0f;
    }

    for (int j = 0; j < tiles; ++j) {
        const unsigned stage = ring.taken % STAGES;
        mbar_wait_bounded(ring.full + stage, (ring.taken / STAGES) & 1u);
        const unsigned char* tile = ring.base + stage * Geo::TILE;
        const int base = (u.tile0 + j) * kTileKeys;
        const bool mask = base + kTileKeys > least_limit;

        float s[NT][2][4];
        scores4<T, D, HR, NT>(rw, tile, q_smem, s);
        Params4 w;
        w.load(tile, tile4_rows(D));
        // log2 scores, weights, and weights times the values' steps, of the keys 2 c4, 2 c4 + 1, 8 + 2 c4, 9 + 2 c4
        float x[NT][HR][4], y[NT][HR][4];
        bool passes = false;
        auto hidden = [&](int n, int h, int i) { return mask && base + 8 * (i >> 1) + 2 * c4 + (i & 1) >= limit[n][h]; };
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < HR; ++h) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[n][h][i] = fmaf(step4_of(w.key(i)) * s[n][i >> 1][(i & 1) + 2 * h], rw.factor[n][h], base4_of<T>(w.key(i)) * rw.sum[n][h]);
                    float weight = exp2_fast(x[n][h][i] - m[n][h]);
                    y[n][h][i] = weight * step4_of(w.value(i)) * range[n][h];
                    if (hidden(n, h, i)) weight = y[n][h][i] = 0.0f;
                    passes = passes || !(weight <= 256.0f) || !(y[n][h][i] <= 16384.0f);
                    s[n][i >> 1][(i & 1) + 2 * (HR - 1) * h] = weight;   // (the scores of this key are done with)
                }
            }
        if (__any_sync(kFullMask, passes)) {
            // a new maximum, or weights that leave the range of fp16: the references move
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < HR; ++h) {
                    // (a row moves its references by its own scores alone: its result does not depend on the rows beside it)
                    float top = -INFINITY;
                    int moves = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (!hidden(n, h, i)) top = fmaxf(top, x[n][h][i]);
                        moves |= !(s[n][i >> 1][(i & 1) + 2 * (HR - 1) * h] <= 256.0f) || !(y[n][h][i] <= 16384.0f);
                    }
                    moves |= __shfl_xor_sync(kFullMask, moves, 1);
                    moves |= __shfl_xor_sync(kFullMask, moves, 2);
                    top = fmaxf(quad_max(top), m[n][h]);
                    if (!__any_sync(kFullMask, moves)) continue;
                    if (!moves) top = m[n][h];
                    const float f = top > m[n][h] ? exp2_fast(m[n][h] - top) : 1.0f;
                    m[n][h] = top;
                    l[n][h] *= f;
                    r[n][h] *= f;
                    float heavy = 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float weight = hidden(n, h, i) ? 0.0f : exp2_fast(x[n][h][i] - top);
                        if (moves) s[n][i >> 1][(i & 1) + 2 * (HR - 1) * h] = weight;
                        heavy = fmaxf(heavy, hidden(n, h, i) ? 0.0f : weight * step4_of(w.value(i)));
                    }
                    heavy = fmaxf(quad_max(heavy), most[n][h] * f);
                    if (!moves) heavy = most[n][h];
                    most[n][h] = heavy;
                    // the largest becomes 2^6: 2^8 above it before the range moves, 2^-31 of it below before bits are lost
                    const int to = heavy > 0.0f ? max(-120, min(120, 6 - exponent_of(heavy))) : 100;
                    const int by = to - exponent_of(range[n][h]);
                    range[n][h] = power_of_two(to);
                    const float f1 = f * power_of_two(by / 2), f2 = power_of_two(by - by / 2);
#pragma unroll
                    for (int d = 0; d < 4 * NG; ++d)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            o[n][d][e + 2 * (HR - 1) * h] = o[n][d][e + 2 * (HR - 1) * h] * f1 * f2;
                            if (HR == 1) o[n][d][e + 2] = o[n][d][e + 2] * f1 * f2;
                        }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[n][h][i] = hidden(n, h, i) ? 0.0f : s[n][i >> 1][(i & 1) + 2 * (HR - 1) * h] * step4_of(w.value(i)) * range[n][h];
                }
        }
        uint32_t pa[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < HR; ++h) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float weight = s[n][i >> 1][(i & 1) + 2 * (HR - 1) * h];
                    l[n][h] += weight;
                    if (!hidden(n, h, i)) r[n][h] = fmaf(weight, base4_of<T>(w.value(i)), r[n][h]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t lead = pack_half2(y[n][h][2 * i], y[n][h][2 * i + 1]);
                    pa[n][2 * i + h] = lead;
                    if (HR == 1) pa[n][2 * i + 1] = F32 ? pack_half2(y[n][h][2 * i] - half_lo(lead), y[n][h][2 * i + 1] - half_hi(lead)) : 0u;
                }
            }

        // O += (P step') C': this lane's codes of the keys 2 c4, 2 c4 + 1, 8 + 2 c4, 9 + 2 c4, halves u = r4
        const unsigned char* vt = tile + 8 * D;
        uint32_t pair[NG][2];
        if constexpr (NG == 4) {
            uint2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint2*>(vt + (c4 + 4 * i) * 64 + ((r4 ^ ((c4 & 2) << 1)) << 3));
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
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t*>(vt + (c4 + 4 * i) * 32 + r4 * 4);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                pair[0][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x5410);
                pair[1][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x7632);
            }
            if constexpr (NG == 3) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const unsigned short*>(vt + 512 + (c4 + 4 * i) * 16 + r4 * 2);
#pragma unroll
                for (int i = 0; i < 2; ++i) pair[2][i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x5410);
            }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t pick = i & 1 ? 0x00f000f0u : 0x000f000fu;
                uint32_t b0 = (i >= 2 ? pair[g][0] >> 8 : pair[g][0]) & pick, b1 = (i >= 2 ? pair[g][1] >> 8 : pair[g][1]) & pick;
                if (F32) {                                           // code - 8, exactly, as ordinary numbers
                    b0 = minus_half2(b0 | 0x64006400u, i & 1 ? 0x64806480u : 0x64086408u);
                    b1 = minus_half2(b1 | 0x64006400u, i & 1 ? 0x64806480u : 0x64086408u);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (F32) {
                        // (the tensor core's accumulation truncates: one tile at a time, added up with rounding)
                        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_f16_16816(sum, pa[n], b0, b1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][4 * g + i][e] += sum[e];
                    } else {
                        mma_f16_16816(o[n][4 * g + i], pa[n], b0, b1);
                    }
                }
            }
        __syncwarp();                                                // every lane has read the slot
        const int ahead = j + STAGES;
        if ((ahead & 31) == 0) {
            now = next;
            next = ahead + 32 < tiles ? tiles4_of(a, u.table, u.head, u.tile0 + ahead + 32, u.tile0 + tiles) : 0;
        }
        const int t = __shfl_sync(kFullMask, now, ahead & 31);
        if (lane == 0 && ahead < tiles) ask(STAGES, t);
        ++ring.taken;
    }

    // the results, eight channels of a row at a time
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < HR; ++h) {
            const int local = (n * HR + h) * 8 + r4, row = u.row0 + local, tok = row / a.group;
            const float ll = quad_sum(l[n][h]), rr = quad_sum(r[n][h]);
            if (row >= rows) continue;
            const float unit = power_of_two(-exponent_of(range[n][h]));
            const int64_t at = (u.token0 + tok) * a.hq + static_cast<int64_t>(u.head) * a.group + (row - tok * a.group);
            const float inv = u.slot >= 0 ? 1.0f : ll > 0.0f ? 1.0f / ll : 0.0f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float c = o[n][4 * g + i][e + 2 * (HR - 1) * h];
                        if (F32) c += o[n][4 * g + i][e + 2];
                        v[4 * e + i] = (c * (F32 ? (i & 1 ? 0.0625f : 1.0f) : i & 1 ? 1048576.0f : 16777216.0f) * unit + rr) * inv;
                    }
                if (u.slot >= 0) store8(a.part_o + (u.slot * Geo::ROWS + local) * D + g * 32 + c4 * 8, v);
                else store8(static_cast<T*>(a.out) + at * D + g * 32 + c4 * 8, v);
            }
            if (c4 != 0) continue;
            if (u.slot >= 0) a.part_ml[u.slot * Geo::ROWS + local] = make_float2(m[n][h], ll);
            else if (p.lse) p.lse[at] = ll > 0.0f || ll != ll ? m[n][h] + log2f(ll) : INFINITY;
        }
}

// ---- the division of the work

// Tiles of sequence b: units (key heads times row tiles) times tiles of its keys, one at least where it has tokens.
struct Share4 {
    int64_t token0;
    int count, keys, row_tiles, tiles;
    __device__ __forceinline__ Share4(const AttnParams& p, int b, int unit_rows) : token0(0), count(0), keys(0), row_tiles(0), tiles(1) {
        if (b >= p.B) return;
        attn_tokens(p, b, token0, count);
        if (count == 0) return;
        keys = attn_length(p, b);
        row_tiles = (count * p.group + unit_rows - 1) / unit_rows;
        tiles = max(1, (keys + kTileKeys - 1) / kTileKeys);
    }
    __device__ __forceinline__ int64_t cost(int hkv) const { return static_cast<int64_t>(hkv) * row_tiles * tiles; }
};

__device__ __forceinline__ int64_t warp_sum64(int64_t x) {
#pragma unroll
    for (int i = 16; i; i >>= 1) x += __shfl_xor_sync(kFullMask, x, i);
    return x;
}
// tiles of the sequences below `upto` (all lanes of a warp together)
__device__ __forceinline__ int64_t tiles4_before(const AttnParams& p, int upto, int unit_rows) {
    const int lane = threadIdx.x & 31;
    int64_t sum = 0;
    for (int b = lane; b < upto; b += 32) sum += Share4(p, b, unit_rows).cost(p.hkv);
    return warp_sum64(sum);
}
__device__ __forceinline__ int64_t run4_tiles(int64_t total, int warps, int least) {
    const int64_t even = (total + warps - 1) / warps;
    return even > least ? even : least;
}

template <typename T, int D, int HR, int NT>
__global__ void __launch_bounds__(32, (Attn4Geo<T, D, HR, NT>::BLOCKS))
attn4_kernel(const Attn4Params p) {
    using Geo = Attn4Geo<T, D, HR, NT>;
    extern __shared__ __align__(128) unsigned char smem4[];
    const AttnParams& a = p.a;
    const int lane = threadIdx.x;
    Ring4 ring{smem4, reinterpret_cast<uint64_t*>(smem4 + Geo::OFF_BARS), 0};
    if (lane == 0) {
        for (int s = 0; s < Geo::STAGES; ++s) mbar_init(ring.full + s, 1);
        fence_mbar_init();
    }
    __syncwarp();
    grid_launch_dependents();
    if (a.q_start != nullptr)
        for (int head = blockIdx.x; head < a.hkv; head += gridDim.x) attn_uncovered<T, D>(a, head);
    const int64_t total = tiles4_before(a, a.B, Geo::ROWS);
    const int64_t run = run4_tiles(total, p.warps, p.least);
    int64_t f = run * blockIdx.x;
    const int64_t stop = min(f + run, total);
    if (f >= stop) return;
    // the sequence in which the run begins
    int b = 0;
    int64_t before = 0;
    for (; b < a.B; b += 32) {
        int64_t upto = Share4(a, b + lane, Geo::ROWS).cost(a.hkv);
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            const int64_t x = __shfl_up_sync(kFullMask, upto, i);
            if (lane >= i) upto += x;
        }
        const unsigned past = __ballot_sync(kFullMask, before + upto > f);
        if (past) {
            const int at = __ffs(past) - 1;
            const int64_t skipped = __shfl_sync(kFullMask, upto, at > 0 ? at - 1 : 0);
            before += at > 0 ? skipped : 0;
            b += at;
            break;
        }
        before += __shfl_sync(kFullMask, upto, 31);
    }
    for (; f < stop && b < a.B; ++b) {
        const Share4 s(a, b, Geo::ROWS);
        const int64_t cost = s.cost(a.hkv);
        while (f < stop && f < before + cost) {
            const int64_t unit = (f - before) / s.tiles, start = before + unit * s.tiles;
            Segment4 u;
            u.token0 = s.token0;
            u.count = s.count;
            u.keys = s.keys;
            u.table = a.page_table + static_cast<int64_t>(b) * a.table_width;
            u.head = static_cast<int>(unit / s.row_tiles);
            u.row0 = static_cast<int>(unit - static_cast<int64_t>(u.head) * s.row_tiles) * Geo::ROWS;
            u.tile0 = static_cast<int>(f - start);
            u.tile1 = static_cast<int>(min(stop - start, static_cast<int64_t>(s.tiles)));
            // a unit that began in an earlier run leaves its part in this one's first place, one that goes on in its second
            u.slot = u.tile0 > 0 ? 2ll * blockIdx.x : u.tile1 < s.tiles ? 2ll * blockIdx.x + 1 : -1;
            attn4_segment<T, D, HR, NT>(p, u, ring, smem4);
            __syncwarp();
            f = start + u.tile1;
        }
        before += cost;
    }
}

// Joins the parts of the rows whose unit lies in several runs: out = sum_s exp(m_s - m) o_s / sum_s exp(m_s - m) l_s.  One warp per row,
// lanes over the channels.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attn4_join_kernel(const Attn4Params p, int unit_rows) {
    grid_dependency_wait();
    grid_launch_dependents();
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (row >= a.T * a.hq) return;
    const int64_t t = row / a.hq;
    const int h = static_cast<int>(row - t * a.hq), head = h / a.group;
    const int b = attn_sequence_of(a, t);
    const Share4 s(a, b, unit_rows);
    if (t < s.token0 || t >= s.token0 + s.count) return;             // a token of no sequence
    const int local = static_cast<int>(t - s.token0) * a.group + (h - head * a.group), rt = local / unit_rows;
    int64_t before = 0, total = 0;
    for (int i = lane; i < a.B; i += 32) {
        const int64_t c = Share4(a, i, unit_rows).cost(a.hkv);
        total += c;
        before += i < b ? c : 0;
    }
    before = warp_sum64(before);
    total = warp_sum64(total);
    const int64_t run = run4_tiles(total, p.warps, p.least);
    const int64_t start = before + (static_cast<int64_t>(head) * s.row_tiles + rt) * s.tiles;
    const int64_t w0 = start / run;
    const int parts = static_cast<int>((start + s.tiles - 1) / run - w0) + 1;
    if (parts == 1) return;
    const int at = local - rt * unit_rows;
    auto slot = [&](int i) { return ((2 * (w0 + i) + (i == 0 ? 1 : 0)) * unit_rows + at); };
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
// A warp takes kWeightTiles tiles of one sequence and key head and goes through all rows that read them; one owner per key, so the sum has
// one order.  Places from the sequence's length on become 0.
constexpr int kWeightTiles = 32;

template <typename T, int D, int HR>
struct Weigh4Geo : Attn4Geo<T, D, HR, 1> {
    static constexpr int STAGE = 8 * D + 128;                        // codes of the keys, then (step, lo)
    static constexpr int STAGES = 4;
    static constexpr int OFF_SUMS = STAGES * STAGE;
    static constexpr int OFF_BARS = OFF_SUMS + kWeightTiles * kTileKeys * 4;
    static constexpr int BYTES = OFF_BARS + STAGES * 8;
};

template <typename T, int D, int HR>
__global__ void __launch_bounds__(32, 16)
attn4_weigh_kernel(const Attn4Params p, int chunks) {
    using Geo = Weigh4Geo<T, D, HR>;
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
    const int key0 = chunk * kWeightTiles * kTileKeys;
    const int64_t at = (static_cast<int64_t>(b) * a.hkv + head) * width;
    for (int i = lane; i < kWeightTiles * kTileKeys; i += 32) sums[i] = 0.0f;
    __syncwarp();
    grid_dependency_wait();                                          // the rows' sums come from the kernels before
    int64_t token0;
    int count;
    attn_tokens(a, b, token0, count);
    const int keys = attn_length(a, b), first_limit = keys - count + 1;
    const int32_t* table = a.page_table + static_cast<int64_t>(b) * a.table_width;
    const int rows = count * a.group;
    const int here = max(0, min(keys, key0 + kWeightTiles * kTileKeys) - key0);      // keys of this chunk
    const int tiles = (here + kTileKeys - 1) / kTileKeys;
    const int tile_no = tiles4_of(a, table, head, key0 / kTileKeys, key0 / kTileKeys + tiles);
    unsigned taken = 0;
    auto ask = [&](unsigned s, int tile) {
        const unsigned char* src = p.cache + static_cast<int64_t>(tile) * tile4_bytes(D);
        mbar_expect_tx(full + s, Geo::STAGE);
        bulk_load(smem4 + s * Geo::STAGE, src, 8 * D, full + s);
        bulk_load(smem4 + s * Geo::STAGE + 8 * D, src + tile4_rows(D), 128, full + s);
    };
    for (int row0 = 0; row0 < rows; row0 += 8 * HR) {
        // rows that see nothing here are passed over: the last of these rows sees the most
        const int end = first_limit + (min(rows, row0 + 8 * HR) - 1) / a.group;
        const int n = min(tiles, max(0, (end - key0 + kTileKeys - 1) / kTileKeys));
        if (n == 0) continue;
#pragma unroll
        for (int j = 0; j < STAGES; ++j) {
            const int tile = __shfl_sync(kFullMask, tile_no, j);
            if (lane == 0 && j < n) ask((taken + j) % STAGES, tile);
        }
        Rows4<T, D, HR, 1> rw;
        rw.load(a, token0, head, row0, rows, nullptr);
        int limit[HR];
        float lse[HR];
#pragma unroll
        for (int h = 0; h < HR; ++h) {
            const int row = row0 + h * 8 + r4, tok = row / a.group;
            limit[h] = row < rows ? first_limit + tok : 0;           // (rows that are not there weigh nothing)
            lse[h] = row < rows ? __ldcg(p.lse + (token0 + tok) * a.hq + static_cast<int64_t>(head) * a.group + (row - tok * a.group)) : INFINITY;
        }
        for (int j = 0; j < n; ++j, ++taken) {
            const unsigned stage = taken % STAGES;
            mbar_wait_bounded(full + stage, (taken / STAGES) & 1u);
            const unsigned char* tile = smem4 + stage * Geo::STAGE;
            float s[1][2][4];
            scores4<T, D, HR, 1>(rw, tile, nullptr, s);
            Params4 w;
            w.load(tile, 8 * D);
            float sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = key0 + j * kTileKeys + 8 * (i >> 1) + 2 * c4 + (i & 1);
                sum[i] = 0.0f;
#pragma unroll
                for (int h = 0; h < HR; ++h) {
                    const float x = fmaf(step4_of(w.key(i)) * s[0][i >> 1][(i & 1) + 2 * h], rw.factor[0][h], base4_of<T>(w.key(i)) * rw.sum[0][h]);
                    if (key < limit[h]) sum[i] += exp2_fast(x - lse[h]);
                }
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum[i] += __shfl_xor_sync(kFullMask, sum[i], d);
            }
            if (r4 == 0) {
                float2* to = reinterpret_cast<float2*>(sums + j * kTileKeys + 2 * c4);
                float2 lower = to[0], upper = to[4];
                lower.x += sum[0]; lower.y += sum[1];
                upper.x += sum[2]; upper.y += sum[3];
                to[0] = lower;
                to[4] = upper;
            }
            __syncwarp();
            const int tile_next = __shfl_sync(kFullMask, tile_no, (j + STAGES) & 31);
            if (lane == 0 && j + STAGES < n) ask(stage, tile_next);
        }
    }
    __syncwarp();
    const int stop = min(width - key0, kWeightTiles * kTileKeys);
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

// Append to the cache held in 4 bits: rotation, quantisation, write; and the rows that the cache holds, read back.
// All inputs are read by ordinary loads, behind the wait for the kernel before, which may have written them.
//
//     q' = rotation(q)     row k' = rotation(k), row v: lo, step and codes (cache4_common.cuh)
//
// A pass over memory: each element is read once; queries are written as they came, keys and values in a quarter of the bytes or less.
// Bounded by it too: 16384 tokens of 32 query heads and 8 key heads of 128 in 73 us, 5.8 TB/s.
// Blocks take either queries or keys and values, whose arithmetic is several times as much.  Four lanes (D = 64) or eight own a row of keys or values, 16 channels each as two groups of eight, so
// that a rotation's pairs never cross lanes, the row's extremes take two or three shuffles, and each group of eight channels is one word of
// codes.  A thread takes the same channels of several heads, all loads in flight at once; they share the angles.
#pragma once
#include "cache4_common.cuh"
#include "kv_append_kernels.cuh"

namespace wht {

struct Append4Params {
    AppendParams a;          // k_cache, v_cache, summary unused; q_blocks, kv_blocks: groups of heads that a thread takes
    unsigned char* cache;
    int kv_grid;             // thread blocks of keys and values
};

// where the tile of a slot's row lies, and its place in the tile
__device__ __forceinline__ unsigned char* tile4_of(unsigned char* cache, int64_t slot, int head, int hkv, int page_shift, int d) {
    const int64_t page = slot >> page_shift;
    const int place = static_cast<int>(slot & ((1 << page_shift) - 1));
    return cache + (((page * hkv + head) << (page_shift - 4)) + (place >> 4)) * tile4_bytes(d);
}

template <typename T>
constexpr int kHeads4 = sizeof(T) == 4 ? 2 : 4;
constexpr int kAppend4Threads = 256, kAppend4Blocks = 3;  // on an SM (two, which the compiler's own choice of 84 registers leaves: 87 us for the prompts above)

// Queries: rotated and written; D / 16 lanes a row.
template <typename T, bool INTERLEAVED, int D>
__device__ __forceinline__ void append4_queries(const AppendParams& a, int64_t i) {
    constexpr int HB = kHeads4<T>, PER = D / 16;
    const int64_t job = i / PER, t = job / a.q_blocks;
    const RowItem<T, INTERLEAVED> it(static_cast<int>(i - job * PER), a.rot);
    if (t >= a.T) return;
    const int h0 = static_cast<int>(job - t * a.q_blocks) * HB, heads = a.hq - h0;
    const T* src = row_of<T>(a.q, t * a.q_st + h0 * a.q_sh);
    T* dst = row_of<T>(a.q_out, (t * a.hq + h0) * D);
    Raw8<T> lo[HB], hi[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        if (h < heads) {
            lo[h].load_written(src + h * a.q_sh + it.lo);
            hi[h].load_written(src + h * a.q_sh + it.hi);
        }
    }
    if (it.angle < 0) {
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            if (h < heads) {
                lo[h].store(dst + h * D + it.lo);
                hi[h].store(dst + h * D + it.hi);
            }
        }
        return;
    }
    const int pos = checked_position(a, append_position<true>(a, t));
    float c[8], s[8];
    load8_written(a.cos_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, c);
    load8_written(a.sin_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, s);
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        if (h < heads) {
            float x[8], y[8];
            lo[h].widen(x);
            hi[h].widen(y);
            it.turn(x, y, c, s);
            store8(dst + h * D + it.lo, x);
            store8(dst + h * D + it.hi, y);
        }
    }
}

template <typename T, bool INTERLEAVED, int D>
__global__ void __launch_bounds__(kAppend4Threads, kAppend4Blocks)
kv_append4_kernel(const Append4Params p) {
    constexpr int HB = kHeads4<T>;
    constexpr int LANES = D == 64 ? 4 : 8;             // of a row
    const AppendParams& a = p.a;
    grid_dependency_wait();
    grid_launch_dependents();
    // (blocks of rows compute where those of queries wait for memory: spread evenly among each other they share the SMs)
    const int64_t before = static_cast<int64_t>(blockIdx.x) * p.kv_grid / gridDim.x, after = static_cast<int64_t>(blockIdx.x + 1ll) * p.kv_grid / gridDim.x;
    if (after == before) {
        append4_queries<T, INTERLEAVED, D>(a, (blockIdx.x - before) * kAppend4Threads + threadIdx.x);
        return;
    }
    const int64_t job = (before * kAppend4Threads + threadIdx.x) / LANES;
    const int item = threadIdx.x % LANES;
    const int64_t t = job / (2 * a.kv_blocks);
    int group = static_cast<int>(job - t * 2 * a.kv_blocks);
    const bool is_k = group < a.kv_blocks;
    if (!is_k) group -= a.kv_blocks;
    const bool there = t < a.T && item < D / 16;       // (no lane leaves: rows fold by shuffles)
    const RowItem<T, INTERLEAVED> it(item < D / 16 ? item : 0, a.rot);
    const int64_t slot = there ? append_slot<true>(a, t) : -1;
    int pos = there && it.angle >= 0 ? append_position<true>(a, t) : 0;
    const int h0 = group * HB, heads = slot < 0 ? 0 : a.hkv - h0;
    const T* src = is_k ? row_of<T>(a.k, t * a.k_st + h0 * a.k_sh) : row_of<T>(a.v, t * a.v_st + h0 * a.v_sh);
    const int64_t step = is_k ? a.k_sh : a.v_sh;
    Raw8<T> lo[HB], hi[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i < heads) {
            lo[i].load_written(src + i * step + it.lo);
            hi[i].load_written(src + i * step + it.hi);
        }
    }
    const bool turns = is_k && slot >= 0 && it.angle >= 0;
    float c[8], s[8];
    if (turns) {
        pos = checked_position(a, pos);
        load8_written(a.cos_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, c);
        load8_written(a.sin_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, s);
    }
    const int place = static_cast<int>(slot & 15);
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (__all_sync(kFullMask, i >= heads)) continue;
        float x[8], y[8];
        float least = INFINITY, most = -INFINITY, nought = 0.0f;   // nought: NaN as soon as a channel is not finite
        const bool mine = i < heads;
        if (mine) {
            lo[i].widen(x);
            hi[i].widen(y);
            if (turns) it.turn(x, y, c, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                least = fminf(least, fminf(x[e], y[e]));
                most = fmaxf(most, fmaxf(x[e], y[e]));
                nought = fmaf(x[e], 0.0f, fmaf(y[e], 0.0f, nought));
            }
        }
#pragma unroll
        for (int n = 1; n < LANES; n <<= 1) {
            least = fminf(least, __shfl_xor_sync(kFullMask, least, n));
            most = fmaxf(most, __shfl_xor_sync(kFullMask, most, n));
            nought += __shfl_xor_sync(kFullMask, nought, n);
        }
        if (!mine) continue;
        const Hold4 hold(least, most, nought == 0.0f);
        unsigned char* tile = tile4_of(p.cache, slot, h0 + i, a.hkv, a.page_shift, D);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int channel = half ? it.hi : it.lo, g = channel >> 5, u = (channel >> 2) & 7;  // u even
            unsigned w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= hold.code(half ? y[e] : x[e]) << (4 * e);
            if (is_k) {
                *reinterpret_cast<unsigned*>(tile + key4_at(D, place, g, u)) = w;
            } else {
                *reinterpret_cast<unsigned short*>(tile + value4_at(D, place, g, u)) = static_cast<unsigned short>(w);
                *reinterpret_cast<unsigned short*>(tile + value4_at(D, place, g, u + 1)) = static_cast<unsigned short>(w >> 16);
            }
        }
        if (item == 0) *reinterpret_cast<unsigned*>(tile + tile4_rows(D) + place * 8 + (is_k ? 0 : 4)) = hold.word();
    }
}

struct Read4Params {
    const unsigned char* cache;
    const int64_t* slots;
    void *k, *v;             // [n x Hkv x D]
    int64_t n, num_slots;
    int hkv, page_shift;
};

// bf16(lo + step * code) of the eight codes of a word, two at a time.  A pair's codes go to the low bits of two bf16 numbers of 128 and above (the
// odd one times 8, with an eighth of the step), less 128, and one fused multiply-add with one rounding: the bf16 number next to lo + step * code.
// (fp32 arithmetic rounded to bf16 would lose a lo below 2^-24 of the product, whose up to 12 bits may lie half way between two bf16 numbers.)
__device__ __forceinline__ uint4 held4_bf16(unsigned word, unsigned row) {
    const unsigned turned = word >> 1, lo2 = __byte_perm(row, 0, 0x3232);
    const unsigned step2 = (row & 0xffffu) | (__float_as_uint(step4_of(row) * 0.125f) & 0xffff0000u);
    unsigned out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned two = (__byte_perm(word, turned, 0x0400 + 0x0101 * i) & 0x0078000fu) | 0x43004300u;
        asm("{ .reg .b32 c; sub.rn.bf16x2 c, %1, %2; fma.rn.bf16x2 %0, c, %3, %4; }" : "=r"(out[i]) : "r"(two), "r"(0x43004300u), "r"(step2), "r"(lo2));
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// A thread: eight channels of the keys and values of two heads at one slot, all loads in flight at once (four heads: 128 us for the rows below).
// Memory bounds it: 1048576 rows of 128 channels to bf16 122 us, 5.6 TB/s (with a shift, a mask, a subtraction, a product and a sum a
// channel 132).
constexpr int kReadHeads4 = 2;

template <typename T, int D>
__global__ void __launch_bounds__(256)
kv_read4_kernel(const Read4Params p) {
    constexpr int PER = D / 8, HB = kReadHeads4;
    grid_dependency_wait();                            // (slots and rows may come from the kernel before)
    grid_launch_dependents();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t job = i / PER;                       // slot number * groups of heads + group
    const int octet = static_cast<int>(i - job * PER), groups = (p.hkv + HB - 1) / HB;
    const int64_t at = job / groups;
    if (at >= p.n) return;
    const int h0 = static_cast<int>(job - at * groups) * HB;
    int64_t slot = p.slots[at];
    if (slot >= p.num_slots) {
        attn_report(kAttnErrIndex);
        slot = -1;
    }
    const int j = static_cast<int>(slot & 15), g = octet >> 2, u = 2 * (octet & 3);
    unsigned kw[HB], vw[HB];
    uint2 w[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        kw[h] = vw[h] = 0;
        w[h] = make_uint2(0, 0);
        if (slot < 0 || h0 + h >= p.hkv) continue;
        const unsigned char* tile = tile4_of(const_cast<unsigned char*>(p.cache), slot, h0 + h, p.hkv, p.page_shift, D);
        kw[h] = *reinterpret_cast<const unsigned*>(tile + key4_at(D, j, g, u));
        vw[h] = *reinterpret_cast<const unsigned short*>(tile + value4_at(D, j, g, u)) |
                static_cast<unsigned>(*reinterpret_cast<const unsigned short*>(tile + value4_at(D, j, g, u + 1))) << 16;
        w[h] = *reinterpret_cast<const uint2*>(tile + tile4_rows(D) + j * 8);
    }
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        if (h0 + h >= p.hkv) break;
        const int64_t row = (at * p.hkv + h0 + h) * D + octet * 8;
        if constexpr (std::is_same<T, float>::value) {
            const float ks = step4_of(w[h].x), kl = lo4_of(w[h].x), vs = step4_of(w[h].y), vl = lo4_of(w[h].y);
            float k[8], v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                k[e] = __fadd_rn(kl, __fmul_rn(ks, code4_value(kw[h], e)));
                v[e] = __fadd_rn(vl, __fmul_rn(vs, code4_value(vw[h], e)));
            }
            store8(static_cast<T*>(p.k) + row, k);
            store8(static_cast<T*>(p.v) + row, v);
        } else {
            *reinterpret_cast<uint4*>(static_cast<T*>(p.k) + row) = held4_bf16(kw[h], w[h].x);
            *reinterpret_cast<uint4*>(static_cast<T*>(p.v) + row) = held4_bf16(vw[h], w[h].y);
        }
    }
}

}  // namespace wht
